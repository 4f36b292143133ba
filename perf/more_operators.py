"""A KV cache held in 8 bits, as cases that can be timed and compared.

The stage's own cache holds bf16.  Three operators carry one of half the bytes, e4m3 codes with a float scale for each page
of 16 tokens, KV head and side (keys, values), for a serving loop whose lengths may stay on the device:

  step_maps         from the lengths of a step: the first row of each sequence, the position and the slot of each row, and
                    the block tables with the pages of new tokens, taken from a list of free ones
  norm_rope_store8  a layer's QKV projection: query and key heads normalised (where the model does that) and rotated, queries
                    returned in bf16, keys and values rounded to 8 bits into their slots, with the scales of their pages
  attention8        one layer's attention over the 8-bit cache, decode rows and prompt chunks in one call; optionally with a
                    sliding window and a few first tokens that stay visible

Head counts are those of the stage shapes ("tiny", "8b", "14b", "70b": query heads, KV heads, head dimension) and of generic
shapes beside them.  K pages are [slot / 4][d / 16][4 slots][16], V pages [d][16 slots].

All kinds describe a batch by
  decodes, lo, hi           sequences with one new token, cached lengths spread over [lo, hi] evenly in the logarithm
  chunks, rows, ragged      prompt chunks of `rows` new tokens (ragged: the first; the others 1 to `rows`)
  prefix                    chunk i continues a prompt of which prefix*i/(chunks-1) tokens are cached (one chunk: prefix)
"step_maps" and "norm_rope_store8" have `pad` rows behind the last sequence too, as a batch padded for a graph has;
"norm_rope_store8" has `norm` (whether heads are normalised) and `dtype` (of the projection), "attention8" `window` (0: none)
and `sinks`.
"""
import math
import random

import torch

own = False        # whether run() calls the framework's operators or computes their plain forms

DEV = "cuda:0"
PAGE = 16
TOP = 448.0                      # the largest e4m3 value
LEAST = 2.0 ** -100              # the smallest scale of a page
EPS = 1e-6
THETA = 500000.0
HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "14b": (40, 8, 128), "70b": (64, 8, 128),
         "g1_64": (8, 8, 64), "g16_128": (16, 1, 128), "g3_128": (12, 4, 128), "g7_64": (14, 2, 64)}


def _batch_of(decodes, lo, hi, chunks=0, rows=0, prefix=0, ragged=False):
    return dict(decodes=decodes, lo=lo, hi=hi, chunks=chunks, rows=rows, prefix=prefix, ragged=ragged)


def _maps(name, pad, batch):
    return dict(name=name, kind="step_maps", pad=pad, **batch)


def _store(name, heads, dtype, norm, pad, batch):
    return dict(name=name, kind="norm_rope_store8", heads=heads, dtype=dtype, norm=norm, pad=pad, **batch)


def _attention(name, heads, window, sinks, batch):
    return dict(name=name, kind="attention8", heads=heads, window=window, sinks=sinks, **batch)


def listed():
    return [
        # the decode-only step that throttling leaves when few requests are decoding; latency
        _maps("maps_decode_64", 0, _batch_of(64, 300, 20000)),
        # a full step of a busy server: chunks beside many decode rows, padded to the size of a captured graph
        _maps("maps_hybrid_512", 371, _batch_of(500, 64, 9000, 12, 700, 6000, True)),
        # the smallest call: the one-layer test shape without norms, three decode rows and a short chunk; latency
        _store("store_tiny_16", "tiny", "bf16", False, 0, _batch_of(3, 17, 64, 1, 13, 48)),
        # decode rows only, each adding one token to a page that holds others; latency
        _store("store_8b_decode_64", "8b", "f32", True, 0, _batch_of(64, 300, 20000)),
        # chunks that begin and end inside pages beside decode rows, with padding rows
        _store("store_14b_hybrid", "14b", "f32", True, 97, _batch_of(251, 64, 4096, 2, 901, 2011)),
        # the largest: two long prompt chunks, a stream through memory
        _store("store_70b_chunks_8192", "70b", "f32", True, 0, _batch_of(0, 0, 0, 2, 4096, 4096)),
        # the smallest call of attention: latency
        _attention("attn_tiny_16", "tiny", 0, 0, _batch_of(3, 17, 64, 1, 13, 48)),
        # chats of very different lengths, one new token each: a stream of keys
        _attention("attn_8b_decode_32", "8b", 0, 0, _batch_of(32, 300, 20000)),
        # long conversations of a model that sees the last 1024 tokens and four first ones
        _attention("attn_8b_window_decode_64", "8b", 1024, 4, _batch_of(64, 1000, 32000)),
        # the micro-batch that throttling aims at: chunks and decode rows together, five query heads per KV head
        _attention("attn_14b_hybrid_2053", "14b", 0, 0, _batch_of(251, 512, 4096, 2, 901, 2011)),
        # a whole odd prompt at once with a window
        _attention("attn_8b_window_chunk_8191", "8b", 2048, 16, _batch_of(0, 0, 0, 1, 8191, 0)),
        # the largest: a long chunk behind a long prefix, eight query heads per KV head, bound by the matrix cores
        _attention("attn_70b_chunk_4096", "70b", 0, 0, _batch_of(0, 0, 0, 1, 4096, 4096)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def _padded_scores(case):
    """Scores that a padded plain form holds at one time."""
    new, cached = _lengths(case)
    if case["kind"] != "attention8" or not new:
        return 0
    n_q = HEADS[case["heads"]][0]
    keys = max(c + n for n, c in zip(new, cached))
    return n_q * keys * max(case["decodes"] + 4, case["chunks"] * case["rows"])


def draw(rng):
    """One more case of the same ranges, no costlier than the costliest listed one of its kind."""
    while True:
        kind = rng.choice(("step_maps", "norm_rope_store8", "norm_rope_store8", "attention8", "attention8", "attention8", "attention8"))
        heads = rng.choice(tuple(HEADS))
        mix = rng.choice(("decodes", "chunks", "both"))
        hi = _log_int(rng, 1, 40000)
        most = {"step_maps": 800, "norm_rope_store8": 600, "attention8": 400}[kind]
        batch = _batch_of(_log_int(rng, 1, most) if mix != "chunks" else 0, max(0, int(hi * rng.uniform(0.0, 1.0))), hi,
                          _log_int(rng, 1, 12) if mix != "decodes" else 0, _log_int(rng, 1, 8192), rng.choice((0, _log_int(rng, 1, 16000))),
                          rng.random() < 0.5)
        if kind == "step_maps":
            c = _maps("", rng.choice((0, rng.randint(0, 300))), batch)
        elif kind == "norm_rope_store8":
            c = _store("", heads, rng.choice(("f32", "bf16")), rng.random() < 0.6, rng.choice((0, rng.randint(0, 300))), batch)
        else:
            window = rng.choice((0, 0, _log_int(rng, 1, 20000)))
            c = _attention("", heads, window, rng.choice((0, rng.randint(1, 70))) if window else 0, batch)
        del c["name"]
        like = [d for d in listed() if d["kind"] == kind]
        if _cost(c) <= max(_cost(d) for d in like) and _padded_scores(c) <= max(_padded_scores(d) for d in like):
            return c


# ---- batches ----------------------------------------------------------------------------------------------------------

def _lengths(case):
    """New and cached tokens of every sequence."""
    d, c, rows = case["decodes"], case["chunks"], case["rows"]
    lo, hi = max(1, case["lo"]), max(1, case["hi"])
    rng = random.Random(d * 8209 + c * 131 + rows)
    seqs = [(1, int(lo * (hi / lo) ** ((i + 0.5) / d))) for i in range(d)]
    seqs += [(rng.randint(1, rows) if case["ragged"] and i else rows, case["prefix"] * i // (c - 1) if c > 1 else case["prefix"]) for i in range(c)]
    rng.shuffle(seqs)
    return [n for n, _ in seqs], [x for _, x in seqs]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages(tokens):
    return -(-tokens // PAGE)


def _codes(gen, *shape):
    """Codes of values that fill the range of their page, as a store with its scales leaves them."""
    x = torch.empty(*shape, device=DEV).normal_(0.0, 110.0, generator=gen).clamp_(-TOP, TOP)
    return x.to(torch.float8_e4m3fn)


def _pool(heads, pages, gen):
    """K codes, V codes and scales of one layer; values have a deviation of about 1.3."""
    _, n_kv, d = HEADS[heads]
    scales = torch.empty(pages, n_kv, 2, device=DEV).uniform_(0.008, 0.016, generator=gen)
    return _codes(gen, pages, n_kv, 4, d // 16, 4, 16), _codes(gen, pages, n_kv, d, PAGE), scales


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def _prepare_maps(case, seed, gen):
    new, cached = _lengths(case)
    held = [_pages(c) for c in cached]
    need = [_pages(c + n) - h for n, c, h in zip(new, cached, held)]
    entries = max(h + m for h, m in zip(held, need)) + 3
    total = sum(held) + sum(need) + 40
    order = torch.randperm(total, device=DEV, generator=gen).to(torch.int32)
    flat = torch.full((len(new), entries), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(entries, device=DEV)
    flat[at[None, :] < _ints(held)[:, None]] = order[:sum(held)]
    rows = sum(new) + case["pad"]
    return dict(case=case, new=_ints(new), cached=_ints(cached), free=order[sum(held):].contiguous(), tables=flat, num_blocks=total,
                row_start=torch.empty(len(new) + 1, dtype=torch.int32, device=DEV), positions=torch.empty(rows, dtype=torch.int32, device=DEV),
                slots=torch.empty(rows, dtype=torch.int32, device=DEV), needed=torch.empty(2, dtype=torch.int32, device=DEV))


def _prepare_store(case, seed, gen):
    n_q, n_kv, d = HEADS[case["heads"]]
    new, cached = _lengths(case)
    rng = random.Random(seed)
    count = [_pages(c + n) - c // PAGE for n, c in zip(new, cached)]                # pages that receive tokens
    ids = list(range(sum(count) + 8))
    rng.shuffle(ids)
    positions, slots, at = [], [], 0
    for n, c, m in zip(new, cached, count):
        positions += range(c, c + n)
        slots += [ids[at + p // PAGE - c // PAGE] * PAGE + p % PAGE for p in range(c, c + n)]
        at += m
    rows, most = len(slots) + case["pad"], max(positions) + 1
    angles = torch.arange(most, dtype=torch.float64, device=DEV)[:, None] * THETA ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEV) / d)
    qkv = torch.empty(rows, (n_q + 2 * n_kv) * d, device=DEV).normal_(0.0, 1.3, generator=gen)
    gains = [torch.empty(d, device=DEV).normal_(1.0, 0.1, generator=gen).bfloat16() if case["norm"] else None for _ in range(2)]
    k, v, scales = _pool(case["heads"], len(ids), gen)
    return dict(case=case, qkv=qkv if case["dtype"] == "f32" else qkv.bfloat16(), q_gain=gains[0], k_gain=gains[1],
                rope=torch.stack((angles.cos(), angles.sin()), -1).float(), positions=_ints(positions + [0] * case["pad"]),
                slots=_ints(slots + [-1] * case["pad"]), q_out=torch.zeros(rows, n_q * d, dtype=torch.bfloat16, device=DEV), k=k, v=v, scales=scales)


def _prepare_attention(case, seed, gen):
    n_q, _, d = HEADS[case["heads"]]
    new, cached = _lengths(case)
    pages = [_pages(c + n) for n, c in zip(new, cached)]
    order = torch.randperm(sum(pages) + 8, device=DEV, generator=gen).to(torch.int32)
    tables = torch.zeros(len(pages), max(pages), dtype=torch.int32, device=DEV)
    at = torch.arange(max(pages), device=DEV)
    tables[at[None, :] < _ints(pages)[:, None]] = order[:sum(pages)]
    k, v, scales = _pool(case["heads"], len(order), gen)
    q = torch.empty(sum(new), n_q * d, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.3, generator=gen)
    groups = [[s for s, n in enumerate(new) if (n == 1) == one] for one in (True, False)]
    sizes = [(max(new[s] for s in g), max(pages[s] for s in g)) if g else (0, 0) for g in groups]
    return dict(case=case, q=q, k=k, v=v, scales=scales, tables=tables, cached=_ints(cached), row_start=_ints(_starts(new)), most=max(new),
                groups=[_ints(g).long() for g in groups], sizes=sizes, out=torch.empty_like(q))


_PREPARE = dict(step_maps=_prepare_maps, norm_rope_store8=_prepare_store, attention8=_prepare_attention)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed, torch.Generator(device=DEV).manual_seed(seed))


# ---- plain forms --------------------------------------------------------------------------------------------------

def _plain_maps(st):
    new, cached, tables, free = st["new"].long(), st["cached"].long(), st["tables"], st["free"]
    ends = new.cumsum(0)
    st["row_start"][:1] = 0
    st["row_start"][1:] = ends
    held = (cached + PAGE - 1) // PAGE
    need = (cached + new + PAGE - 1) // PAGE - held
    before = need.cumsum(0) - need
    entry = torch.arange(tables.shape[1], device=DEV)[None, :] - held[:, None]
    fresh = (entry >= 0) & (entry < need[:, None])
    tables.copy_(torch.where(fresh, free[(before[:, None] + entry).clamp(0, len(free) - 1)], tables))
    row = torch.arange(len(st["slots"]), device=DEV)
    seq = torch.searchsorted(ends, row, right=True)
    real = seq < len(new)
    seq = seq.clamp(max=len(new) - 1)
    pos = torch.where(real, cached[seq] + row - (ends - new)[seq], 0)
    st["positions"].copy_(pos)
    st["slots"].copy_(torch.where(real, tables[seq, pos // PAGE].long() * PAGE + pos % PAGE, -1))
    st["needed"].copy_(torch.stack((new.sum(), need.sum())))
    return [st["row_start"], st["positions"], st["slots"], st["needed"], tables]


def _normed(x, gain):
    if gain is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()


def _rotated(x, angle):
    a, b = x.chunk(2, -1)
    cos, sin = angle[:, None, :, 0], angle[:, None, :, 1]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _grown(scales, biggest, first):
    """Scales of all pages with the new values' largest magnitudes, and the halvings of the codes that pages keep."""
    fit = biggest / TOP
    (m, e), (mo, eo) = torch.frexp(fit), torch.frexp(scales)
    twice = (e - eo + (m > mo)).clamp(min=0)
    first = first[:, None]
    grown = torch.where(first == 0, fit.clamp(min=LEAST), torch.ldexp(scales, twice))
    return torch.where(first < PAGE, grown, scales), torch.where((first > 0) & (first < PAGE), twice, 0)


def _plain_store(st):
    n_q, n_kv, d = HEADS[st["case"]["heads"]]
    rows = (st["slots"] >= 0).nonzero()[:, 0]
    x = st["qkv"][rows].float().view(len(rows), n_q + 2 * n_kv, d)
    angle = st["rope"][st["positions"].long()[rows]]
    st["q_out"][rows] = _rotated(_normed(x[:, :n_q], st["q_gain"]), angle).bfloat16().view(len(rows), n_q * d)
    new = (_rotated(_normed(x[:, n_q:n_q + n_kv], st["k_gain"]), angle), x[:, n_q + n_kv:])
    slots = st["slots"].long()[rows]
    page, slot = slots // PAGE, slots % PAGE
    pages = st["k"].shape[0]
    first = torch.full((pages,), PAGE, device=DEV).scatter_reduce(0, page, slot, "amin")
    at = torch.arange(PAGE, device=DEV)
    pools = (st["k"], st["v"])
    shown = (at.view(1, 1, 4, 1, 4, 1), at.view(1, 1, 1, PAGE))
    for side in (0, 1):
        value, pool = new[side], pools[side]
        biggest = torch.zeros(pages, n_kv, device=DEV).scatter_reduce(0, page[:, None].expand(-1, n_kv), value.abs().amax(-1), "amax")
        scale, twice = _grown(st["scales"][:, :, side], biggest, first)
        st["scales"][:, :, side] = scale
        wide = (pages, n_kv) + (1,) * (pool.dim() - 2)
        kept = (shown[side] < first.view(-1, *(1,) * (pool.dim() - 1))) & (twice > 0).view(wide)
        pool.copy_(torch.where(kept, torch.ldexp(pool.float(), -twice.view(wide)), pool.float()).to(pool.dtype))
        code = (value / scale[page][:, :, None]).clamp(-TOP, TOP).to(pool.dtype).view(torch.uint8)
        if side == 0:
            pool.view(torch.uint8)[page, :, slot // 4, :, slot % 4, :] = code.view(len(rows), n_kv, d // 16, 16)
        else:
            pool.view(torch.uint8)[page, :, :, slot] = code
    return [st["q_out"], st["k"], st["v"], st["scales"]]


def _attend(st, seqs, most, pages):
    """Attention of the sequences `seqs`, of up to `most` rows and `pages` pages, padded to these."""
    c = st["case"]
    n_q, n_kv, d = HEADS[c["heads"]]
    g, S = n_q // n_kv, len(seqs)
    first, last = st["row_start"].long()[seqs], st["row_start"].long()[seqs + 1]
    at = torch.arange(most, device=DEV)
    rows, valid = torch.minimum(first[:, None] + at, last[:, None] - 1), at < (last - first)[:, None]
    tables = st["tables"].long()[seqs, :pages]
    scale = st["scales"][tables]                                                                # [s][page][h][side]
    k = st["k"].view(torch.uint8)[tables].view(torch.float8_e4m3fn).float() * scale[..., 0].view(S, pages, n_kv, 1, 1, 1, 1)
    k = k.permute(0, 2, 4, 6, 1, 3, 5).reshape(S, n_kv, d, pages * PAGE)                        # [s][h][d][key]
    v = st["v"].view(torch.uint8)[tables].view(torch.float8_e4m3fn).float() * scale[..., 1].view(S, pages, n_kv, 1, 1)
    v = v.permute(0, 2, 1, 4, 3).reshape(S, n_kv, pages * PAGE, d)                              # [s][h][key][d]
    q = st["q"][rows].float().view(S, most, n_kv, g, d).permute(0, 2, 1, 3, 4).reshape(S, n_kv, most * g, d)
    key, pos = torch.arange(pages * PAGE, device=DEV), st["cached"].long()[seqs][:, None, None] + at[:, None]
    seen = key <= pos
    if c["window"]:
        seen = seen & ((key > pos - c["window"]) | (key < c["sinks"]))
    score = (q @ k).view(S, n_kv, most, g, -1).mul_(1.0 / math.sqrt(d))
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    p = score.sub_(score.amax(-1, keepdim=True)).exp_()
    o = p.view(S, n_kv, most * g, -1) @ v / p.sum(-1).view(S, n_kv, most * g, 1)
    st["out"][rows[valid]] = o.view(S, n_kv, most, g, d).transpose(1, 2)[valid].reshape(-1, n_q * d).bfloat16()


def _plain_attention(st):
    if len(st["groups"][0]):
        _attend(st, st["groups"][0], *st["sizes"][0])
    if len(st["groups"][1]):
        _attend(st, st["groups"][1], *st["sizes"][1])
    return [st["out"]]


_PLAIN = dict(step_maps=_plain_maps, norm_rope_store8=_plain_store, attention8=_plain_attention)


# ---- the framework's operators --------------------------------------------------------------------------------------

def _own_run(st):
    from paper_2504_14775_amd import cache8
    c = st["case"]
    kind = c["kind"]
    if kind == "step_maps":
        cache8.gllm_op_step_maps(st["new"], st["cached"], st["free"], st["tables"], st["num_blocks"], st["row_start"], st["positions"], st["slots"],
                                 st["needed"])
        return [st["row_start"], st["positions"], st["slots"], st["needed"], st["tables"]]
    if kind == "norm_rope_store8":
        cache8.gllm_op_norm_rope_store8(st["qkv"], st["q_gain"], st["k_gain"], EPS, st["rope"], st["positions"], st["slots"], st["q_out"],
                                        st["k"], st["v"], st["scales"])
        return [st["q_out"], st["k"], st["v"], st["scales"]]
    if "workspace" not in st:                                   # kept beside the inputs as a serving loop keeps it
        n_q, n_kv, d = HEADS[c["heads"]]
        st["workspace"] = torch.empty(cache8.gllm_op_attention8_workspace_bytes(n_q, n_kv, d, st["most"]), dtype=torch.uint8, device=DEV)
    cache8.gllm_op_attention8(st["q"], st["k"], st["v"], st["scales"], st["tables"], st["cached"], st["row_start"], st["out"], st["most"],
                              window=c["window"], sinks=c["sinks"], workspace=st["workspace"])
    return [st["out"]]


def run(st):
    if own:
        return _own_run(st)
    return _PLAIN[st["case"]["kind"]](st)


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------

def _exact_maps(case, st):
    new, cached = _lengths(case)
    tables, free = st["tables"].tolist(), st["free"].tolist()
    positions, slots, used = [], [], 0
    for s, (n, c) in enumerate(zip(new, cached)):
        for p in range(c, c + n):
            if p % PAGE == 0:
                tables[s][p // PAGE] = free[used]
                used += 1
            positions.append(p)
            slots.append(tables[s][p // PAGE] * PAGE + p % PAGE)
    return [_ints(_starts(new)), _ints(positions + [0] * case["pad"]), _ints(slots + [-1] * case["pad"]), _ints([sum(new), used]), _ints(tables)]


def _to_e4m3(x):
    """The nearest e4m3 value, even where two are as near, of numbers in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(x / step) * step).clamp(-TOP, TOP)


def _exact_store(case, st):
    n_q, n_kv, d = HEADS[case["heads"]]
    total = len(st["slots"]) - case["pad"]
    x = st["qkv"][:total].double().view(total, n_q + 2 * n_kv, d)
    turn = st["rope"][st["positions"][:total].long()].double()
    turn = torch.complex(turn[..., 0], turn[..., 1])[:, None]

    def head(y, gain):
        if gain is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
        z = torch.complex(y[..., :d // 2].contiguous(), y[..., d // 2:].contiguous()) * turn
        return torch.cat((z.real, z.imag), -1)

    q = torch.zeros(total + case["pad"], n_q * d, dtype=torch.float64, device=DEV)
    q[:total] = head(x[:, :n_q], st["q_gain"]).reshape(total, n_q * d)
    values = torch.stack((head(x[:, n_q:n_q + n_kv], st["k_gain"]), x[:, n_q + n_kv:]), 2)     # [row][h][side][d]
    pages = st["k"].shape[0]
    held = torch.stack((st["k"].double().permute(0, 2, 4, 1, 3, 5).reshape(pages, PAGE, n_kv, d), st["v"].double().permute(0, 3, 1, 2)), 3)
    slot = st["slots"][:total].long()
    old = st["scales"].double()
    top = torch.zeros(pages * PAGE, n_kv, 2, dtype=torch.float64, device=DEV)
    top[slot] = values.abs().amax(-1)
    top = top.view(pages, PAGE, n_kv, 2).amax(1) / TOP
    wrote = torch.zeros(pages * PAGE, dtype=torch.bool, device=DEV)
    wrote[slot] = True
    wrote = wrote.view(pages, PAGE)
    some, begun = wrote.any(1)[:, None, None], wrote[:, 0][:, None, None]
    grow = torch.exp2(torch.ceil(torch.log2((top / old).clamp(min=1.0))))
    scale = torch.where(some, torch.where(begun, top.clamp(min=LEAST), old * grow), old)
    before = (wrote.int().cumsum(1) == 0)[:, :, None, None, None] & (some & ~begun)[:, None, :, :, None]
    held = torch.where(before, _to_e4m3(held / grow[:, None, :, :, None]), held)
    held = held.reshape(pages * PAGE, n_kv, 2, d)
    held[slot] = _to_e4m3(values / scale[slot // PAGE][..., None])
    held = held.view(pages, 4, 4, n_kv, 2, d // 16, 16)
    k = held[:, :, :, :, 0].permute(0, 3, 1, 4, 2, 5).contiguous()
    v = held[:, :, :, :, 1].reshape(pages, PAGE, n_kv, d).permute(0, 2, 3, 1).contiguous()
    return [q, k, v, scale]


def _exact_attention(case, st):
    n_q, n_kv, d = HEADS[case["heads"]]
    g, out, at = n_q // n_kv, [], 0
    for s, (n, c) in enumerate(zip(*_lengths(case))):
        ids = st["tables"][s, :_pages(c + n)].long()
        of = st["scales"][ids].double()
        k = (st["k"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * of[:, :, 0, None, None, None, None]).permute(1, 0, 2, 4, 3, 5).reshape(n_kv, -1, d)
        v = (st["v"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * of[:, :, 1, None, None]).permute(1, 0, 3, 2).reshape(n_kv, -1, d)
        q = st["q"][at:at + n].double().view(n, n_kv, g, d)
        at += n
        o = torch.empty(n, n_kv, g, d, dtype=torch.float64, device=DEV)
        j, p = torch.arange(k.shape[1], device=DEV), torch.arange(c, c + n, device=DEV)[:, None]
        hide = j > p
        if case["window"]:
            hide = hide | ((p - j >= case["window"]) & (j >= case["sinks"]))
        for h in range(n_kv):
            x = torch.matmul(q[:, h].reshape(n * g, d), k[h].t().contiguous()).view(n, g, -1) * d ** -0.5
            w = torch.softmax(x.masked_fill_(hide[:, None], -math.inf), -1)
            o[:, h] = torch.matmul(w.view(n * g, -1), v[h]).view(n, g, d)
        out.append(o.view(n, n_q * d))
    return [torch.cat(out)]


_EXACT = dict(step_maps=_exact_maps, norm_rope_store8=_exact_store, attention8=_exact_attention)


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def _seen(n, c, window, sinks):
    """Positions that a sequence's rows see, added up, and how many different ones."""
    if not window:
        return n * c + n * (n + 1) // 2, c + n
    pairs = sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(c, c + n))
    low = max(0, c - window + 1)
    return pairs, c + n - low + min(sinks, low)


def work(case):
    new, cached = _lengths(case)
    total = sum(new)
    fresh = sum(_pages(c + n) - _pages(c) for n, c in zip(new, cached))
    touched = sum(_pages(c + n) - c // PAGE for n, c in zip(new, cached))
    if case["kind"] == "step_maps":
        return {"bytes": 4 * (3 * len(new) + 3 + 2 * (total + case["pad"]) + 2 * fresh + (touched - fresh)), "flops": 0}
    n_q, n_kv, d = HEADS[case["heads"]]
    if case["kind"] == "norm_rope_store8":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": total * ((n_q + 2 * n_kv) * d * size + 2 * n_q * d + 4 * d + 8 + 2 * n_kv * d) + 8 * n_kv * (2 * touched - fresh),
                "flops": 10 * total * (n_q + n_kv) * d}
    pairs, keys = (sum(x) for x in zip(*(_seen(n, c, case["window"], case["sinks"]) for n, c in zip(new, cached))))
    return {"bytes": keys * n_kv * (2 * d + 0.5) + 4 * total * n_q * d, "flops": 4 * d * n_q * pairs}
