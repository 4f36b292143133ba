"""Several continuations of one sequence over the paged KV cache, as cases that can be timed and compared.

A serving loop that drafts tokens, or searches with beams, keeps more than one continuation of a sequence on the pages of
the stage's KV pool.  Four operators carry that:

  tree_attention  one layer's attention of a tree of drafted tokens: node i sees the cached prefix, its ancestors and itself
  tree_commit     the walk down the tree along the tokens that the sampler drew, and the accepted nodes' keys and values,
                  of all layers, moved to the slots behind the prefix
  beam_select     the best next (beam, token) pairs of every sequence by accumulated log probability
  copy_pages      pages of the pool copied, of all layers: a beam that forks takes a copy of its last, partly filled page

Head counts are those of the stage shapes ("tiny", "8b", "14b", "70b": query heads, KV heads, head dimension) and of
generic shapes beside them; pages hold 16 tokens, K pages are [d/8][16][8], V pages [d][16], all bf16; logits are float32
with rows padded to a multiple of 256.

A case of kind "tree_attention": heads, seqs, nodes (of the largest tree), ragged (trees of 1 to `nodes` nodes), width
  (drafted tokens per level), lo, hi (cached tokens, spread evenly in the logarithm).
A case of kind "tree_commit": heads, layers, seqs, nodes, width, accept (levels of the tree that are accepted).
A case of kind "beam_select": seqs, beams, vocab, keep (pairs returned per sequence).
A case of kind "copy_pages": heads, layers, pages.
"""
import math
import random

import torch

own = False        # whether run() calls the framework's operators or computes their plain forms

DEV = "cuda:0"
PAGE = 16
HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "14b": (40, 8, 128), "70b": (64, 8, 128),
         "g1_64": (8, 8, 64), "g16_128": (16, 1, 128), "g3_128": (12, 4, 128), "g7_64": (14, 2, 64)}
VOCABS = (128256, 152064)


def _attention(name, heads, seqs, nodes, width, lo, hi, ragged=False):
    return dict(name=name, kind="tree_attention", heads=heads, seqs=seqs, nodes=nodes, width=width, lo=lo, hi=hi, ragged=ragged)


def _commit(name, heads, layers, seqs, nodes, width, accept):
    return dict(name=name, kind="tree_commit", heads=heads, layers=layers, seqs=seqs, nodes=nodes, width=width, accept=accept)


def _beams(name, seqs, beams, vocab, keep):
    return dict(name=name, kind="beam_select", seqs=seqs, beams=beams, vocab=vocab, keep=keep)


def _copy(name, heads, layers, pages):
    return dict(name=name, kind="copy_pages", heads=heads, layers=layers, pages=pages)


def listed():
    return [
        # the smallest call: the one-layer test shape, three short sequences with small trees; latency
        _attention("tree_tiny_3x5", "tiny", 3, 5, 2, 17, 64),
        # one user at the keyboard: a usual tree of drafted tokens behind one long chat
        _attention("tree_8b_1x26", "8b", 1, 26, 8, 2500, 2500),
        # speculation off for a while: single tokens through the same call, beside an agent's long context
        _attention("tree_8b_32x1", "8b", 32, 1, 1, 300, 20000),
        # a serving batch with five query heads per KV head and trees pruned to different sizes
        _attention("tree_14b_48_ragged", "14b", 48, 60, 8, 100, 6000, ragged=True),
        # the largest: eight query heads per KV head, 64 nodes each, where the matrix cores begin to bound it
        _attention("tree_70b_16x64", "70b", 16, 64, 8, 1000, 8000),
        # behind a verified tree of one user, all eight layers of a stage
        _commit("commit_8b_1x26", "8b", 8, 1, 26, 8, 3),
        # behind a verified serving batch
        _commit("commit_14b_64x60", "14b", 12, 64, 60, 10, 5),
        # one request with four beams
        _beams("beams_1x4", 1, 4, VOCABS[0], 8),
        # translation-like serving: sixteen requests of five beams, an odd number of logits
        _beams("beams_16x5_odd", 16, 5, 50261, 10),
        # the largest: sixty-four requests of eight beams
        _beams("beams_64x8", 64, 8, VOCABS[1], 16),
        # three of one request's four beams fork
        _copy("copy_8b_3", "8b", 8, 3),
        # all beams of a serving batch fork
        _copy("copy_70b_160", "70b", 20, 160),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def draw(rng):
    """One more case of the same ranges, no costlier than the costliest listed one of its kind."""
    while True:
        kind = rng.choice(("tree_attention", "tree_attention", "tree_commit", "beam_select", "copy_pages"))
        heads = rng.choice(tuple(HEADS))
        if kind == "tree_attention":
            hi = _log_int(rng, 16, 40000)
            c = _attention("", heads, _log_int(rng, 1, 200), _log_int(rng, 1, 256), rng.randint(1, 16),
                           max(0, int(hi * rng.uniform(0.0, 1.0))), hi, ragged=rng.random() < 0.5)
        elif kind == "tree_commit":
            width, depth = rng.randint(2, 16), rng.randint(1, 12)
            c = _commit("", heads, rng.randint(1, 20), _log_int(rng, 1, 128), 1 + width * depth, width, rng.randint(0, min(depth, width)))
        elif kind == "beam_select":
            beams = _log_int(rng, 1, 32)
            c = _beams("", _log_int(rng, 1, 64), beams, rng.choice(VOCABS + (_log_int(rng, 500, 200000), _log_int(rng, 500, 200000))),
                       rng.randint(beams, 2 * beams))
        else:
            c = _copy("", heads, rng.randint(1, 20), _log_int(rng, 1, 300))
        del c["name"]
        if _cost(c) <= max(_cost(d) for d in listed() if d["kind"] == kind):
            return c


def _spread(case):
    """Cached tokens per sequence."""
    s, lo, hi = case["seqs"], max(1, case["lo"]), max(1, case["hi"])
    lens = [int(lo * (hi / lo) ** ((i + 0.5) / s)) for i in range(s)]
    random.Random(s * 8209 + hi).shuffle(lens)
    return lens


def _nodes(case):
    """Nodes per sequence."""
    s, n = case["seqs"], case["nodes"]
    if not case.get("ragged"):
        return [n] * s
    rng = random.Random(s * 4099 + n)
    return [n] + [rng.randint(1, n) for _ in range(s - 1)]


def _tree(n, width, rng):
    """Parents of a draft tree: a root (the last token the sequence has), then levels of `width` nodes, each a child of some
    node of the level before."""
    level = [0]
    parents = [-1]
    while len(parents) < n:
        new = range(len(parents), min(n, len(parents) + width))
        parents += [rng.choice(level) for _ in new]
        level = list(new)
    return parents


def _trees(case):
    return [_tree(n, case["width"], random.Random(17 * i + n)) for i, n in enumerate(_nodes(case))]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pool(case, layers, pages, gen):
    """K pool and V pool, [layer][page][KV head] pages."""
    _, n_kv, d = HEADS[case["heads"]]
    k = torch.empty(layers, pages, n_kv, d // 8, PAGE, 8, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.3, generator=gen)
    v = torch.empty(layers, pages, n_kv, d, PAGE, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.3, generator=gen)
    return k, v


def _prepare_attention(case, seed, gen):
    n_q, _, d = HEADS[case["heads"]]
    cached, trees = _spread(case), _trees(case)
    pages = [-(-(c + len(t)) // PAGE) for c, t in zip(cached, trees)]
    order = torch.randperm(sum(pages) + 8, device=DEV, generator=gen).to(torch.int32)
    tables = torch.zeros(len(pages), max(pages), dtype=torch.int32, device=DEV)
    at = 0
    for s, p in enumerate(pages):
        tables[s, :p] = order[at:at + p]
        at += p
    k, v = _pool(case, 1, len(order), gen)
    starts = [0]
    for t in trees:
        starts.append(starts[-1] + len(t))
    q = torch.empty(starts[-1], n_q * d, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.3, generator=gen)
    return dict(case=case, q=q, k=k[0], v=v[0], tables=tables, cached=_ints(cached), starts=_ints(starts),
                parents=_ints(sum(trees, [])), most=max(len(t) for t in trees), out=torch.empty_like(q))


def _prepare_commit(case, seed, gen):
    rng, trees, vocab = random.Random(seed), _trees(case), VOCABS[0]
    starts, tokens, sampled = [0], [], []
    for parents in trees:
        # siblings are drafted with different tokens; the sampler draws the token of the next node of an accepted path, and
        # at the path's end one that nobody drafted.  The path's second node is the first of its level or one whose slot lies
        # behind the accepted ones, so that no key or value moves to a slot that is read, and a pass can be made again
        toks = [rng.randrange(vocab // 2) * 2 for _ in parents]
        drawn = [2 * rng.randrange(vocab // 2) + 1 for _ in parents]
        toks = [t - t % 512 + 2 * (i % 256) for i, t in enumerate(toks)]
        cur = 0
        for level in range(case["accept"]):
            kids = [i for i, p in enumerate(parents) if p == cur and (level > 0 or i == 1 or i > case["accept"])]
            if not kids:
                break
            nxt = rng.choice(kids)
            drawn[cur] = toks[nxt]
            cur = nxt
        tokens += toks
        sampled += drawn
        starts.append(starts[-1] + len(parents))
    # prefixes end anywhere in a page; their whole pages are not touched and all name page 0
    lens = random.Random(31 * len(trees) + case["nodes"])
    cached = [lens.randrange(64 * PAGE) for _ in trees]
    first = [c // PAGE for c in cached]
    count = [(c + len(t) - 1) // PAGE - f + 1 for c, t, f in zip(cached, trees, first)]
    order = (torch.randperm(sum(count), device=DEV, generator=gen) + 1).to(torch.int32)
    tables = torch.zeros(len(trees), max(f + n for f, n in zip(first, count)), dtype=torch.int32, device=DEV)
    at = 0
    for s, (f, n) in enumerate(zip(first, count)):
        tables[s, f:f + n] = order[at:at + n]
        at += n
    k, v = _pool(case, case["layers"], sum(count) + 1, gen)
    rows, s = starts[-1], len(trees)
    return dict(case=case, tokens=_ints(tokens), sampled=_ints(sampled), parents=_ints(sum(trees, [])), starts=_ints(starts),
                cached=_ints(cached), tables=tables, k=k, v=v, most=max(len(t) for t in trees), path=torch.empty(rows, dtype=torch.int32, device=DEV),
                count=torch.empty(s, dtype=torch.int32, device=DEV), next=torch.empty(s, dtype=torch.int32, device=DEV))


def _prepare_beams(case, seed, gen):
    s, w, vocab, keep = case["seqs"], case["beams"], case["vocab"], case["keep"]
    # logits of a standard deviation of 4 to 5 share nearly all of the probability among a few to a few thousand tokens, as
    # a trained model's do; padding columns hold zeros
    logits = torch.zeros(s * w, -(-vocab // 256) * 256, device=DEV)
    logits[:, :vocab].normal_(0.0, 4.5, generator=gen)
    scores = -(torch.rand(s, w, device=DEV, generator=gen) * 6.0 + 8.0)
    return dict(case=case, logits=logits, scores=scores, out_scores=torch.empty(s, keep, device=DEV),
                out_beams=torch.empty(s, keep, dtype=torch.int32, device=DEV), out_tokens=torch.empty(s, keep, dtype=torch.int32, device=DEV))


def _prepare_copy(case, seed, gen):
    n, rng = case["pages"], random.Random(seed)
    k, v = _pool(case, case["layers"], 2 * n + 4, gen)
    ids = rng.sample(range(2 * n + 4), 2 * n)
    # beams that come from the same beam copy the same page
    src = [ids[i - i % 3] if i % 3 == 1 else ids[i] for i in range(n)]
    return dict(case=case, k=k, v=v, src=src, dst=ids[n:])


_PREPARE = dict(tree_attention=_prepare_attention, tree_commit=_prepare_commit, beam_select=_prepare_beams, copy_pages=_prepare_copy)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed, torch.Generator(device=DEV).manual_seed(seed))


# ---- plain forms --------------------------------------------------------------------------------------------------

def _padded(st):
    """Rows [sequence][node] with the rows past a sequence's last node clamped, and which of them exist."""
    starts = st["starts"].long()
    n = starts[1:] - starts[:-1]
    at = torch.arange(st["most"], device=DEV)
    return torch.minimum(starts[:-1, None] + at, starts[1:, None] - 1), at < n[:, None]


def _ancestors(parents, valid):
    """[sequence][node][node]: whether the second node is the first one or an ancestor of it.  Powers of (parent links + 1)."""
    n = parents.shape[1]
    at = torch.arange(n, device=DEV)
    step = ((parents[:, :, None] == at) & valid[:, :, None]).float() + torch.eye(n, device=DEV)
    step = ((step @ step) > 0).float()                    # two links
    step = ((step @ step) > 0).float()                    # four
    step = ((step @ step) > 0).float()
    step = ((step @ step) > 0).float()                    # sixteen
    step = ((step @ step) > 0).float()
    step = ((step @ step) > 0).float()
    step = ((step @ step) > 0).float()
    return (step @ step) > 0                              # 256: the deepest tree there is


def _plain_attention(st):
    n_q, n_kv, d = HEADS[st["case"]["heads"]]
    g, S, N = n_q // n_kv, st["tables"].shape[0], st["most"]
    rows, valid = _padded(st)
    anc = _ancestors(st["parents"].long()[rows], valid)
    tables = st["tables"].long()
    k = st["k"][tables].float().permute(0, 2, 3, 5, 1, 4).reshape(S, n_kv, d, -1)               # [s][h][d][key]
    v = st["v"][tables].float().permute(0, 2, 1, 4, 3).reshape(S, n_kv, -1, d)                  # [s][h][key][d]
    q = st["q"][rows].float().view(S, N, n_kv, g, d).permute(0, 2, 1, 3, 4).reshape(S, n_kv, N * g, d)
    key = torch.arange(k.shape[-1], device=DEV) - st["cached"].long()[:, None]                  # < 0: cached
    node = key.clamp(0, N - 1)[:, None, :].expand(S, N, -1)
    seen = (key < 0)[:, None] | ((key >= 0) & (key < valid.sum(1)[:, None]))[:, None] & anc.gather(2, node)
    score = (q @ k).view(S, n_kv, N, g, -1) / math.sqrt(d)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    p = (score - score.amax(-1, keepdim=True)).exp_()
    o = p.view(S, n_kv, N * g, -1) @ v / p.sum(-1).view(S, n_kv, N * g, 1)
    st["out"].copy_(o.view(S, n_kv, N, g, d).transpose(1, 2)[valid].reshape(-1, n_q * d))
    return [st["out"]]


def _plain_commit(st):
    rows, valid = _padded(st)
    parents, tokens, sampled = (st[x].long()[rows] for x in ("parents", "tokens", "sampled"))
    anc = _ancestors(parents, valid)
    at = torch.arange(rows.shape[1], device=DEV)
    twin = (parents[:, :, None] == parents[:, None, :]) & (tokens[:, :, None] == tokens[:, None, :]) & (at < at[:, None])
    match = (sampled.gather(1, parents.clamp(min=0)) == tokens) & ~twin.any(2)
    match[:, 0] = True
    accepted = valid & ~(anc & ~match[:, None, :]).any(2)
    rank = accepted.cumsum(1) - 1
    count = accepted.sum(1)
    s, node = accepted.nonzero(as_tuple=True)                                                  # in order of the node: of the path
    at = rank[s, node]
    st["path"].fill_(-1)[st["starts"].long()[s] + at] = node.int()
    st["count"].copy_(count)
    last = (accepted * torch.arange(1, rows.shape[1] + 1, device=DEV)).amax(1) - 1
    st["next"].copy_(sampled.gather(1, last[:, None])[:, 0])
    tables, cached = st["tables"].long(), st["cached"].long()
    src, dst = cached[s] + node, cached[s] + at
    sp, dp, ss, ds = tables[s, src // PAGE], tables[s, dst // PAGE], src % PAGE, dst % PAGE
    st["k"][:, dp, :, :, ds] = st["k"][:, sp, :, :, ss]
    st["v"][:, dp, :, :, ds] = st["v"][:, sp, :, :, ss]
    return [st["path"], st["count"], st["next"], st["k"], st["v"]]


def _plain_beams(st):
    c = st["case"]
    s, w, vocab, keep = c["seqs"], c["beams"], c["vocab"], c["keep"]
    x = st["logits"][:, :vocab].double()                                     # scores next to each other decide the order
    x = x - x.amax(1, keepdim=True)
    x = x - x.exp().sum(1, keepdim=True).log() + st["scores"].double().view(-1, 1)
    best = x.view(s, -1).topk(min(2 * keep, w * vocab), dim=1).indices.sort(dim=1).values       # by index, so that equal
    score = x.view(s, -1).gather(1, best)                                    # scores stay in that order
    order = score.sort(dim=1, descending=True, stable=True).indices[:, :keep]
    best = best.gather(1, order)
    st["out_scores"].copy_(score.gather(1, order))
    st["out_beams"].copy_(best // vocab)
    st["out_tokens"].copy_(best % vocab)
    return [st["out_scores"], st["out_beams"], st["out_tokens"]]


def _plain_copy(st):
    src, dst = (torch.tensor(st[x], device=DEV) for x in ("src", "dst"))
    st["k"][:, dst] = st["k"][:, src]
    st["v"][:, dst] = st["v"][:, src]
    return [st["k"], st["v"]]


_PLAIN = dict(tree_attention=_plain_attention, tree_commit=_plain_commit, beam_select=_plain_beams, copy_pages=_plain_copy)


# ---- the framework's operators --------------------------------------------------------------------------------------

def _workspace(st, size):
    """The operator's workspace, kept beside the inputs as a serving loop keeps it."""
    if "workspace" not in st:
        st["workspace"] = torch.empty(size(), dtype=torch.uint8, device=DEV)
    return st["workspace"]


def _own_run(st):
    from paper_2504_14775_amd import branch
    c = st["case"]
    kind = c["kind"]
    if kind == "tree_attention":
        n_q, n_kv, d = HEADS[c["heads"]]
        ws = _workspace(st, lambda: branch.gllm_op_tree_attention_workspace_bytes(n_q, n_kv, d, st["most"]))
        branch.gllm_op_tree_attention(st["q"], st["k"], st["v"], st["tables"], st["cached"], st["starts"], st["parents"], st["out"],
                                      st["most"], workspace=ws)
        return [st["out"]]
    if kind == "tree_commit":
        branch.gllm_op_tree_commit(st["tokens"], st["parents"], st["sampled"], st["starts"], st["cached"], st["tables"], st["k"], st["v"],
                                   st["path"], st["count"], st["next"])
        return [st["path"], st["count"], st["next"], st["k"], st["v"]]
    if kind == "beam_select":
        ws = _workspace(st, lambda: branch.gllm_op_beam_select_workspace_bytes(c["seqs"], c["beams"], c["vocab"], c["keep"]))
        branch.gllm_op_beam_select(st["logits"], c["vocab"], st["scores"], st["out_scores"], st["out_beams"], st["out_tokens"], workspace=ws)
        return [st["out_scores"], st["out_beams"], st["out_tokens"]]
    branch.gllm_op_copy_pages(st["k"], st["v"], st["src"], st["dst"])
    return [st["k"], st["v"]]


def run(st):
    if own:
        return _own_run(st)
    return _PLAIN[st["case"]["kind"]](st)


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------

def _chain(parents, i):
    up = [i]
    while parents[up[-1]] >= 0:
        up.append(parents[up[-1]])
    return sorted(up)


def _exact_attention(case, st):
    n_q, n_kv, d = HEADS[case["heads"]]
    g, out, at = n_q // n_kv, [], 0
    for s, (c, parents) in enumerate(zip(_spread(case), _trees(case))):
        n = len(parents)
        pages = st["tables"][s, :-(-(c + n) // PAGE)].long()
        k = st["k"][pages].double().permute(1, 0, 3, 2, 4).reshape(n_kv, -1, d)[:, :c + n].contiguous()
        v = st["v"][pages].double().permute(1, 0, 3, 2).reshape(n_kv, -1, d)[:, :c + n].contiguous()
        q = st["q"][at:at + n].double().view(n, n_kv, g, d)
        at += n
        o = torch.empty(n, n_kv, g, d, dtype=torch.float64, device=DEV)
        hide = torch.ones(n, c + n, dtype=torch.bool)
        hide[:, :c] = False
        for i in range(n):
            hide[i, [c + a for a in _chain(parents, i)]] = False
        hide = hide.to(DEV)
        for h in range(n_kv):
            x = torch.matmul(q[:, h].reshape(n * g, d), k[h].t().contiguous()).view(n, g, -1) * d ** -0.5
            w = torch.softmax(x.masked_fill(hide[:, None], -math.inf), -1)
            o[:, h] = torch.matmul(w.view(n * g, -1), v[h]).view(n, g, d)
        out.append(o.view(n, n_q * d))
    return [torch.cat(out)]


def _exact_commit(case, st):
    tokens, sampled = st["tokens"].tolist(), st["sampled"].tolist()
    path, count, follow, at = [], [], [], 0
    k, v = st["k"].clone(), st["v"].clone()
    for s, parents in enumerate(_trees(case)):
        walk = [0]
        while True:
            kids = [i for i, p in enumerate(parents) if p == walk[-1] and tokens[at + i] == sampled[at + walk[-1]]]
            if not kids:
                break
            walk.append(kids[0])
        table, c = st["tables"][s].tolist(), int(st["cached"][s])
        for i, j in enumerate(walk):
            (a, b), (x, y) = divmod(c + i, PAGE), divmod(c + j, PAGE)
            k[:, table[a], :, :, b] = st["k"][:, table[x], :, :, y]
            v[:, table[a], :, :, b] = st["v"][:, table[x], :, :, y]
        path += walk + [-1] * (len(parents) - len(walk))
        count.append(len(walk))
        follow.append(sampled[at + walk[-1]])
        at += len(parents)
    return [_ints(path), _ints(count), _ints(follow), k, v]


def _exact_beams(case, st):
    s, w, vocab, keep = case["seqs"], case["beams"], case["vocab"], case["keep"]
    scores, beams, tokens = [], [], []
    for i in range(s):
        logp = torch.log_softmax(st["logits"][i * w:(i + 1) * w, :vocab].double(), -1) + st["scores"][i].double()[:, None]
        value, at = torch.sort(logp.reshape(-1), descending=True, stable=True)
        scores.append(value[:keep])
        beams.append(at[:keep] // vocab)
        tokens.append(at[:keep] % vocab)
    return [torch.stack(scores), torch.stack(beams).int(), torch.stack(tokens).int()]


def _exact_copy(case, st):
    k, v = st["k"].clone(), st["v"].clone()
    for a, b in zip(st["src"], st["dst"]):
        k[:, b], v[:, b] = st["k"][:, a], st["v"][:, a]
    return [k, v]


_EXACT = dict(tree_attention=_exact_attention, tree_commit=_exact_commit, beam_select=_exact_beams, copy_pages=_exact_copy)


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def _depth_sum(parents):
    """Nodes that the nodes of a tree see, themselves among them, added up."""
    depth = []
    for p in parents:
        depth.append(1 + (depth[p] if p >= 0 else 0))
    return sum(depth)


def work(case):
    if case["kind"] == "beam_select":
        rows = case["seqs"] * case["beams"]
        return {"bytes": 4 * rows * (case["vocab"] + 1) + 12 * case["seqs"] * case["keep"], "flops": 0}
    n_q, n_kv, d = HEADS[case["heads"]]
    if case["kind"] == "copy_pages":
        return {"bytes": 2 * 2 * 2 * case["pages"] * case["layers"] * n_kv * d * PAGE, "flops": 0}
    trees = _trees(case)
    rows = sum(len(t) for t in trees)
    if case["kind"] == "tree_commit":
        return {"bytes": 16 * rows + 2 * 2 * 2 * case["seqs"] * case["accept"] * case["layers"] * n_kv * d, "flops": 0}
    cached = _spread(case)
    keys = sum(c + len(t) for c, t in zip(cached, trees))
    pairs = sum(c * len(t) + _depth_sum(t) for c, t in zip(cached, trees))
    return {"bytes": keys * n_kv * d * 2 * 2 + 2 * rows * n_q * d * 2 + 4 * rows, "flops": 4 * d * n_q * pairs}
