"""The branch operators run together as a serving loop uses them: trees of drafted tokens through the stage, acceptance, the cache that goes
on; and beam search over decode rows with forked pages.  Tiny two-layer model, one page pool.

The stage over trees is held to the oracle: a node's output is that of the last row of the chain from its root to it, within the tolerance
of the one-layer and two-layer stage cases (max abs 2e-2, sum|d|/sum|ref| 5e-3 on the float32 stream).  The loops are held to loops without
branches on the same stage: tokens equal.  (Greedy tokens and beams of two such loops can differ only where scores agree to the stage's
rounding, about 1e-2; inputs are seeded and the kernels deterministic.)"""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
from oracle import branch_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import branch as BR
from paper_2504_14775_amd import head as HD
from paper_2504_14775_amd import synth
from gpu_util import DEV, bits_of, to_dev_bits
from helpers import layer_weights_np

pytestmark = pytest.mark.gpu
PAGE = 16


def dev_ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


class Model:
    def __init__(self, seed, pages, vocab=300, layers=2, max_tokens=512, max_seqs=64, context=256, **shape):
        self.shape = s = dataclasses.replace(synth.SHAPES["tiny"], num_layers=layers, name="branch", **shape)
        self.vocab, self.pages = vocab, pages
        self.weights = layer_weights_np(s, seed)
        self.stage = B.Stage(B.make_config(s, max_tokens, max_seqs, context // PAGE, context))
        self.stage.bind_workspace(torch.empty(self.stage.workspace_bytes(), dtype=torch.uint8, device=DEV))
        for l, w in enumerate(self.weights):
            self.stage.load_layer(l, {k: to_dev_bits(v) for k, v in w.items()})
        self.k = torch.zeros(layers, pages, s.n_kv_heads, s.head_dim // 8, PAGE, 8, dtype=torch.bfloat16, device=DEV)
        self.v = torch.zeros(layers, pages, s.n_kv_heads, s.head_dim, PAGE, dtype=torch.bfloat16, device=DEV)
        self.stage.bind_kv_pool(self.k, self.v, pages)
        self.table = synth.normal_bf16(seed, 1, 0, vocab * s.hidden, 1.0, 0.0).reshape(vocab, s.hidden).to(DEV)
        self.head = HD.Head(s.hidden, vocab, max_tokens, s.rms_eps)
        self.head.load(synth.normal_bf16(seed, 2, 0, s.hidden, 0.1, 1.0).to(DEV), synth.normal_bf16(seed, 3, 0, vocab * s.hidden, 0.05, 0.0).reshape(vocab, s.hidden).to(DEV))

    def logits(self, new_tokens, cached, tables, ids, rows, parents=None):
        """Logits of `rows` of a batch of token ids."""
        T = len(ids)
        x = torch.empty(T, self.shape.hidden, dtype=torch.bfloat16, device=DEV)
        out, out32 = torch.empty_like(x), torch.empty(T, self.shape.hidden, device=DEV)
        HD.gllm_op_embedding(dev_ints(ids), self.table, x)
        if parents is None:
            self.stage.forward(new_tokens, cached, tables, x, out, out32)
        else:
            self.stage.forward_tree(new_tokens, cached, tables, parents, x, out, out32)
        lg = torch.empty(len(rows), self.head.padded_vocab, device=DEV)
        self.head.logits(out32, dev_ints(rows), lg)
        return lg

    def greedy(self, lg):
        m = lg.shape[0]
        out = dev_ints(np.zeros(m))
        HD.gllm_op_sample(lg, self.vocab, torch.zeros(m, device=DEV), dev_ints(np.zeros(m)), torch.ones(m, device=DEV), torch.zeros(m, device=DEV), out)
        return out

    def close(self):
        torch.cuda.synchronize()
        self.head.destroy()
        self.stage.destroy()


@pytest.mark.parametrize("n_q,n_kv,d,hidden", [(4, 2, 64, 256), (8, 1, 128, 256), (6, 2, 64, 384)])
def test_stage_over_trees_is_the_stage_over_each_of_their_paths(n_q, n_kv, d, hidden):
    print(f"stage over trees {n_q}/{n_kv}/{d}", flush=True)
    rng = np.random.default_rng(n_q)
    shape = dataclasses.replace(synth.SHAPES["tiny"], num_layers=2, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, hidden=hidden, name="trees")
    weights = layer_weights_np(shape, 7)
    # two trees, a chunk, a decode row and a wide tree, in one batch
    trees = [[-1, 0, 0, 1, 1, 2, 5, 5], list(range(-1, 12)), [-1], [-1, 0, 1, 1, 0, -1, 5], [-1] + [0] * 30 + [int(rng.integers(1, 31)) for _ in range(20)]]
    cached = [21, 40, 77, 0, 15]
    new = [len(t) for t in trees]
    parents = np.concatenate(trees).astype(np.int32)
    pages = [-(-(c + n) // PAGE) for c, n in zip(cached, new)]
    order = rng.permutation(sum(pages) + 3)
    tables = np.zeros((5, max(pages)), dtype=np.int32)
    at = 0
    for s, p in enumerate(pages):
        tables[s, :p] = order[at:at + p]
        at += p
    num_blocks = len(order)
    T = sum(new)
    k0, v0 = (synth.bf16_bits(x).copy() for x in synth.make_pool(shape, 7, num_blocks))
    hidden_in = synth.bf16_bits(synth.make_hidden(shape, 7, T))
    stage = B.Stage(B.make_config(shape, T, 5, max(pages), max(pages) * PAGE))
    stage.bind_workspace(torch.empty(stage.workspace_bytes(), dtype=torch.uint8, device=DEV))
    for l, w in enumerate(weights):
        stage.load_layer(l, {k: to_dev_bits(v) for k, v in w.items()})
    dk, dv = to_dev_bits(k0), to_dev_bits(v0)
    stage.bind_kv_pool(dk, dv, num_blocks)
    out, out32 = torch.empty(T, hidden, dtype=torch.bfloat16, device=DEV), torch.empty(T, hidden, device=DEV)
    x = to_dev_bits(hidden_in)
    stage.forward_tree(new, cached, tables, parents, x, out, out32)
    torch.cuda.synchronize()
    got = out32.cpu().numpy().astype(np.float64)
    # slots of no new token keep their bits
    from helpers import written_mask
    mk, mv = written_mask(shape, synth.Batch(np.array(new, dtype=np.int32), np.array(cached, dtype=np.int32), tables, num_blocks))
    gk, gv = bits_of(dk), bits_of(dv)
    assert np.array_equal(gk[~mk], k0[~mk]) and np.array_equal(gv[~mv], v0[~mv])
    # every path from a root to a leaf as a chunk of its own, over pages of its own that start as copies of the sequence's
    paths, starts = [], np.concatenate([[0], np.cumsum(new)])
    for s, t in enumerate(trees):
        leaves = [i for i in range(len(t)) if i not in t]
        paths += [(s, O.chain(t, i)) for i in leaves]
    per = synth.pool_elems_per_layer(shape, num_blocks) // num_blocks
    K, V = (z.reshape(2, num_blocks, per) for z in (k0, v0))
    ptab, kk, vv, nb = np.zeros((len(paths), max(pages)), dtype=np.int32), [], [], 0
    for i, (s, path) in enumerate(paths):
        p = -(-(cached[s] + len(path)) // PAGE)
        ptab[i, :p] = np.arange(nb, nb + p)
        kk.append(K[:, tables[s, :p]])
        vv.append(V[:, tables[s, :p]])
        nb += p
    kk, vv = (np.ascontiguousarray(np.concatenate(z, 1)).reshape(-1) for z in (kk, vv))
    rows = np.concatenate([starts[s] + np.array(path) for s, path in paths])
    ref, _ = oracle.stage_forward(shape, weights, np.array([len(p) for _, p in paths], dtype=np.int32), np.array([cached[s] for s, _ in paths], dtype=np.int32),
                                  ptab, nb, kk, vv, hidden_in[rows])
    d_ = np.abs(got[rows] - ref)
    print(f"[parity] trees: max_abs={d_.max():.4g} mean_rel={d_.sum() / np.abs(ref).sum():.4g} over {len(rows)} rows", flush=True)
    assert set(rows) == set(range(T))
    assert d_.max() <= 2e-2 * max(1.0, np.sqrt((ref ** 2).mean())) and d_.sum() / np.abs(ref).sum() <= 5e-3
    # parents that make every sequence a chain: the same bits as forward()
    chain = np.concatenate([np.arange(-1, n - 1) for n in new])
    results = []
    for call in (lambda o: stage.forward(new, cached, tables, x, o), lambda o: stage.forward_tree(new, cached, tables, chain, x, o)):
        dk.copy_(to_dev_bits(k0))
        dv.copy_(to_dev_bits(v0))
        o = torch.empty_like(out)
        call(o)
        torch.cuda.synchronize()
        results.append((bits_of(o).copy(), bits_of(dk).copy(), bits_of(dv).copy()))
    assert all(np.array_equal(a, b) for a, b in zip(*results))
    # refusals
    for bad, status in (([0] + list(parents[1:]), -1), ([-2] + list(parents[1:]), -1), ([-1, 1] + list(parents[2:]), -1)):
        with pytest.raises(B.GllmError) as e:
            stage.forward_tree(new, cached, tables, np.array(bad), x, out)
        assert e.value.status == status
    stage.destroy()


def test_a_pass_over_trees_replayed_from_a_graph():
    print("stage over trees from a graph", flush=True)
    m = Model(17, 40)
    rng = np.random.default_rng(17)
    trees = [[-1, 0, 0, 1, 1, 2, 5, 5], [-1], list(range(-1, 20)), [-1, -1, 0, 1, 3]]
    new, cached = [len(t) for t in trees], [50, 33, 10, 0]
    T, tables = sum(new), np.arange(32).reshape(4, 8)[:, ::-1].copy()
    m.k.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    m.v.normal_(generator=torch.Generator(device=DEV).manual_seed(2))
    pools = m.k.clone(), m.v.clone()
    x = torch.empty(T, m.shape.hidden, dtype=torch.bfloat16, device=DEV)
    out, again = torch.empty_like(x), torch.empty_like(x)
    call = lambda o: m.stage.forward_tree(new, cached, tables, np.concatenate(trees), x, o)
    x.normal_()
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(again)
    for i in range(3):
        x.copy_(torch.tensor(rng.standard_normal((T, m.shape.hidden)), device=DEV))
        for a, b in zip((m.k, m.v), pools):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        replayed = again.clone(), m.k.clone(), m.v.clone()
        for a, b in zip((m.k, m.v), pools):
            a.copy_(b)
        call(out)
        torch.cuda.synchronize()
        assert torch.isfinite(out.float()).all()
        for a, b in zip(replayed, (out, m.k, m.v)):
            assert torch.equal(a, b)
    m.close()


def test_trees_of_too_many_nodes_are_refused_by_the_stage():
    m = Model(3, 64, layers=1, max_tokens=300, context=512)
    x = torch.zeros(257, m.shape.hidden, dtype=torch.bfloat16, device=DEV)
    parents = np.zeros(257, dtype=np.int32)
    parents[0] = -1
    with pytest.raises(B.GllmError) as e:
        m.stage.forward_tree([257], [0], np.arange(17)[None], parents, x[:257], torch.empty_like(x))
    assert e.value.status == -2 and "256 nodes" in e.value.message
    m.stage.forward_tree([256], [0], np.arange(16)[None], parents[:256], x[:256], torch.empty_like(x))
    m.stage.forward_tree([257], [0], np.arange(17)[None], np.arange(-1, 256), x, torch.empty_like(x))      # a chunk
    m.close()


def plain_greedy(m, tables, prompts, steps):
    """Tokens that decoding one at a time gives."""
    tokens = [list(p) for p in prompts]
    lg = m.logits([len(p) for p in prompts], [0] * len(prompts), tables, np.concatenate(prompts), np.cumsum([len(p) for p in prompts]) - 1)
    for _ in range(steps):
        for t, n in zip(tokens, m.greedy(lg).cpu().numpy()):
            t.append(int(n))
        lg = m.logits([1] * len(tokens), [len(t) - 1 for t in tokens], tables, [t[-1] for t in tokens], np.arange(len(tokens)))
    return tokens


def test_decoding_with_drafted_trees_gives_the_tokens_of_decoding_one_by_one():
    print("speculative decoding", flush=True)
    rng = np.random.default_rng(21)
    prompts = [rng.integers(0, 300, n).tolist() for n in (37, 16, 5, 63)]
    m = Model(21, 80)
    tables = rng.permutation(80)[:64].reshape(4, 16).astype(np.int32)
    want = plain_greedy(m, tables, prompts, 40)
    m.k.fill_(float("nan"))
    m.v.fill_(float("nan"))
    tables = rng.permutation(80)[:64].reshape(4, 16).astype(np.int32)
    d_tables = dev_ints(tables)
    lg = m.logits([len(p) for p in prompts], [0] * 4, tables, np.concatenate(prompts), np.cumsum([len(p) for p in prompts]) - 1)
    tokens = [p + [int(t)] for p, t in zip(prompts, m.greedy(lg).cpu().numpy())]
    cached, passes, accepted = [len(p) for p in prompts], 0, 0
    while min(len(t) - len(p) for t, p in zip(tokens, prompts)) < 30:
        trees, ids = [], []
        for s in range(4):
            done = len(tokens[s])
            follow = want[s][done:done + 4]
            if s == 3 or not follow:                                             # no drafts: a decode row
                trees.append([-1])
                ids.append([tokens[s][-1]])
                continue
            # levels of three: the token that comes (now and then none of them) among others, below a node of the level before
            up, tok, level, right = [-1], [tokens[s][-1]], [0], 0
            for depth in range(min(len(follow), 1 + s)):
                good = int(rng.integers(0, 4))
                new = []
                for j in range(3):
                    parent = right if j == good and right is not None else int(rng.choice(level))
                    up.append(parent)
                    tok.append(follow[depth] if j == good and right is not None else int(rng.integers(0, 300)))
                    new.append(len(up) - 1)
                right = new[good] if good < 3 and right is not None else None
                level = new
            trees.append(up)
            ids.append(tok)
        new = [len(t) for t in trees]
        starts = np.concatenate([[0], np.cumsum(new)])
        flat = np.concatenate(ids)
        sampled = m.greedy(m.logits(new, cached, tables, flat, np.arange(len(flat)), parents=np.concatenate(trees)))
        path, count, follow = dev_ints(np.zeros(len(flat))), dev_ints(np.zeros(4)), dev_ints(np.zeros(4))
        BR.gllm_op_tree_commit(dev_ints(flat), dev_ints(np.concatenate(trees)), sampled, dev_ints(starts), dev_ints(cached), d_tables, m.k, m.v, path, count, follow)
        path, count, follow = (x.cpu().numpy() for x in (path, count, follow))
        for s in range(4):
            way = path[starts[s]:starts[s] + count[s]]
            tokens[s] += [int(flat[starts[s] + j]) for j in way[1:]] + [int(follow[s])]
            cached[s] += int(count[s])
            accepted += int(count[s]) - 1
        passes += 1
    print(f"{passes} passes, {accepted} drafted tokens accepted", flush=True)
    assert accepted > passes
    for s in range(4):
        n = min(len(tokens[s]), len(want[s]))
        assert tokens[s][:n] == want[s][:n], s
        assert cached[s] == len(tokens[s]) - 1
    m.close()


def test_beam_search_over_forked_pages_is_beam_search_from_scratch():
    """Against beams that are computed anew from their first token at every step, selected by the oracle."""
    print("beam search", flush=True)
    rng = np.random.default_rng(33)
    W, keep, seqs, steps = 4, 8, 2, 20
    prompts = [rng.integers(0, 300, n).tolist() for n in (29, 14)]
    m, ref = Model(33, 200), Model(33, 200)
    free = [int(p) for p in rng.permutation(200)]
    first = [[free.pop() for _ in range(-(-len(p) // PAGE))] for p in prompts]
    width = 8
    def rows_of(tables):
        t = np.zeros((len(tables), width), dtype=np.int32)
        for i, r in enumerate(tables):
            t[i, :len(r)] = r
        return t
    lg = m.logits([len(p) for p in prompts], [0, 0], rows_of(first), np.concatenate(prompts), np.cumsum([len(p) for p in prompts]) - 1)
    lg = lg.repeat_interleave(W, 0)
    scores = torch.full((seqs, W), float("-inf"), device=DEV)
    scores[:, 0] = 0.0
    tables = [[list(f) for _ in range(W)] for f in first]
    beams = [[list(p) for _ in range(W)] for p in prompts]
    for step in range(steps):
        out = torch.empty(seqs, keep, device=DEV), dev_ints(np.zeros((seqs, keep))), dev_ints(np.zeros((seqs, keep)))
        BR.gllm_op_beam_select(lg, m.vocab, scores, *out)
        value, beam, token = (x.cpu().numpy() for x in out)
        # against all beams from scratch
        ids = [b for s in range(seqs) for b in beams[s]]
        scratch = np.arange(seqs * W * width).reshape(seqs * W, width) % 200
        full = ref.logits([len(b) for b in ids], [0] * len(ids), scratch, np.concatenate(ids), np.cumsum([len(b) for b in ids]) - 1)
        want = O.beam_select(full[:, :m.vocab].cpu().numpy(), scores.cpu().numpy(), keep)
        assert np.array_equal(beam[:, :W], want[1][:, :W]) and np.array_equal(token[:, :W], want[2][:, :W]), step
        assert np.abs(value - want[0]).max() <= 5e-2, step
        scores = out[0][:, :W].contiguous()
        src, dst, tables_new, beams_new = [], [], [], []
        for s in range(seqs):
            length, t_new, taken = len(beams[s][0]), [], set()
            partial = length % PAGE
            for w in range(W):
                b = int(beam[s, w])
                row = list(tables[s][b])
                if partial and b in taken:                  # the page is written next, and another beam goes on in it
                    page = free.pop()
                    src.append(row[-1])
                    dst.append(page)
                    row[-1] = page
                taken.add(b)
                if not partial:
                    row.append(free.pop())
                t_new.append(row)
            tables_new.append(t_new)
            beams_new.append([beams[s][int(beam[s, w])] + [int(token[s, w])] for w in range(W)])
        used = {p for t in tables_new for r in t for p in r}
        BR.gllm_op_copy_pages(m.k, m.v, src, dst)
        tables, beams = tables_new, beams_new
        free = [p for p in free if p not in used] + [p for p in range(200) if p not in used and p not in free]
        flat = [r for t in tables for r in t]
        lg = m.logits([1] * (seqs * W), [len(b) - 1 for s in range(seqs) for b in beams[s]], rows_of(flat), [b[-1] for s in range(seqs) for b in beams[s]], np.arange(seqs * W))
    assert len({tuple(b) for b in beams[0]}) == W
    m.close()
    ref.close()
