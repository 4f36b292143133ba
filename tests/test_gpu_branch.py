"""GPU parity of the operators for several continuations of one sequence (include/gllm_branch.h) against oracle/branch_oracle.py.

Tree attention: the weights of the softmax and the output are rounded to bf16 (2^-8 relative each, eps/2 of the type), the scores
summed in float32.  With A = sum p|v| and M the largest sum |q_i k_i| * scale of a row, an output is off by at most
2^-8 |out| + (2^-8 + 2 M (d + 8) 2^-24 + 2^-18) A: the middle term is what an error of a score does to p and to its sum (d products
and sums of 2^-24 each, twice: numerator and denominator), the last the exponentials and the sums over keys.
Beam selection: tokens and beams exact, scores to float32's 2^-24.  Commit and copies: bits."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import branch as BR
from gpu_util import DEV

pytestmark = pytest.mark.gpu
PAGE = 16


def dev_ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def random_tree(rng, n, kind):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "flat":
        return [-1] + [0] * (n - 1)
    if kind == "forest":
        return [-1 if i == 0 or rng.random() < 0.2 else int(rng.integers(0, i)) for i in range(n)]
    return [-1] + [int(rng.integers(max(0, i // 2 - 2), i)) for i in range(1, n)]


class Trees:
    """Inputs of one call: sequences of given cached lengths and trees over a pool with spare pages."""

    def __init__(self, heads, cached, trees, seed=0, spare=3, tail_rows=0, table_extra=0, pool_pages=None, perm_seed=None, q_pad=0):
        self.n_q, self.n_kv, self.d = heads
        self.cached, self.trees = list(cached), [list(t) for t in trees]
        self.starts = np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)
        self.parents = np.array([p for t in self.trees for p in t] + [0] * tail_rows, dtype=np.int32)
        rows = len(self.parents)
        g = torch.Generator(device=DEV).manual_seed(seed)
        pages = [max(1, -(-(max(c, 0) + len(t)) // PAGE)) for c, t in zip(cached, trees)]
        total = pool_pages or sum(pages) + spare
        order = np.random.default_rng(seed if perm_seed is None else perm_seed).permutation(total)
        self.tables = np.zeros((len(trees), max(pages) + table_extra), dtype=np.int32)
        at = 0
        for s, p in enumerate(pages):
            self.tables[s, :p] = order[at:at + p]
            at += p
        self.k = torch.empty(total, self.n_kv, self.d // 8, PAGE, 8, dtype=torch.bfloat16, device=DEV)
        self.v = torch.empty(total, self.n_kv, self.d, PAGE, dtype=torch.bfloat16, device=DEV)
        # contents by logical position, so that another order of the pages holds the same keys
        self.k.fill_(float("nan"))
        self.v.fill_(float("nan"))
        for s, p in enumerate(pages):
            self.k[self.tables[s, :p]] = torch.randn(p, *self.k.shape[1:], generator=g, device=DEV).bfloat16()
            self.v[self.tables[s, :p]] = torch.randn(p, *self.v.shape[1:], generator=g, device=DEV).bfloat16()
        q = torch.randn(rows, self.n_q * self.d + q_pad, generator=g, device=DEV).bfloat16()
        self.q = q[:, :self.n_q * self.d]
        self.out = torch.full((rows, self.n_q * self.d + q_pad), 7.0, dtype=torch.bfloat16, device=DEV)[:, :self.n_q * self.d]
        self.dev = [dev_ints(x) for x in (self.tables, self.cached, self.starts, self.parents)]

    def slot(self, s, pos):
        return int(self.tables[s, pos // PAGE]), pos % PAGE

    def run(self, max_nodes=None, scale=None, **kw):
        most = max_nodes or max(len(t) for t in self.trees)
        tables, cached, starts, parents = self.dev
        BR.gllm_op_tree_attention(self.q, self.k, self.v, tables, cached, starts, parents, self.out, most, scale=scale, **kw)
        torch.cuda.synchronize()
        return self.out

    def check(self, scale=None, max_nodes=256, label="", skip_rows=()):
        sc = self.d ** -0.5 if scale is None else scale
        q = f64(self.q).reshape(-1, self.n_q, self.d)
        ref, weight, mass = O.tree_attention(q, f64(self.k), f64(self.v), self.tables, self.cached, self.starts, self.parents, sc, max_nodes)
        got = f64(self.out).reshape(ref.shape)
        rows = np.ones(len(ref), dtype=bool)
        rows[self.starts[-1]:] = False
        rows[list(skip_rows)] = False
        assert np.all(got[self.starts[-1]:] == 7.0)                          # rows of no sequence stay as they were
        assert np.isfinite(got[rows]).all()
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * mass[..., None] * (self.d + 8) * 2.0 ** -24 + 2.0 ** -18) * weight
        off = np.abs(got - ref)[rows] - tol[rows]
        print(f"[parity] tree attention {label}: max abs {np.abs(got - ref)[rows].max():.3g}, of the bound {(np.abs(got - ref)[rows] / (tol[rows] + 1e-30)).max():.2f}", flush=True)
        assert off.max() <= 1e-30, label
        return ref, got


HEADS = [(4, 2, 64), (32, 8, 128), (10, 2, 128), (16, 1, 128), (8, 8, 64), (12, 4, 128), (7, 1, 64)]


@pytest.mark.parametrize("kind", ["tree", "chain", "flat", "forest"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_tree_attention(heads, kind):
    rng = np.random.default_rng(len(kind))
    cached = [0, 1, 15, 16, 31, 32, 33, 100, 517, 64, 95]
    sizes = [1, 5, 17, 2, 33, 1, 64, 12, 26, 31, 1]
    print(f"tree attention {heads} {kind}", flush=True)
    t = Trees(heads, cached, [random_tree(rng, n, kind) for n in sizes], seed=1)
    t.run()
    t.check(label=f"{heads} {kind}")


@pytest.mark.parametrize("n,c", [(1, 0), (1, 40), (2, 31), (65, 0), (128, 77), (200, 1000), (255, 31), (256, 63), (256, 3)])
@pytest.mark.parametrize("heads", [(4, 2, 64), (40, 8, 128)], ids=str)
def test_tree_sizes(heads, n, c):
    print(f"tree of {n} nodes behind {c}, {heads}", flush=True)
    rng = np.random.default_rng(n)
    t = Trees(heads, [c, 5], [random_tree(rng, n, "tree"), [-1, 0]], seed=n)
    t.run()
    t.check(label=f"{heads} {n} nodes behind {c}")


@pytest.mark.parametrize("seqs,c,n,heads", [(1, 20000, 3, (32, 8, 128)), (1, 9001, 40, (32, 8, 128)), (2, 6000, 64, (16, 2, 64)), (3, 4000, 1, (16, 1, 128)),
                                            (70, 300, 4, (4, 2, 64)), (300, 20, 2, (2, 1, 64))])
def test_tree_attention_long_and_many(seqs, c, n, heads):
    print(f"{seqs} sequences of {c} keys, {n} nodes, {heads}", flush=True)
    rng = np.random.default_rng(seqs)
    cached = [max(0, c - int(rng.integers(0, c // 3 + 1))) for _ in range(seqs)]
    trees = [random_tree(rng, int(rng.integers(1, n + 1)) if i else n, "tree") for i in range(seqs)]
    t = Trees(heads, cached, trees, seed=seqs)
    t.run()
    t.check(label=f"{seqs} x {c} keys")


def test_scores_of_any_size_and_scale():
    print("large scores", flush=True)
    t = Trees((8, 2, 64), [700, 40], [random_tree(np.random.default_rng(3), 20, "tree"), [-1, 0, 0]], seed=3)
    t.q.mul_(30.0)
    # ascending scores along the keys, so that the reference of the softmax has to move again and again
    for p in range(43):
        page, _ = t.slot(0, p * 16)
        t.k[page] *= 0.1 + 0.05 * p
    t.run(scale=0.5)
    t.check(scale=0.5, label="large scores")
    t.run(scale=1e-4)
    t.check(scale=1e-4, label="flat scores")


def test_unused_nodes_and_what_lies_around():
    """Parents that are no parents make a node and those below it unused: zeros, and nobody sees them, whatever their slots hold."""
    print("unused nodes", flush=True)
    bad = [[-1, 0, 2, 1, 2, 3, -2, 6, 9, 8, 1000000], [-2], [5, 0, 1], [-1, 0, 1, 2]]
    t = Trees((10, 2, 128), [37, 16, 0, 96], bad, seed=4, tail_rows=5, table_extra=2)
    nan = float("nan")
    for s, (c, tree) in enumerate(zip(t.cached, t.trees)):
        for i in range(len(tree)):
            if O.chain(tree, i) is None:
                page, slot = t.slot(s, c + i)
                t.k[page, :, :, slot] = nan
                t.v[page, :, :, slot] = float("inf")
        for pos in range(c + len(tree), -(-(c + len(tree)) // PAGE) * PAGE):     # slots that hold no data yet
            page, slot = t.slot(s, pos)
            t.k[page, :, :, slot] = nan
            t.v[page, :, :, slot] = nan
    t.tables[:, -2:] = 1 << 29                                                  # entries that no position needs
    t.dev[0] = dev_ints(t.tables)
    t.run()
    ref, got = t.check(label="unused nodes")
    rows = [i for s, tree in enumerate(bad) for i in range(t.starts[s], t.starts[s + 1]) if O.chain(tree, i - t.starts[s]) is None]
    assert len(rows) == 11 and not got[rows].any()


def test_values_that_are_not_finite_reach_only_those_that_see_them():
    print("NaN in one branch", flush=True)
    tree = [-1, 0, 0, 1, 2, 2, 3, 4]
    t = Trees((8, 2, 128), [45], [tree], seed=5)
    clean = f64(t.run()).copy()
    for node, what, pool in ((2, float("nan"), "v"), (6, float("inf"), "v"), (5, float("nan"), "k")):
        page, slot = t.slot(0, 45 + node)
        if pool == "k":
            t.k[page, 0, :, slot, 3] = what
        else:
            t.v[page, 0, 9, slot] = what
    got = f64(t.run()).reshape(8, 8, 128)
    clean = clean.reshape(8, 8, 128)
    see2, see6, see5 = [2, 4, 5, 7], [6], [5]
    for i in range(8):
        for h in range(8):
            mine = np.ones(128, dtype=bool)
            if h < 4 and i in see5:
                assert np.isnan(got[i, h]).all()
                continue
            if h < 4 and i in see2 + see6:
                assert not np.isfinite(got[i, h, 9])
                mine[9] = False
            # (a slot's value at place 3 of another element was set to zero for none: only column 9 changed)
            assert np.array_equal(got[i, h][mine], clean[i, h][mine]), (i, h)


def test_sequences_that_break_a_rule_receive_zeros():
    print("sequences out of the rules", flush=True)
    t = Trees((4, 2, 64), [20, -1, 20, 5, 100], [[-1, 0, 0], [-1, 0], [-1] * 9, [], [-1, 0, 1]], seed=6, tail_rows=2)
    t.dev[1] = dev_ints([20, -1, 2 ** 31 - 1, 5, 100])
    t.run(max_nodes=8)
    t.cached[2] = 2 ** 31 - 1
    t.check(label="out of the rules", max_nodes=8)
    got = f64(t.out)
    assert not got[3:14].any() and got[:3].any() and got[14:17].any()
    t.out.fill_(7.0)
    t.dev[1] = dev_ints([20, 3, 5, 5, 100])
    t.dev[0][0, 0], t.dev[0][4, 3] = -5, 2 ** 30                                # page ids that do not exist: read as the nearest
    t.run(max_nodes=8)
    t.cached = [20, 3, 5, 5, 100]
    t.tables[0, 0], t.tables[4, 3] = 0, t.k.shape[0] - 1
    t.k.nan_to_num_(0.5)
    t.v.nan_to_num_(0.5)
    t.out.fill_(7.0)
    t.run(max_nodes=8)
    t.check(label="page ids out of the pool", max_nodes=8)
    assert not f64(t.out)[5:14].any()                                           # nine nodes where eight are the most
    for starts in ([0, 3, 5, 14, 14, 99], [0, -3, 5, 14, 14, 17], [3, 2, 1, 0, 0, 0]):
        t.dev[2] = dev_ints(starts)
        t.run(max_nodes=8)                                                      # (row ranges outside the arrays are left out)
        assert np.all(f64(t.out)[17:] == 7.0)


def test_strides_streams_and_the_order_of_pages():
    print("strides, streams, order of pages", flush=True)
    rng = np.random.default_rng(7)
    trees = [random_tree(rng, n, "tree") for n in (26, 3, 40)]
    a = Trees((32, 8, 128), [2500, 10, 600], trees, seed=7)
    b = Trees((32, 8, 128), [2500, 10, 600], trees, seed=7, perm_seed=99, spare=40, q_pad=64)
    b.q.copy_(a.q)
    first = a.run().clone()
    assert torch.equal(a.run(), first) and torch.equal(b.run(), first)
    a.out.fill_(7.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.run(stream=side)
    assert torch.equal(a.out, first)
    ws = torch.empty(BR.gllm_op_tree_attention_workspace_bytes(32, 8, 128, 40), dtype=torch.uint8, device=DEV).fill_(255)
    a.out.fill_(7.0)
    assert torch.equal(a.run(workspace=ws), first)
    with pytest.raises(B.GllmError) as e:
        a.run(workspace=ws[:-16])
    assert e.value.status == -2
    with pytest.raises(B.GllmError):
        BR.gllm_op_tree_attention(a.q.float(), a.k, a.v, *a.dev, a.out, 40)


def test_a_pool_beyond_four_gigabytes():
    print("pool of more than 4 GiB", flush=True)
    d, n_kv = 128, 8
    pages = (1 << 32) // (n_kv * d * PAGE * 2) + 50
    t = Trees((8, 8, 128), [70], [[-1, 0, 0, 1]], seed=8)
    k, v = (torch.empty(pages, *x.shape[1:], dtype=torch.bfloat16, device=DEV) for x in (t.k, t.v))
    want = t.run().clone()
    for j in range(5):
        k[pages - 1 - j], v[pages - 1 - j] = t.k[t.tables[0, j]], t.v[t.tables[0, j]]
    t.k, t.v = k, v
    t.dev[0] = dev_ints([[pages - 1 - j for j in range(5)]])
    t.out.fill_(7.0)
    assert torch.equal(t.run(), want)


def test_tree_attention_replayed_from_a_graph():
    print("graph", flush=True)
    rng = np.random.default_rng(9)
    t = Trees((16, 2, 128), [900, 30, 300], [random_tree(rng, 30, "tree"), random_tree(rng, 7, "tree"), random_tree(rng, 1, "tree")], seed=9)
    ws = torch.empty(BR.gllm_op_tree_attention_workspace_bytes(16, 2, 128, 32), dtype=torch.uint8, device=DEV)
    t.run(max_nodes=32, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        BR.gllm_op_tree_attention(t.q, t.k, t.v, *t.dev, t.out, 32, workspace=ws)
    for cached in ([900, 30, 300], [100, 29, 310], [3, 0, 17]):
        t.dev[1].copy_(dev_ints(cached))
        t.cached = cached
        t.out.fill_(7.0)
        want = t.run(max_nodes=32).clone()
        t.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.out, want)
        t.check(label=f"replayed, {cached}")


@pytest.mark.parametrize("seqs,heads,most", [(65, (4, 2, 64), 2), (129, (16, 1, 128), 3), (1000, (2, 1, 64), 40), (4500, (2, 1, 64), 2)])
def test_more_sequences_than_a_wave_plans_for_itself(seqs, heads, most):
    """Some of them cut, some without rows, some that break a rule (zeros); and rows in no order (nothing written)."""
    print(f"{seqs} sequences, {heads}, at most {most} nodes", flush=True)
    rng = np.random.default_rng(seqs)
    cached = [int(rng.integers(0, 40)) for _ in range(seqs)]
    for s in rng.integers(0, seqs, 12):
        cached[s] = int(rng.integers(500, 5000))
    trees = [random_tree(rng, int(rng.integers(0, most + 1)) or 1, "tree") if rng.random() < 0.9 else [] for _ in range(seqs)]
    t = Trees(heads, cached, trees, seed=seqs, tail_rows=3)
    broken = [s for s in rng.integers(0, seqs, 5) if trees[s]]
    for s in broken:
        t.cached[s] = -1
    t.dev[1].copy_(dev_ints(t.cached))
    t.run(max_nodes=most)
    ref, got = t.check(max_nodes=most, label=f"{seqs} sequences")
    for s in broken:
        assert not got[t.starts[s]:t.starts[s + 1]].any()
    swapped = t.starts.copy()
    swapped[seqs // 2] = t.starts[-1]
    t.dev[2].copy_(dev_ints(swapped))
    t.out.fill_(7.0)
    t.run(max_nodes=most)
    assert bool((t.out == 7.0).all())


@pytest.mark.parametrize("heads", [(8, 2, 64), (16, 4, 128)], ids=str)
def test_any_bound_on_the_nodes_of_a_tree_and_two_calls_at_once(heads):
    """Trees of 1 to 4 nodes under bounds from 4 to 256: every kernel, with tiles that are mostly empty, over more sequences than a wave has
    lanes, a few of them cut; then two such calls on streams of their own."""
    rng = np.random.default_rng(21)
    cached = [int(rng.integers(0, 90)) for _ in range(80)] + [9000, 5001, 0, 2600]
    t = Trees(heads, cached, [random_tree(rng, int(rng.integers(1, 5)), "tree") for _ in cached], seed=21, tail_rows=2)
    whole = {}
    for most in (4, 8, 9, 64, 65, 127, 128, 256):
        print(f"{heads}, at most {most} nodes", flush=True)
        t.out.fill_(7.0)
        t.run(max_nodes=most)
        t.check(max_nodes=most, label=f"{heads}, at most {most} nodes")
        whole[most] = t.out.clone()
    torch.cuda.synchronize()
    pairs = []
    for most in (4, 128):
        s = torch.cuda.Stream()
        ws = torch.empty(BR.gllm_op_tree_attention_workspace_bytes(*heads, most), dtype=torch.uint8, device=DEV)
        pairs.append((most, s, ws, torch.full_like(t.out, 7.0)))
    torch.cuda.synchronize()
    for _ in range(4):
        for most, s, ws, out in pairs:
            BR.gllm_op_tree_attention(t.q, t.k, t.v, *t.dev, out, most, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for most, _, _, out in pairs:
        assert torch.equal(out, whole[most])


# ---- commit -----------------------------------------------------------------------------------------------------------------

class Commit:
    def __init__(self, heads, layers, cached, trees, seed=0, accept=0.8, vocab=6, duplicates=True):
        rng = np.random.default_rng(seed)
        self.n_kv, self.d = heads
        self.trees, self.cached = trees, np.array(cached, dtype=np.int32)
        self.starts = np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)
        self.parents = np.array([p for t in trees for p in t], dtype=np.int32)
        rows = len(self.parents)
        self.tokens = rng.integers(0, vocab if duplicates else 10 ** 6, rows).astype(np.int32)
        self.sampled = rng.integers(0, vocab, rows).astype(np.int32)
        for s, t in enumerate(trees):                                            # long walks
            for i, p in enumerate(t):
                if 0 <= p < i and rng.random() < accept:
                    self.sampled[self.starts[s] + p] = self.tokens[self.starts[s] + i]
        pages = [-(-(c + len(t)) // PAGE) for c, t in zip(cached, trees)]
        total = sum(pages) + 4
        order = rng.permutation(total)
        self.tables = np.full((len(trees), max(pages) + 1), 1 << 30, dtype=np.int32)
        at = 0
        for s, p in enumerate(pages):
            self.tables[s, :p] = order[at:at + p]
            at += p
        g = torch.Generator(device=DEV).manual_seed(seed)
        bits = lambda *shape: torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device=DEV, dtype=torch.int16).view(torch.bfloat16)
        self.k, self.v = bits(layers, total, self.n_kv, self.d // 8, PAGE, 8), bits(layers, total, self.n_kv, self.d, PAGE)

    def run(self, pools=True, stream=None):
        path, count, follow = (torch.full((n,), -7, dtype=torch.int32, device=DEV) for n in (len(self.parents), len(self.cached), len(self.cached)))
        BR.gllm_op_tree_commit(dev_ints(self.tokens), dev_ints(self.parents), dev_ints(self.sampled), dev_ints(self.starts), dev_ints(self.cached),
                               dev_ints(self.tables), self.k if pools else None, self.v if pools else None, path, count, follow, stream=stream)
        torch.cuda.synchronize()
        return [x.cpu().numpy() for x in (path, count, follow)]

    def check(self):
        bits = lambda t: t.view(torch.int16).cpu().numpy()
        k, v = bits(self.k).copy(), bits(self.v).copy()
        want = O.tree_commit(self.tokens, self.parents, self.sampled, self.starts, self.cached, self.tables, k, v)
        before = self.k.clone(), self.v.clone()
        for a, b in zip(self.run(pools=False), want):
            assert np.array_equal(a, b)
        assert torch.equal(before[0].view(torch.int16), self.k.view(torch.int16)) and torch.equal(before[1].view(torch.int16), self.v.view(torch.int16))
        for a, b in zip(self.run(), want):
            assert np.array_equal(a, b)
        assert np.array_equal(bits(self.k), k) and np.array_equal(bits(self.v), v)
        return want


@pytest.mark.parametrize("heads,layers", [((2, 64), 1), ((8, 128), 3), ((1, 128), 5), ((3, 64), 2)])
@pytest.mark.parametrize("kind", ["tree", "chain", "flat", "forest"])
def test_commit(heads, layers, kind):
    print(f"commit {heads} {layers} {kind}", flush=True)
    rng = np.random.default_rng(11)
    sizes = [1, 2, 26, 64, 65, 130, 256, 9, 40]
    c = Commit(heads, layers, [0, 15, 16, 100, 31, 47, 8, 200, 1], [random_tree(rng, n, kind) for n in sizes], seed=layers, accept=0.95)
    path, count, _ = c.check()
    print(f"accepted {count.tolist()}", flush=True)


def test_commit_moves_long_paths_in_order():
    """A chain whose second node is a dud: every accepted node moves by one slot, through many pages."""
    print("commit of a shifted chain", flush=True)
    tree = [-1, 0, 0] + list(range(2, 255))
    c = Commit((2, 128), 2, [13, 0], [tree, tree], seed=12, duplicates=False)
    for s in range(2):
        r0 = c.starts[s]
        for i, p in enumerate(tree):
            if i > 1:
                c.sampled[r0 + p] = c.tokens[r0 + i]
    _, count, _ = c.check()
    assert count.tolist() == [255, 255]


@pytest.mark.parametrize("heads,layers,seqs", [((16, 64), 37, 9), ((7, 128), 61, 20)])
def test_commit_of_many_layers_and_sequences(heads, layers, seqs):
    """More (sequence, layer, head)s than one workgroup each, and not a whole number of them to a workgroup."""
    print(f"commit {heads} {layers} layers {seqs} sequences", flush=True)
    rng = np.random.default_rng(layers)
    c = Commit(heads, layers, [int(rng.integers(0, 60)) for _ in range(seqs)], [random_tree(rng, int(rng.integers(1, 30)), "tree") for _ in range(seqs)],
               seed=layers, accept=0.95)
    _, count, _ = c.check()
    print(f"accepted {count.tolist()}", flush=True)


def test_commit_where_a_rule_is_broken():
    print("commit out of the rules", flush=True)
    c = Commit((2, 64), 2, [5, 3, 0, 40, 7], [[-1, 0, 0, 1], [0, 0, 1], [-1, 5, 1, -3, 0], [-1, 0, 0, 2, 3], [-1, 0, 0, 2]], seed=13, accept=1.0)
    c.tables[3, 2] = -1                                                          # moves from and to this page are left out
    c.check()
    c.cached = np.array([-1, 3, 2 ** 31 - 1, 41, 16 * c.tables.shape[1] - 3], dtype=np.int32)
    _, count, follow = c.check()
    assert count[[0, 1, 2, 4]].tolist() == [0] * 4 and follow[[0, 1, 2, 4]].tolist() == [-1] * 4


def test_commit_on_a_stream_and_replayed_from_a_graph():
    print("commit from a graph", flush=True)
    rng = np.random.default_rng(31)
    c = Commit((2, 128), 2, [13, 40, 0], [random_tree(rng, n, "tree") for n in (60, 7, 200)], seed=31, accept=0.9)
    pools = c.k.clone(), c.v.clone()
    ints = [dev_ints(x) for x in (c.tokens, c.parents, c.sampled, c.starts, c.cached, c.tables)]
    out = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (len(c.parents), 3, 3)]
    call = lambda stream=None: BR.gllm_op_tree_commit(*ints, c.k, c.v, *out, stream=stream)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    bits = lambda t: t.view(torch.int16).cpu().numpy()
    for i in range(3):
        if i:
            c.sampled = rng.permutation(c.sampled)                               # other tokens at every replay
        ints[2].copy_(dev_ints(c.sampled))
        for x, y in zip((c.k, c.v), pools):
            x.copy_(y)
        k, v = bits(c.k).copy(), bits(c.v).copy()
        want = O.tree_commit(c.tokens, c.parents, c.sampled, c.starts, c.cached, c.tables, k, v)
        for x in out:
            x.fill_(-7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, want))
        assert np.array_equal(bits(c.k), k) and np.array_equal(bits(c.v), v)
        print(f"replay {i}: {want[1].tolist()} accepted", flush=True)


# ---- beams --------------------------------------------------------------------------------------------------------------------

def check_beams(x, scores, keep, vocab=None, label="", dev=None, **kw):
    """x: float32 [S*W][V] on the host, checked against the oracle."""
    vocab = vocab or x.shape[1]
    s = scores.shape[0]
    want = O.beam_select(x[:, :vocab], scores, keep)
    lg = torch.from_numpy(x).to(DEV) if dev is None else dev
    out = torch.full((s, keep), 7.0, device=DEV), dev_ints(np.full((s, keep), -9)), dev_ints(np.full((s, keep), -9))
    BR.gllm_op_beam_select(lg, vocab, torch.from_numpy(scores.astype(np.float32)).to(DEV), *out, **kw)
    torch.cuda.synchronize()
    got = [t.cpu().numpy() for t in out]
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2]), label
    there = want[1] >= 0
    assert np.all(got[0][~there] == -np.inf)
    assert np.all(np.abs(got[0][there] - want[0][there]) <= 2.0 ** -24 * 1.001 * np.abs(want[0][there]) + 1e-9), label
    return got


@pytest.mark.parametrize("seqs,beams,vocab,keep", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 63, 6), (3, 4, 1000, 8), (1, 32, 4097, 64), (5, 2, 5003, 4), (16, 5, 50261, 10),
                                                   (1, 4, 128256, 8), (3, 8, 152064, 16), (1, 1, 300001, 64), (40, 1, 777, 2),
                                                   (2, 16, 197294, 26), (8, 32, 20000, 64), (6, 32, 33333, 40), (300, 1, 9001, 5)])
def test_beam_select(seqs, beams, vocab, keep):
    print(f"beams {seqs} x {beams}, {vocab}, {keep}", flush=True)
    rng = np.random.default_rng(vocab)
    x = (rng.standard_normal((seqs * beams, -(-vocab // 256) * 256)) * 4.5).astype(np.float32)
    x[:, vocab:] = 1e9                                                           # columns past the vocabulary
    scores = (-rng.random((seqs, beams)) * 5 - 3).astype(np.float32)
    check_beams(x, scores, keep, vocab, label="aligned rows")
    odd = torch.from_numpy(np.concatenate([x, np.full((x.shape[0], 3), 1e9, np.float32)], 1)).to(DEV)
    check_beams(x, scores, keep, vocab, label="rows off a 16-byte boundary", dev=odd)


@pytest.mark.parametrize("vocab", [7, 900, 40000])
def test_equal_scores_go_by_beam_and_token(vocab):
    print(f"ties, {vocab}", flush=True)
    rng = np.random.default_rng(vocab)
    same = np.zeros((6, vocab), dtype=np.float32)
    check_beams(same, np.full((2, 3), -1.0, dtype=np.float32), 9, label="all alike")
    few = rng.integers(0, 4, (6, vocab)).astype(np.float32)
    few[3:] = few[:3]                                                            # beams alike, so that their sums are
    check_beams(few, np.full((2, 3), -1.0, dtype=np.float32), 12, label="few values")
    check_beams(few[[0, 0, 0]] * -0.0, np.full((1, 3), -1.0, dtype=np.float32), 12, label="zeros of either sign")
    up = np.arange(vocab, dtype=np.float32)[None].repeat(4, 0)
    check_beams(up * 1e-3, np.zeros((1, 4), dtype=np.float32), 12, label="ascending")
    check_beams(-up * 1e-3, np.zeros((1, 4), dtype=np.float32), 64, label="descending")


def test_masked_and_odd_logits():
    print("masked logits", flush=True)
    rng = np.random.default_rng(3)
    inf, low = np.inf, np.finfo(np.float32).min
    x = (rng.standard_normal((12, 6000)) * 4).astype(np.float32)
    x[0, 5:] = -inf                     # five candidates
    x[1] = -inf                         # none
    x[2, ::2] = np.nan
    x[3] = np.nan
    x[4, [17, 4000]] = inf              # forced tokens share the probability
    x[5, 100:] = low                    # the type's lowest value is a number
    x[6] = low
    x[7] *= 1e30
    x[8, 3000] = 200.0                  # far above the rest, behind the first pass
    x[9, 5999] = 3e38
    scores = np.array([[-1, -2], [-3, -1], [-2, -2], [-inf, -4], [-1, -0.5], [np.nan, inf]], dtype=np.float32)
    got = check_beams(x, scores, 8)
    assert got[1][5].tolist() == [-1] * 8
    check_beams(x[:6], scores[:3], 64, label="more than there are")
    first = np.full((2, 4), -inf, dtype=np.float32)
    first[:, 0] = 0.0                   # the first step of a search: one beam
    got = check_beams(x[[7, 8, 9, 10, 8, 9, 10, 11]] * np.float32(1e-6), first, 8)
    assert not got[1].any()


def test_beam_select_streams_graph_and_workspace():
    print("beams: stream, graph", flush=True)
    rng = np.random.default_rng(4)
    x = (rng.standard_normal((24, 20000)) * 4).astype(np.float32)
    scores = -rng.random((3, 8)).astype(np.float32)
    ws = torch.empty(BR.gllm_op_beam_select_workspace_bytes(3, 8, 20000, 16), dtype=torch.uint8, device=DEV).fill_(255)
    want = check_beams(x, scores, 16, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    check_beams(x, scores, 16, stream=side)
    with pytest.raises(B.GllmError) as e:
        check_beams(x, scores, 16, workspace=ws[:-16])
    assert e.value.status == -2
    lg, sc = torch.from_numpy(x).to(DEV), torch.from_numpy(scores).to(DEV)
    out = torch.empty(3, 16, device=DEV), dev_ints(np.zeros((3, 16))), dev_ints(np.zeros((3, 16)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        BR.gllm_op_beam_select(lg, 20000, sc, *out, workspace=ws)
    for k in range(3):
        y = np.roll(x, k * 77, axis=1)
        lg.copy_(torch.from_numpy(y))
        g.replay()
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in out]
        ref = check_beams(y, scores, 16)
        assert all(np.array_equal(a, b) for a, b in zip(got, ref))


# ---- page copies ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,layers,n", [((2, 64), 1, 1), ((8, 128), 3, 5), ((1, 64), 2, 460), ((3, 128), 20, 17)])
def test_copy_pages(heads, layers, n):
    print(f"copy {heads} {layers} layers {n} pages", flush=True)
    n_kv, d = heads
    rng = np.random.default_rng(n)
    total = 2 * n + 3
    g = torch.Generator(device=DEV).manual_seed(n)
    bits = lambda *shape: torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device=DEV, dtype=torch.int16).view(torch.bfloat16)
    k, v = bits(layers, total, n_kv, d // 8, PAGE, 8), bits(layers, total, n_kv, d, PAGE)
    ids = rng.permutation(total)
    src, dst = ids[rng.integers(0, n, n)], ids[n:2 * n]
    want = [x.view(torch.int16).clone() for x in (k, v)]
    for w in want:
        w[:, dst] = w[:, src]
    BR.gllm_op_copy_pages(k, v, src, dst)
    torch.cuda.synchronize()
    for w, x in zip(want, (k, v)):
        assert torch.equal(w, x.view(torch.int16))
    for bad_src, bad_dst, status in (([0], [total], -3), ([-1], [0], -3), ([0, 0], [1, 1], -4), ([0, 1], [1, 2], -4)):
        with pytest.raises(B.GllmError) as e:
            BR.gllm_op_copy_pages(k, v, bad_src, bad_dst)
        assert e.value.status == status
    BR.gllm_op_copy_pages(k, v, [], [])
    torch.cuda.synchronize()
    for w, x in zip(want, (k, v)):
        assert torch.equal(w, x.view(torch.int16))


def test_copies_on_a_stream_and_replayed_from_a_graph():
    print("copies from a graph", flush=True)
    k = torch.arange(2 * 9 * 2 * 8 * PAGE * 8, device=DEV).remainder(251).bfloat16().reshape(2, 9, 2, 8, PAGE, 8)
    v = torch.arange(2 * 9 * 2 * 64 * PAGE, device=DEV).remainder(241).bfloat16().reshape(2, 9, 2, 64, PAGE)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    BR.gllm_op_copy_pages(k, v, [0, 0], [1, 2], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(k[:, 1], k[:, 0]) and torch.equal(v[:, 2], v[:, 0])
    ids = [np.array([3, 4], dtype=np.int32), np.array([5, 6], dtype=np.int32)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        BR.gllm_op_copy_pages(k, v, *ids)
    ids[0][:], ids[1][:] = 7, 8                                                  # (the pages of the graph are those of the call)
    for i in range(3):
        k[:, 3] += 1
        want = [x.clone() for x in (k, v)]
        for w in want:
            w[:, [5, 6]] = w[:, [3, 4]]
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
