"""GPU tests of the operators for several continuations of one sequence (include/gllm_branch.h) where their sizes send them through other
kernels and paths than tests/test_gpu_branch.py does with the same contents; helpers and bounds are that file's."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV, to_dev_bits
from helpers import layer_weights_np
from oracle import branch_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import branch as BR
from paper_2504_14775_amd import synth
from test_gpu_branch import Trees, check_beams, dev_ints, f64
from test_gpu_branch_loop import Model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["-inf", "nan", "both"])
@pytest.mark.parametrize("beams,vocab,keep", [(8, 128256, 16), (4, 152064, 8), (32, 33333, 64), (2, 700001, 64)])
def test_beams_without_any_continuation_among_many_candidates(beams, vocab, keep, what):
    """Whole rows of logits that are no continuations, of beams whose score is the best: the first, a middle one, several, all but one, all.
    More than 1024 places of kept logits a sequence."""
    rng = np.random.default_rng(vocab + keep)
    x = (rng.standard_normal((beams, vocab)) * 4.5).astype(np.float32)
    rows = [[0], [beams // 2], sorted({0, beams // 2, beams - 1}), list(range(1, beams)), list(range(beams))]
    for empty in rows:
        print(f"{beams} beams, {vocab}, keep {keep}: {what} in rows {empty}", flush=True)
        y, scores = x.copy(), (-rng.random((1, beams)) * 3 - 20).astype(np.float32)
        for i, r in enumerate(empty):
            y[r] = -np.inf if what == "-inf" or (what == "both" and i % 2) else np.nan
            scores[0, r] = -1.0
        if what == "both" and len(empty) == 1:
            y[empty[0], ::2] = -np.inf
        got = check_beams(y, scores, keep, label=f"{what} in rows {empty}")
        assert len(empty) < beams or got[1].max() == -1


@pytest.mark.parametrize("beams,vocab,keep", [(8, 128256, 16), (32, 33333, 64)])
def test_odd_logits_among_many_candidates(beams, vocab, keep):
    """Rows with continuations in one segment only, with fewer than are kept, with +infinity, with the type's lowest value, far apart."""
    rng = np.random.default_rng(keep)
    x = (rng.standard_normal((3 * beams, vocab)) * 4.5).astype(np.float32)
    scores = (-rng.random((3, beams)) * 3 - 2).astype(np.float32)
    print(f"odd logits, {beams} beams, {vocab}, keep {keep}", flush=True)
    x[0, :-7] = -np.inf
    x[1, 5:] = np.nan
    x[2, [17, vocab // 2, vocab - 1]] = np.inf
    x[3, 100:] = np.finfo(np.float32).min
    x[beams:2 * beams, 3:] = -np.inf                # fewer in the whole sequence than are kept
    x[beams + 1] = np.nan
    x[2 * beams] *= 1e30
    x[2 * beams + 1, vocab - 2] = 3e38
    scores[2, 2] = -np.inf
    scores[2, 3] = np.nan
    check_beams(x, scores, keep, label="odd logits")
    first = np.full((3, beams), -np.inf, dtype=np.float32)
    first[:, beams - 1] = 0.0                       # one beam
    got = check_beams(x, first, keep, label="one beam")
    assert set(got[1].flatten()) <= {beams - 1, -1}


@pytest.mark.parametrize("beams,vocab", [(4, 20000), (8, 152064), (32, 60000)])
def test_beams_of_equal_sums_tie_wherever_their_largest_logit_stands(beams, vocab):
    """Every row's weights are ones (its logits 0 but for one of 1e-20, at another place in each), so all continuations tie in 64 bits."""
    print(f"equal sums, {beams} beams, {vocab}", flush=True)
    x = torch.zeros(beams, vocab, device=DEV)
    for b in range(beams):
        x[b, (b + 1) * vocab // beams - 1] = 1e-20
    scores = torch.full((1, beams), -2.0, device=DEV)
    out = torch.empty(1, 8, device=DEV), dev_ints(np.zeros((1, 8))), dev_ints(np.zeros((1, 8)))
    BR.gllm_op_beam_select(x, vocab, scores, *out)
    torch.cuda.synchronize()
    assert (out[1] == 0).all()
    want = -2.0 - np.log(vocab)
    assert np.all(np.abs(out[0].cpu().numpy() - want) <= 2.0 ** -24 * 1.001 * abs(want) + 1e-9)


@pytest.mark.parametrize("seqs,beams,vocab,keep", [(2, 3, 700, 8), (1, 4, 60000, 8), (1, 8, 128256, 16), (2, 32, 33333, 64), (1, 1, 300001, 64)])
def test_sums_that_agree_in_64_bits_go_by_beam_logit_and_token(seqs, beams, vocab, keep):
    """Logits whose differences the sum swallows: next to nothing beside log(vocabulary), or behind a score of -1e18 (64 bits there are 128 apart)."""
    print(f"equal sums, {seqs} x {beams} beams, {vocab}, keep {keep}", flush=True)
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((seqs * beams, vocab)).astype(np.float32)
    x[:, ::7] = x[:, :1]                            # equal ones among them
    check_beams(x * np.float32(1e-20), np.full((seqs, beams), -1.0, dtype=np.float32), keep, label="small logits")
    scores = np.full((seqs, beams), -1e18, dtype=np.float32)
    check_beams(x, scores, keep, label="large scores")
    scores[:, beams // 2] = -1e17
    got = check_beams(x, scores, keep, label="one beam ahead")
    assert (got[1] == beams // 2).all()


@pytest.mark.parametrize("beams,vocab,keep", [(3, 9000, 4), (8, 128256, 16), (2, 300001, 64)])
def test_more_logits_of_infinity_than_are_kept(beams, vocab, keep):
    """Infinities that fill the lists at once or bit by bit, among numbers of any size: they share the probability, the lowest tokens come first."""
    print(f"infinities, {beams} beams, {vocab}, keep {keep}", flush=True)
    rng = np.random.default_rng(vocab)
    for step in (1, 3, vocab // (keep + 1)):
        x = (rng.standard_normal((beams, vocab)) * 4.5).astype(np.float32)
        x[:, ::step] = np.inf
        x[beams - 1] = np.sort(rng.standard_normal(vocab) * 1e37)
        x[beams - 1, vocab // 2:] = np.finfo(np.float32).max
        check_beams(x, (-rng.random((1, beams)) * 3 - 2).astype(np.float32), keep, label=f"every {step}th")


def test_positions_up_to_where_32_bits_end():
    """One sequence of nearly 2^31 positions, every page of it the same one, and one that goes past: its rows receive zeros, its walk is empty.
    The sums of a column are of 2^26 / 512 blocks at most in a wave, of 2^-24 each, in numerator and denominator."""
    print("2^31 positions", flush=True)
    limit, n, d = 2 ** 31 - 64, 3, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    k = torch.randn(2, 1, d // 8, 16, 8, generator=g, device=DEV).bfloat16()
    v = torch.randn(2, 1, d, 16, generator=g, device=DEV).bfloat16()
    q = torch.randn(n, 2 * d, generator=g, device=DEV).bfloat16()
    tables = torch.zeros(1, 2 ** 27, dtype=torch.int32, device=DEV)
    starts, parents, out = dev_ints([0, n]), dev_ints([-1, 0, 0]), torch.full((n, 2 * d), 7.0, dtype=torch.bfloat16, device=DEV)
    BR.gllm_op_tree_attention(q, k, v, tables, dev_ints([limit - n]), starts, parents, out, n)
    torch.cuda.synchronize()
    kk, vv, qq = k[0, 0].double().permute(1, 0, 2).reshape(16, d), v[0, 0].double().t(), q.double().view(n, 2, d)
    x = torch.einsum("rhd,kd->rhk", qq.cpu(), kk.cpu()) * d ** -0.5
    p = torch.softmax(x, -1)
    ref, weight = (torch.einsum("rhk,kd->rhd", p, y.cpu()) for y in (vv, vv.abs()))
    mass = torch.einsum("rhd,kd->rhk", qq.cpu().abs(), kk.cpu().abs()).amax(-1, keepdim=True) * d ** -0.5
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * mass * (d + 8) * 2.0 ** -24 + 2.0 ** -18 + 2 * 2.0 ** 17 / 2 ** 24) * weight
    off = (out.double().cpu().view(n, 2, d) - ref).abs()
    print(f"[parity] 2^31 positions: max abs {off.max():.3g}, of the bound {(off / tol).max():.2f}", flush=True)
    assert (off <= tol).all()
    BR.gllm_op_tree_attention(q, k, v, tables, dev_ints([limit - n + 1]), starts, parents, out, n)
    torch.cuda.synchronize()
    assert not out.any()
    # the walk: the second child is accepted, from the last slots there are
    page, slot = (limit - n) // 16, (limit - n) % 16
    assert slot + n == 16
    tables[0, page] = 1
    pools = torch.randn(1, 2, 1, d // 8, 16, 8, generator=g, device=DEV).bfloat16(), torch.randn(1, 2, 1, d, 16, generator=g, device=DEV).bfloat16()
    want = [x.clone() for x in pools]
    want[0][:, 1, :, :, slot + 1], want[1][:, 1, :, :, slot + 1] = want[0][:, 1, :, :, slot + 2], want[1][:, 1, :, :, slot + 2]
    for cached, result in ((limit - n, [0, 2, -1, 2, 8]), (limit - n + 1, [-1, -1, -1, 0, -1]), (2 ** 31 - 1, [-1, -1, -1, 0, -1])):
        path, count, follow = dev_ints([-7] * n), dev_ints([-7]), dev_ints([-7])
        BR.gllm_op_tree_commit(dev_ints([5, 6, 7]), parents, dev_ints([7, 9, 8]), starts, dev_ints([cached]), tables, *pools, path, count, follow)
        torch.cuda.synchronize()
        assert path.tolist() + count.tolist() + follow.tolist() == result
        assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])


def test_parents_that_are_no_32_bit_numbers_are_refused():
    print("parents modulo 2^32", flush=True)
    m = Model(5, 8, layers=1)
    x = torch.zeros(3, m.shape.hidden, dtype=torch.bfloat16, device=DEV)
    for bad in ([-1, 1 << 32, 0], [-1, 0, (1 << 32) + 1], [(1 << 32) - 1, 0, 0], [-1, 0.5, 1], [-1, 0, 1 << 70]):
        with pytest.raises(B.GllmError) as e:
            m.stage.forward_tree([3], [0], np.zeros((1, 1)), bad, x, torch.empty_like(x))
        assert e.value.status == -1
    m.stage.forward_tree([3], [0], np.zeros((1, 1)), np.array([-1, 0, 0]), x, torch.empty_like(x))
    m.close()


def test_the_stage_reads_parents_only_behind_lengths_that_hold():
    """How many parents there are goes by the lengths: one that is refused is named, not the parents in front of it."""
    print("parents and lengths", flush=True)
    m = Model(6, 8, layers=1)
    x = torch.zeros(4, m.shape.hidden, dtype=torch.bfloat16, device=DEV)
    for new, cached, status in (([3, -1], [0, 0], -1), ([1, 1, 0], [0, 0, 0], -1), ([1, 1], [0, -1], -1), ([1, 1], [0, 1 << 20], -2)):
        with pytest.raises(B.GllmError) as e:
            m.stage.forward_tree(new, cached, np.zeros((len(new), 1)), [5] * sum(new), x, torch.empty_like(x))
        assert e.value.status == status and "parent" not in e.value.message, e.value.message
    m.close()


def test_tensors_of_other_dimensions_are_refused():
    print("dimensions", flush=True)
    i, b = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(4, 128, dtype=torch.bfloat16, device=DEV)
    k, v = torch.zeros(1, 3, 2, 8, 16, 8, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 3, 2, 64, 16, dtype=torch.bfloat16, device=DEV)
    x, f = torch.zeros(8, 100, device=DEV), torch.zeros(2, 4, device=DEV)
    attention = dict(q=b, k_pool=k[0], v_pool=v[0], block_tables=i.view(1, 4), cached_len=i[:1], row_start=i[:2], parents=i, out=b.clone(), max_nodes=4)
    commit = dict(tokens=i, parents=i, sampled=i, row_start=i[:2], cached_len=i[:1], block_tables=i.view(1, 4), k_pool=k, v_pool=v, path=i.clone(), count=i[:1], next_token=i[:1])
    beams = dict(logits=x, vocab=100, scores=f, out_scores=f.clone(), out_beams=f.int(), out_tokens=f.int())
    for call, args, names in ((BR.gllm_op_tree_attention, attention, ("q", "out", "block_tables")), (BR.gllm_op_tree_commit, commit, ("block_tables",)),
                              (BR.gllm_op_beam_select, beams, ("logits", "scores", "out_scores", "out_beams", "out_tokens"))):
        for name in names:
            for other in (args[name].reshape(-1)[0], args[name].reshape(-1), args[name][None]):
                with pytest.raises(B.GllmError) as e:
                    call(**{**args, name: other})
                assert e.value.status == -1, name
    for name in ("cached_len", "row_start", "parents"):
        with pytest.raises(B.GllmError) as e:
            BR.gllm_op_tree_attention(**{**attention, name: i[0]})
        assert e.value.status == -1, name


@pytest.mark.parametrize("cached", [58, 3003])
@pytest.mark.parametrize("heads,most", [((2, 2, 64), 8), ((2, 2, 128), 8), ((8, 2, 128), 8), ((8, 2, 64), 16), ((8, 2, 128), 16), ((8, 2, 128), 65), ((8, 2, 64), 128),
                                        ((8, 2, 128), 128), ((32, 2, 128), 256)], ids=str)
def test_values_that_are_not_finite_in_every_kernel(heads, most, cached):
    """Tiles of 16, 32, 64 and 128 columns, uncut and cut keys, nodes in two blocks: keys and values of nodes, and a value of the prefix in the
    tree's first block, that are not finite change the rows and dims that see them only, the others not by a bit."""
    print(f"not finite, {heads}, at most {most} nodes, {cached} cached", flush=True)
    n_q, n_kv, d = heads
    g = n_q // n_kv
    tree = [-1, 0, 0, 1, 2, 2, 3, 4]
    t = Trees(heads, [cached], [tree], seed=most)
    clean = f64(t.run(max_nodes=most)).reshape(8, n_q, d).copy()
    assert np.isfinite(clean).all()
    nan, inf = float("nan"), float("inf")
    hit = np.zeros(clean.shape, dtype=bool)
    for node, what, dim in ((2, nan, 9), (6, inf, d - 3), (1, -inf, d // 2 + 1)):
        page, slot = t.slot(0, cached + node)
        t.v[page, 0, dim, slot] = what
        see = [i for i in range(8) if node in O.chain(tree, i)]
        hit[see, :g, dim] = True
    page, slot = t.slot(0, cached - 3)
    t.v[page, 1, d - 1, slot] = nan
    hit[:, g:2 * g, d - 1] = True
    page, slot = t.slot(0, cached + 5)
    t.k[page, 1, :, slot, 3] = nan
    hit[5, g:2 * g] = True
    got = f64(t.run(max_nodes=most)).reshape(8, n_q, d)
    assert not np.isfinite(got[hit]).any()
    assert np.array_equal(got[~hit], clean[~hit])


def test_many_candidates_from_a_graph_and_two_calls_at_once():
    """The path of many kept logits: a workspace that holds anything, replays with other logits, two calls on streams of their own."""
    print("many candidates: graph, streams", flush=True)
    rng = np.random.default_rng(41)
    vocab, keep = 128256, 16
    x = (rng.standard_normal((16, vocab)) * 4.5).astype(np.float32)
    x[3] = -np.inf
    scores = -rng.random((2, 8)).astype(np.float32)
    size = BR.gllm_op_beam_select_workspace_bytes(2, 8, vocab, keep)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255)
    check_beams(x, scores, keep, workspace=ws)
    lg, sc = torch.from_numpy(x).to(DEV), torch.from_numpy(scores).to(DEV)
    new = lambda: (torch.full((2, keep), 7.0, device=DEV), dev_ints(np.full((2, keep), -9)), dev_ints(np.full((2, keep), -9)))
    out = new()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        BR.gllm_op_beam_select(lg, vocab, sc, *out, workspace=ws)
    for shift in (0, 77, 9001):
        y = np.roll(x, shift, axis=1)
        if shift:
            y[3], y[12] = rng.standard_normal(vocab), np.nan
        lg.copy_(torch.from_numpy(y))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        ref = check_beams(y, scores, keep, label=f"replayed, {shift}")
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, ref))
    calls = [(torch.cuda.Stream(), torch.from_numpy(z).to(DEV), torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255), new()) for z in (x, np.roll(x, 5, axis=1))]
    torch.cuda.synchronize()
    for _ in range(4):
        for stream, z, w, o in calls:
            BR.gllm_op_beam_select(z, vocab, sc, *o, workspace=w, stream=stream)
    torch.cuda.synchronize()
    for _, z, _, o in calls:
        ref = check_beams(z.cpu().numpy(), scores, keep)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(o, ref))


def test_the_stage_over_more_trees_than_a_wave_plans_for_itself():
    """70 trees and a few decode rows, some of the trees behind keys that are cut: every path from a root to a leaf against the oracle, within
    the tolerance of tests/test_gpu_branch_loop.py."""
    print("stage over 70 trees", flush=True)
    rng = np.random.default_rng(70)
    shape = dataclasses.replace(synth.SHAPES["tiny"], num_layers=1, name="trees")
    weights = layer_weights_np(shape, 9)
    trees = [[-1] if s % 12 == 5 else [-1, 0, 0] + [int(rng.integers(0, i)) for i in range(3, int(rng.integers(3, 8)))] for s in range(76)]
    cached = [int(rng.integers(400, 700)) if s % 15 == 3 else int(rng.integers(0, 50)) for s in range(76)]
    new = [len(t) for t in trees]
    assert sum(n > 1 for n in new) >= 65
    pages = [-(-(c + n) // 16) for c, n in zip(cached, new)]
    order = rng.permutation(sum(pages) + 2)
    tables, at = np.zeros((76, max(pages)), dtype=np.int32), 0
    for s, p in enumerate(pages):
        tables[s, :p] = order[at:at + p]
        at += p
    k0, v0 = (synth.bf16_bits(x).copy() for x in synth.make_pool(shape, 9, len(order)))
    hidden = synth.bf16_bits(synth.make_hidden(shape, 9, sum(new)))
    stage = B.Stage(B.make_config(shape, sum(new), 76, max(pages), max(pages) * 16))
    stage.bind_workspace(torch.empty(stage.workspace_bytes(), dtype=torch.uint8, device=DEV))
    stage.load_layer(0, {k: to_dev_bits(v) for k, v in weights[0].items()})
    dk, dv, x = to_dev_bits(k0), to_dev_bits(v0), to_dev_bits(hidden)
    stage.bind_kv_pool(dk, dv, len(order))
    out, out32 = torch.empty(sum(new), shape.hidden, dtype=torch.bfloat16, device=DEV), torch.empty(sum(new), shape.hidden, device=DEV)
    stage.forward_tree(new, cached, tables, np.concatenate(trees), x, out, out32)
    torch.cuda.synchronize()
    starts = np.concatenate([[0], np.cumsum(new)])
    paths = [(s, O.chain(t, i)) for s, t in enumerate(trees) for i in range(len(t)) if i not in t]
    per = synth.pool_elems_per_layer(shape, len(order)) // len(order)
    K, V = (z.reshape(len(order), per) for z in (k0, v0))
    ptab, ids = np.zeros((len(paths), max(pages)), dtype=np.int32), []
    for i, (s, path) in enumerate(paths):
        p = -(-(cached[s] + len(path)) // 16)
        ptab[i, :p] = np.arange(len(ids), len(ids) + p)
        ids += tables[s, :p].tolist()
    rows = np.concatenate([starts[s] + np.array(path) for s, path in paths])
    ref, _ = oracle.stage_forward(shape, weights, np.array([len(p) for _, p in paths], dtype=np.int32), np.array([cached[s] for s, _ in paths], dtype=np.int32),
                                  ptab, len(ids), K[ids].reshape(-1), V[ids].reshape(-1), hidden[rows])
    off = np.abs(out32.cpu().numpy().astype(np.float64)[rows] - ref)
    print(f"[parity] 70 trees: max_abs={off.max():.4g} mean_rel={off.sum() / np.abs(ref).sum():.4g} over {len(rows)} rows", flush=True)
    assert set(rows) == set(range(sum(new)))
    assert off.max() <= 2e-2 * max(1.0, np.sqrt((ref ** 2).mean())) and off.sum() / np.abs(ref).sum() <= 5e-3
    stage.destroy()
