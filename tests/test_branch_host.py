"""Several continuations of one sequence: the ABI, what its calls refuse (on the host, before anything is enqueued), and the
oracle against brute force.  No GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from oracle import branch_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import branch as BR

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gllm_branch.h")
INVALID, CAPACITY, RANGE, ALIAS, UNSUPPORTED = -1, -2, -3, -4, -7
P = 1 << 20        # an aligned address that no refused call looks at


def test_library_exports_every_function_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(gllm_[a-z0-9_]+)\s*\(", text)))
    lib = B.load_library()
    for n in declared:
        assert hasattr(lib, n), n
    assert set(declared) == set(BR.EXPORTS)


ATTENTION = dict(q=P, ld_q=512, k=P, v=P, num_blocks=9, tables=P, stride=4, cached=P, starts=P, parents=P, seqs=2, rows=5, max_nodes=8,
                 n_q=4, n_kv=2, d=128, scale=0.1, out=P, ld_o=512, ws=P, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(tables=None), INVALID), (dict(cached=None), INVALID),
    (dict(starts=None), INVALID), (dict(parents=None), INVALID), (dict(out=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws_bytes=0), CAPACITY), (dict(seqs=-1), INVALID), (dict(rows=-1), INVALID), (dict(max_nodes=0), INVALID), (dict(max_nodes=257), UNSUPPORTED),
    (dict(num_blocks=0), INVALID), (dict(num_blocks=1 << 31), INVALID), (dict(stride=0), INVALID), (dict(n_q=5), UNSUPPORTED), (dict(n_q=0), INVALID),
    (dict(n_q=34, n_kv=2, ld_q=8192, ld_o=8192), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(ld_q=504), INVALID), (dict(ld_q=516), INVALID), (dict(ld_o=508), INVALID),
    (dict(ld_o=514), INVALID), (dict(q=P + 8), INVALID), (dict(k=P + 8), INVALID), (dict(v=P + 2), INVALID), (dict(out=P + 4), INVALID), (dict(ws=P + 8), INVALID),
    (dict(rows=1 << 30), CAPACITY),
    (dict(seqs=0, q=None), 0), (dict(rows=0, q=None), 0),
])
def test_tree_attention_refuses(change, status):
    assert BR._lib().gllm_op_tree_attention(*{**ATTENTION, **change}.values()) == status


COMMIT = dict(tokens=P, parents=P, sampled=P, starts=P, cached=P, tables=P, stride=4, seqs=2, rows=5, k=P, v=P, layers=3, num_blocks=9, n_kv=2, d=64,
              path=P, count=P, next=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=None), INVALID), (dict(parents=None), INVALID), (dict(sampled=None), INVALID), (dict(starts=None), INVALID), (dict(cached=None), INVALID),
    (dict(tables=None), INVALID), (dict(path=None), INVALID), (dict(count=None), INVALID), (dict(next=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(seqs=-1), INVALID), (dict(rows=-1), INVALID), (dict(stride=0), INVALID), (dict(layers=0), INVALID), (dict(num_blocks=0), INVALID),
    (dict(n_kv=0), INVALID), (dict(d=32), UNSUPPORTED), (dict(k=P + 8), INVALID), (dict(v=P + 8), INVALID), (dict(seqs=1 << 30), CAPACITY), (dict(seqs=0, tokens=None), 0),
])
def test_tree_commit_refuses(change, status):
    assert BR._lib().gllm_op_tree_commit(*{**COMMIT, **change}.values()) == status


BEAMS = dict(logits=P, ld=1024, scores=P, seqs=2, beams=4, vocab=1000, keep=8, out_scores=P, out_beams=P, out_tokens=P, ws=P, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(logits=None), INVALID), (dict(scores=None), INVALID), (dict(out_scores=None), INVALID), (dict(out_beams=None), INVALID), (dict(out_tokens=None), INVALID),
    (dict(ws=None), INVALID), (dict(ws_bytes=8), CAPACITY), (dict(ld=999), INVALID), (dict(beams=0), INVALID), (dict(beams=33), UNSUPPORTED), (dict(keep=0), INVALID),
    (dict(keep=65), UNSUPPORTED), (dict(vocab=0), INVALID), (dict(vocab=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED), (dict(seqs=-1), INVALID), (dict(logits=P + 2), INVALID),
    (dict(ws=P + 8), INVALID), (dict(seqs=0, logits=None), 0),
])
def test_beam_select_refuses(change, status):
    assert BR._lib().gllm_op_beam_select(*{**BEAMS, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(src=None), INVALID), (dict(dst=None), INVALID), (dict(k=P + 8), INVALID), (dict(layers=0), INVALID),
    (dict(n=-1), INVALID), (dict(num_blocks=0), INVALID), (dict(d=48), UNSUPPORTED), (dict(n_kv=0), INVALID),
    (dict(src=[1, 9]), RANGE), (dict(src=[1, -1]), RANGE), (dict(dst=[3, 9]), RANGE), (dict(dst=[-1, 3]), RANGE),
    (dict(dst=[3, 3]), ALIAS), (dict(dst=[1, 3]), ALIAS), (dict(src=[4, 3]), ALIAS), (dict(n=0, k=None, src=None), 0),
])
def test_copy_pages_refuses(change, status):
    a = {**dict(k=P, v=P, layers=2, num_blocks=9, n_kv=2, d=64, src=[1, 2], dst=[3, 4], n=2, stream=None), **change}
    keep = []
    for x in ("src", "dst"):
        if a[x] is not None:
            keep.append(np.array(a[x], dtype=np.int32))
            a[x] = keep[-1].ctypes.data
    assert BR._lib().gllm_op_copy_pages(*a.values()) == status


def test_workspace_sizes():
    f, g = BR.gllm_op_tree_attention_workspace_bytes, BR.gllm_op_beam_select_workspace_bytes
    assert f(32, 8, 128, 64) > 0 and f(32, 8, 128, 0) == 0 and f(32, 8, 128, 257) == 0 and f(33, 8, 128, 8) == 0 and f(32, 8, 80, 8) == 0
    assert g(4, 8, 128256, 16) > 0 and g(4, 33, 128256, 16) == 0 and g(4, 8, 0, 16) == 0 and g(4, 8, 128256, 65) == 0 and g(-1, 8, 128256, 16) == 0


def test_wrappers_refuse_tensors_on_the_host():
    i, b = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 128, dtype=torch.bfloat16)
    k, v = torch.zeros(2, 3, 2, 8, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 64, 16, dtype=torch.bfloat16)
    f = torch.zeros(2, 4)
    calls = [lambda: BR.gllm_op_tree_attention(b, k[0], v[0], i.view(1, 4), i[:1], i[:2], i, b, 4),
             lambda: BR.gllm_op_tree_commit(i, i, i, i[:2], i[:1], i.view(1, 4), k, v, i, i[:1], i[:1]),
             lambda: BR.gllm_op_beam_select(torch.zeros(8, 100), 100, f, f, f.int(), f.int()),
             lambda: BR.gllm_op_copy_pages(k, v, [0], [1])]
    for call in calls:
        with pytest.raises(B.GllmError) as e:
            call()
        assert e.value.status == INVALID
    with pytest.raises(B.GllmError) as e:
        BR.gllm_op_copy_pages(k, v[:, :, :1], [0], [1])                   # pools of different head counts
    assert "shapes" in e.value.message


def test_oracle_attention_is_plain_causal_attention_on_a_chain():
    rng = np.random.default_rng(0)
    n_q, n_kv, d, c, n = 4, 2, 8, 19, 6
    table = [3, 0]
    k, v = rng.standard_normal((4, n_kv, 1, 16, 8)), rng.standard_normal((4, n_kv, d, 16))
    q = rng.standard_normal((n, n_q, d))
    out, _, _ = O.tree_attention(q, k, v, [table], [c], [0, n], np.arange(-1, n - 1), d ** -0.5)
    at = np.arange(c + n)
    kk, vv = O.gather_k(k, table, at), O.gather_v(v, table, at)
    assert np.array_equal(kk[17, 1], k[0, 1, 0, 1]) and np.array_equal(vv[17, 1], v[0, 1, :, 1])
    for i in range(n):
        for h in range(n_q):
            x = kk[:c + i + 1, h // 2] @ q[i, h] * d ** -0.5
            p = np.exp(x) / np.exp(x).sum()
            assert np.allclose(out[i, h], p @ vv[:c + i + 1, h // 2], atol=1e-12)


def test_oracle_trees_and_walks():
    parents = np.array([-1, 0, 0, 1, 7, 4, 2, 2])
    assert O.chain(parents, 3) == [0, 1, 3] and O.chain(parents, 4) is None and O.chain(parents, 5) is None
    tokens, sampled = np.array([5, 8, 9, 1, 1, 1, 7, 7]), np.array([9, 0, 7, 0, 0, 0, 3, 4])
    path, count, follow = O.tree_commit(tokens, parents, sampled, [0, 8], [0], [[0]])
    assert path.tolist() == [0, 2, 6, -1, -1, -1, -1, -1] and count.tolist() == [3] and follow.tolist() == [3]


def test_oracle_beams_by_brute_force():
    rng = np.random.default_rng(1)
    x, s = rng.standard_normal((6, 11)), rng.standard_normal((2, 3))
    s[1, 2] = -np.inf
    score, beam, token = O.beam_select(x, s, 5)
    for i in range(2):
        every = [(s[i, b] + x[3 * i + b, t] - np.log(np.exp(x[3 * i + b]).sum()), b, t) for b in range(3) for t in range(11)]
        every.sort(key=lambda e: (-e[0], e[1], e[2]))
        assert [(b, t) for _, b, t in every[:5]] == list(zip(beam[i], token[i]))
        assert np.allclose(score[i], [e[0] for e in every[:5]])


def test_oracle_beams_of_equal_sums():
    """Differences of the logits that the sum in 64 bits swallows still order the continuations of a beam, and not those of two."""
    x = np.array([[1e-20, 3e-20, 2e-20, 3e-20], [9e-20, 0.0, 5e-20, 0.0]], dtype=np.float32)
    score, beam, token = O.beam_select(x, np.zeros((1, 2), dtype=np.float32), 6)
    assert beam[0].tolist() == [0, 0, 0, 0, 1, 1] and token[0].tolist() == [1, 3, 2, 0, 0, 2] and len(set(score[0])) == 1
    score, beam, token = O.beam_select(x * 1e20, np.full((1, 2), -1e18, dtype=np.float32), 6)
    assert beam[0].tolist() == [0, 0, 0, 0, 1, 1] and token[0].tolist() == [1, 3, 2, 0, 0, 2]


def test_tree_attention_refuses_more_sequences_than_the_plan_adds_up():
    for seqs in ((1 << 22) + 1, 1 << 30):
        assert BR._lib().gllm_op_tree_attention(*{**ATTENTION, "seqs": seqs}.values()) == CAPACITY


@pytest.mark.parametrize("scale,status", [(2.4e38, INVALID), (3.4e38, INVALID), (2.3e38, CAPACITY)])
def test_tree_attention_refuses_a_scale_that_is_not_finite_in_base_2(scale, status):
    assert BR._lib().gllm_op_tree_attention(*{**ATTENTION, "scale": scale, "ws_bytes": 0}.values()) == status


@pytest.mark.parametrize("src,dst,status", [([1 << 32], [1], RANGE), ([0], [(1 << 32) + 1], RANGE), ([0], [-(1 << 32) + 1], RANGE), ([0], [1 << 70], RANGE),
                                            ([0.5], [1], INVALID), ([0], [float("nan")], INVALID), ([0], [[1]], INVALID), ([0], ["1"], INVALID), ([0], [None], INVALID)])
def test_page_ids_that_are_no_32_bit_numbers_are_refused(src, dst, status):
    """Not taken modulo 2^32, not rounded (and before a look at the pools, which lie on the host here)."""
    k, v = torch.zeros(2, 3, 2, 8, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 64, 16, dtype=torch.bfloat16)
    with pytest.raises(B.GllmError) as e:
        BR.gllm_op_copy_pages(k, v, src, dst)
    assert e.value.status == status and "cpu" not in e.value.message


def test_pools_without_a_head_dimension_are_refused():
    b, i = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    k, v = torch.zeros(2, 3, 2, 0, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 0, 16, dtype=torch.bfloat16)
    for call in (lambda: BR.gllm_op_tree_attention(b, k[0], v[0], i.view(1, 4), i[:1], i[:2], i, b, 4), lambda: BR.gllm_op_copy_pages(k, v, [0], [1])):
        with pytest.raises(B.GllmError) as e:
            call()
        assert e.value.status == INVALID and "shapes" in e.value.message


@pytest.mark.parametrize("change", [dict(layers=(1 << 31) - 1, n_kv=(1 << 31) - 1, seqs=4), dict(layers=1 << 30, n_kv=1 << 30, seqs=16), dict(layers=1 << 16, n_kv=1 << 15, seqs=1),
                                    dict(layers=1 << 15, n_kv=1 << 10, seqs=1 << 6)], ids=str)
def test_tree_commit_refuses_more_moves_than_a_launch_has_places(change):
    assert BR._lib().gllm_op_tree_commit(*{**COMMIT, **change}.values()) == CAPACITY


@pytest.mark.parametrize("ids", [[[1], [1, 2]], torch.zeros(2, device="meta", dtype=torch.int32)], ids=["ragged", "meta"])
def test_page_ids_that_are_no_array_of_the_host_are_refused(ids):
    k, v = torch.zeros(2, 3, 2, 8, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 64, 16, dtype=torch.bfloat16)
    with pytest.raises(B.GllmError) as e:
        BR.gllm_op_copy_pages(k, v, ids, [1])
    assert e.value.status == INVALID and "page ids" in e.value.message
