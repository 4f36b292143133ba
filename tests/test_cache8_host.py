"""A KV cache held in 8 bits: the ABI, what its calls refuse (on the host, before anything is enqueued), and the oracle against the
statements of its header.  No GPU."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import cache8_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import cache8 as C8

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gllm_cache8.h")
INVALID, CAPACITY, UNSUPPORTED = -1, -2, -7
P = 1 << 20        # an aligned address that no refused call looks at


def test_library_exports_every_function_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(gllm_[a-z0-9_]+)\s*\(", text)))
    lib = B.load_library()
    for n in declared:
        assert hasattr(lib, n), n
    assert set(declared) == set(C8.EXPORTS)


MAPS = dict(new=P, cached=P, seqs=2, free=P, num_free=9, tables=P, stride=4, num_blocks=9, rows=5, row_start=P, positions=P, slots=P, needed=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(new=None), INVALID), (dict(cached=None), INVALID), (dict(free=None), INVALID), (dict(tables=None), INVALID), (dict(row_start=None), INVALID),
    (dict(positions=None), INVALID), (dict(slots=None), INVALID), (dict(needed=None), INVALID), (dict(seqs=-1), INVALID), (dict(num_free=-1), INVALID),
    (dict(stride=0), INVALID), (dict(num_blocks=0), INVALID), (dict(num_blocks=1 << 27), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(seqs=(1 << 20) + 1), CAPACITY),
    (dict(seqs=0, row_start=None), INVALID),
])
def test_step_maps_refuses(change, status):
    assert C8._lib().gllm_op_step_maps(*{**MAPS, **change}.values()) == status


STORE = dict(qkv=P, ld_qkv=1024, rows_type=0, q_gain=P, k_gain=P, eps=1e-6, rope=P, max_position=100, positions=P, slots=P, rows=5, n_q=4, n_kv=2, d=128,
             q_out=P, ld_q=512, k=P, v=P, scales=P, num_blocks=9, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(qkv=None), INVALID), (dict(rope=None), INVALID), (dict(positions=None), INVALID), (dict(slots=None), INVALID), (dict(q_out=None), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(scales=None), INVALID), (dict(rows=-1), INVALID), (dict(rows_type=2), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(max_position=0), INVALID), (dict(n_q=0), INVALID),
    (dict(n_kv=0), INVALID), (dict(num_blocks=0), INVALID), (dict(num_blocks=1 << 27), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(n_q=65534), UNSUPPORTED),
    (dict(ld_qkv=1020), INVALID), (dict(ld_qkv=1026), INVALID), (dict(ld_q=508), INVALID), (dict(ld_q=514), INVALID), (dict(qkv=P + 8), INVALID),
    (dict(qkv=P + 4, rows_type=1), INVALID), (dict(q_gain=P + 4), INVALID), (dict(k_gain=P + 2), INVALID), (dict(rope=P + 8), INVALID), (dict(q_out=P + 4), INVALID),
    (dict(k=P + 8), INVALID), (dict(v=P + 8), INVALID), (dict(scales=P + 4), INVALID), (dict(rows=0, qkv=None), 0),
])
def test_norm_rope_store_refuses(change, status):
    assert C8._lib().gllm_op_norm_rope_store8(*{**STORE, **change}.values()) == status


@pytest.mark.parametrize("eps", [1e-60, 2.0 ** -150, 3.5e38, 1e300])
def test_norm_rope_store_refuses_an_eps_that_float_does_not_hold(eps):
    """Rounded to 0 it would make heads of zeros no numbers, rounded to infinity every head zeros."""
    assert C8._lib().gllm_op_norm_rope_store8(*{**STORE, "eps": eps}.values()) == INVALID
    assert C8._lib().gllm_op_norm_rope_store8(*{**STORE, "eps": eps, "rows": 0}.values()) == INVALID


ATTENTION = dict(q=P, ld_q=512, k=P, v=P, scales=P, num_blocks=9, tables=P, stride=4, cached=P, starts=P, seqs=2, rows=5, max_new=8, window=0, sinks=0,
                 n_q=4, n_kv=2, d=128, scale=0.1, out=P, ld_o=512, ws=P, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(scales=None), INVALID), (dict(tables=None), INVALID),
    (dict(cached=None), INVALID), (dict(starts=None), INVALID), (dict(out=None), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=0), CAPACITY),
    (dict(seqs=-1), INVALID), (dict(seqs=(1 << 20) + 1), CAPACITY), (dict(rows=-1), INVALID), (dict(max_new=0), INVALID), (dict(window=-1), INVALID),
    (dict(sinks=-1, window=5), INVALID), (dict(sinks=3), INVALID), (dict(num_blocks=0), INVALID), (dict(num_blocks=1 << 27), UNSUPPORTED), (dict(stride=0), INVALID),
    (dict(n_q=5), UNSUPPORTED), (dict(n_q=0), INVALID), (dict(n_q=34, n_kv=2, ld_q=8192, ld_o=8192), UNSUPPORTED), (dict(d=96), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(ld_q=504), INVALID),
    (dict(ld_q=516), INVALID), (dict(ld_o=508), INVALID), (dict(ld_o=514), INVALID), (dict(q=P + 8), INVALID), (dict(k=P + 8), INVALID), (dict(v=P + 2), INVALID),
    (dict(scales=P + 4), INVALID), (dict(out=P + 4), INVALID), (dict(ws=P + 8), INVALID), (dict(rows=2147483647, n_q=16, n_kv=1, ld_q=2048, ld_o=2048), CAPACITY),
    (dict(seqs=0, q=None), 0), (dict(rows=0, q=None), 0),
])
def test_attention_refuses(change, status):
    assert C8._lib().gllm_op_attention8(*{**ATTENTION, **change}.values()) == status


def test_more_work_than_a_launch_takes_is_refused():
    for rows in (1 << 27, 1 << 30):
        assert C8._lib().gllm_op_norm_rope_store8(*{**STORE, "rows": rows}.values()) == CAPACITY
    large = dict(seqs=1 << 20, max_new=17, n_q=128, n_kv=64, ld_q=16384, ld_o=16384)
    assert C8._lib().gllm_op_attention8(*{**ATTENTION, **large}.values()) == CAPACITY


@pytest.mark.parametrize("max_new", [1, 17])
def test_more_work_than_the_joining_takes_is_refused(max_new):
    """64 sequences and 2^18 KV heads: the first launch takes them, the joining would not (before anything is enqueued, or the outputs would be half done)."""
    heads = 1 << 18
    much = dict(seqs=64, rows=64, stride=100, max_new=max_new, n_q=heads, n_kv=heads, d=64, ld_q=64 * heads, ld_o=64 * heads)
    assert C8._lib().gllm_op_attention8(*{**ATTENTION, **much}.values()) == CAPACITY


@pytest.mark.parametrize("shape", [(0, 1, 128, 1), (4, 0, 128, 1), (5, 2, 128, 1), (34, 2, 64, 1), (4, 2, 96, 1), (4, 2, 128, 0)])
def test_no_workspace_for_what_attention_does_not_take(shape):
    assert C8.gllm_op_attention8_workspace_bytes(*shape) == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    i = torch.zeros(3, dtype=torch.int32)
    k, v, s = torch.zeros(2, 2, 4, 4, 4, 16, dtype=torch.uint8), torch.zeros(2, 2, 64, 16, dtype=torch.uint8), torch.zeros(2, 2, 2)
    q = torch.zeros(3, 256, dtype=torch.bfloat16)
    with pytest.raises(B.GllmError):
        C8.gllm_op_step_maps(i, i, i, i.view(3, 1), 4, torch.zeros(4, dtype=torch.int32), i, i, i[:2])
    with pytest.raises(B.GllmError):
        C8.gllm_op_norm_rope_store8(torch.zeros(3, 512), None, None, 1e-6, torch.zeros(5, 32, 2), i, i, q, k, v, s)
    with pytest.raises(B.GllmError):
        C8.gllm_op_attention8(q, k, v, s, i.view(3, 1), i, torch.zeros(4, dtype=torch.int32), q, 1)
    with pytest.raises(B.GllmError):
        C8.gllm_op_attention8(q, k[:, :, :, :3], v, s, i.view(3, 1), i, torch.zeros(4, dtype=torch.int32), q, 1)


# ---- the oracle ------------------------------------------------------------------------------------------------------------

def test_values_of_the_codes_are_those_of_the_type():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, O.VALUES, equal_nan=True)


def test_rounding_goes_to_the_nearest_value_and_to_even():
    x = np.concatenate([np.linspace(-448, 448, 20011), O.VALUES[np.isfinite(O.VALUES)], 2.0 ** np.arange(-14, 8) * 1.03, [2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10]])
    want = torch.tensor(x, dtype=torch.float64).float().to(torch.float8_e4m3fn).double().numpy()
    single = x.astype(np.float32).astype(np.float64)                    # torch rounds from float32
    assert np.array_equal(O.round_e4m3(single), want)
    assert (np.abs(O.round_e4m3(single) - single) <= O.half_step(single)).all()


def test_step_maps_by_hand():
    free = [70, 71, 72, 73]
    tables = np.array([[5, -9, -9], [6, 7, -9], [-9, -9, -9], [8, 9, -9]])
    start, pos, slots, needed, out = O.step_maps([17, 1, 0, 2], [15, 32, 0, 16], free, tables, 80, 22)
    assert start.tolist() == [0, 17, 18, 18, 20] and needed.tolist() == [20, 3]
    assert out.tolist() == [[5, 70, -9], [6, 7, 71], [-9, -9, -9], [8, 72, -9]]
    assert slots.tolist() == [5 * 16 + 15] + list(range(70 * 16, 70 * 16 + 16)) + [71 * 16] + [72 * 16, 72 * 16 + 1] + [-1, -1]
    assert pos.tolist() == list(range(15, 32)) + [32, 16, 17, 0, 0]


def test_step_maps_without_room():
    tables = np.full((4, 2), -9)
    start, pos, slots, needed, out = O.step_maps([16, 17, 3, 16], [0, 0, -1, 0], [4, 99], tables, 50, 40)
    assert start.tolist() == [0, 16, 33, 36, 36] and needed.tolist() == [52, 4]
    assert out.tolist() == [[4, -9], [99, -1], [-9, -9], [-9, -9]]
    assert slots[:16].tolist() == list(range(64, 80)) and (slots[16:] == -1).all() and (pos[33:] == 0).all()


def test_attention_by_hand():
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((3, 16, 1, 4)), rng.standard_normal((3, 16, 1, 4))
    q = rng.standard_normal((2, 1, 4))
    out, _, _ = O.attention(q, k, v, [[2, 0]], [19], [0, 2], 0.5, window=3, sinks=1)
    keys = lambda pool, ps: np.array([pool[[2, 0][p // 16], p % 16, 0] for p in ps])
    for i, ps in enumerate(([0, 17, 18, 19], [0, 18, 19, 20])):
        w = np.exp(keys(k, ps) @ q[i, 0] * 0.5)
        assert np.allclose(out[i, 0], w @ keys(v, ps) / w.sum())
