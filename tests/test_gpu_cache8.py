"""GPU parity of the operators over a KV cache held in 8 bits (include/gllm_cache8.h) against oracle/cache8_oracle.py.

Step maps: equal.
Store: a head's norm and rotation are computed in float32.  The sum of at most 128 squares is off by at most 2^-20 of itself in any order
that adds fewer than 16 terms in a row and is halved by the square root; with the roundings of the root, the products and the rotation
an element is off by at most 2^-20 T, T = |x_i cos| + |x_j sin| of the normalised pair, with room 2^-19 T.  Queries: 2^-8 |q| more (bf16).
Scales: 2^-19 of the largest T of the page relative, and 2^-23 for the division.  A stored value is off by half a step of its code at its
scale, and 2^-19 T.  Kept codes are equal to the rounded ones.
Attention: the weights of the softmax, times the scale of the value's page, and the output are rounded to bf16 (2^-8 relative each, eps/2
of the type), the scores summed in float32.  With A = sum p|v| and M the largest sum |q_i k_i| * scale of a row, an output is off by at
most 2^-8 |out| + (2^-8 + 2 M (d + 10) 2^-24 + 2^-17) A: the middle term is what an error of a score does to p and to its sum (d products
and sums of 2^-24 each, the scales, twice: numerator and denominator), the last the exponentials, the logarithm of a scale and the sums over keys."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache8_oracle as O
from paper_2504_14775_amd import binding as B
from paper_2504_14775_amd import cache8 as C8
from gpu_util import DEV

pytestmark = pytest.mark.gpu
PAGE = 16
NAN_CODE = 0x7F
HIP, INVALID_VALUE = -6, 1     # gllm_status, hipError_t
HEADS = [(4, 2, 64), (32, 8, 128), (10, 2, 128), (16, 1, 128), (8, 8, 64), (12, 4, 128), (7, 1, 64)]


def dev_ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def values(codes, side):
    """[pages][16][n_kv][d] of a pool's codes."""
    c = codes.view(torch.uint8).cpu().numpy()
    return O.VALUES[O.slots_of_k(c) if side == 0 else O.slots_of_v(c)]


def empty_pool(pages, n_kv, d):
    """Codes that are no numbers, scales that are none: what nothing may read."""
    return (torch.full((pages, n_kv, 4, d // 16, 4, 16), NAN_CODE, dtype=torch.uint8, device=DEV),
            torch.full((pages, n_kv, d, 16), NAN_CODE, dtype=torch.uint8, device=DEV), torch.full((pages, n_kv, 2), float("nan"), device=DEV))


# ---- step maps -------------------------------------------------------------------------------------------------------------

class Maps:
    def __init__(self, new, cached, num_free, rows, entries, num_blocks=None, seed=0):
        rng = np.random.default_rng(seed)
        held = [max(0, -(-c // PAGE)) for c in cached]
        total = sum(min(h, entries) for h in held) + num_free + 2
        self.blocks = num_blocks or total
        order = rng.permutation(total)
        self.tables = np.full((len(new), entries), -77)
        at = 0
        for s, h in enumerate(held):
            h = min(h, entries)
            self.tables[s, :h] = order[at:at + h]
            at += h
        self.new, self.cached, self.free, self.rows = list(new), list(cached), order[at:at + num_free], rows

    def run(self, stream=None):
        i = [dev_ints(x) for x in (self.new, self.cached, self.free, self.tables)]
        out = [torch.full((n,), -99, dtype=torch.int32, device=DEV) for n in (len(self.new) + 1, self.rows, self.rows, 2)]
        C8.gllm_op_step_maps(i[0], i[1], i[2], i[3], self.blocks, *out, stream=stream)
        torch.cuda.synchronize()
        return [x.cpu().numpy() for x in out + [i[3]]]

    def check(self):
        got = self.run()
        want = O.step_maps(self.new, self.cached, self.free, self.tables, self.blocks, self.rows)
        for name, a, b in zip(("row_start", "positions", "slots", "needed", "tables"), got, want):
            assert np.array_equal(a, b), name
        return got


@pytest.mark.parametrize("seqs,most,pad", [(1, 1, 0), (1, 40, 3), (3, 17, 0), (64, 1, 0), (257, 9, 100), (1024, 3, 0), (1025, 3, 7), (2600, 2, 1), (5, 4000, 50)])
def test_step_maps(seqs, most, pad):
    print(f"step maps of {seqs} sequences of up to {most}", flush=True)
    rng = np.random.default_rng(seqs)
    new = rng.integers(0 if seqs > 3 else 1, most + 1, seqs)
    cached = rng.integers(0, 200, seqs)
    Maps(new, cached, int(new.sum()) // PAGE + 2 * seqs, int(new.sum()) + pad, (200 + most) // PAGE + 2, seed=seqs).check()


def test_step_maps_of_odd_lengths():
    print("step maps: broken sequences, no pages left, page ids outside the pool", flush=True)
    big = 2 ** 31 - 1
    Maps([3, -5, 4, 16, 2, 0, 7], [5, 3, -1, 32, 900, big, big], 9, 60, 8, seed=1).check()
    Maps([40, 50, 60], [0, 7, 16], 5, 150, 10, seed=2).check()
    Maps([40, 50, 60], [0, 7, 16], 0, 150, 10, seed=2).check()
    Maps([20, 30, 40], [16, 0, 5], 9, 90, 10, num_blocks=4, seed=3).check()
    Maps([big, big, big], [0, 0, 0], 3, 20, 4, seed=4).check()
    Maps([5, 6], [0, 0], 3, 0, 4, seed=4).check()


@pytest.mark.parametrize("rows", [0, 1, 9, 10, 29, 30, 700, 2999])
def test_step_maps_with_too_few_rows(rows):
    print(f"step maps: {rows} rows", flush=True)
    rng = np.random.default_rng(rows)
    Maps([10, 20, 0, 30, 0, 5], [1, 16, 3, 0, 9, 2], 12, rows, 6, seed=rows).check()
    Maps(rng.integers(0, 4, 2000), rng.integers(0, 40, 2000), 2500, rows, 6, seed=rows).check()


def test_step_maps_without_sequences():
    out = [torch.full((n,), 9, dtype=torch.int32, device=DEV) for n in (1, 3, 3, 2)]
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    C8.gllm_op_step_maps(none, none, none, none.view(0, 4), 5, *out)
    assert [x.tolist() for x in out] == [[0], [0, 0, 0], [-1, -1, -1], [0, 0]]


# ---- norm, rotation and store ----------------------------------------------------------------------------------------------

def rope_table(most, d, theta=10000.0):
    a = torch.arange(most, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    return torch.stack((a.cos(), a.sin()), -1).float().to(DEV)


class Store:
    """runs: (slot of the first row, rows) of one page each."""

    def __init__(self, heads, runs, dtype=torch.float32, norm=True, seed=0, skip=(), pad=0, size=1.0):
        self.n_q, self.n_kv, self.d = n_q, n_kv, d = heads
        rng = np.random.default_rng(seed)
        g = torch.Generator(device=DEV).manual_seed(seed)
        pages = len(runs) + 2
        order = rng.permutation(pages)
        slots = [int(order[i]) * PAGE + f + t for i, (f, n) in enumerate(runs) for t in range(n)]
        rows = len(slots)
        self.slots = np.array(slots)
        for i in skip:
            self.slots[i] = -1 if i % 2 else pages * PAGE + 3
        self.positions = rng.integers(0, 5000, rows)
        self.rope = rope_table(5000, d)
        full = torch.randn(rows, (n_q + 2 * n_kv) * d + pad, generator=g, device=DEV) * size
        self.qkv = full.to(dtype)[:, :(n_q + 2 * n_kv) * d]
        self.gains = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).bfloat16() if norm else None for _ in range(2)]
        self.q_out = torch.full((rows, n_q * d + pad), 7.0, dtype=torch.bfloat16, device=DEV)[:, :n_q * d]
        self.k = torch.randint(0, 256, (pages, n_kv, 4, d // 16, 4, 16), generator=g, device=DEV).to(torch.uint8)
        self.v = torch.randint(0, 256, (pages, n_kv, d, 16), generator=g, device=DEV).to(torch.uint8)
        self.scales = torch.rand(pages, n_kv, 2, generator=g, device=DEV) * 0.02 * size + 1e-5 * size
        self.eps = 1e-6

    def run(self, **kw):
        C8.gllm_op_norm_rope_store8(self.qkv, *self.gains, self.eps, self.rope, dev_ints(self.positions), dev_ints(self.slots), self.q_out, self.k, self.v,
                                    self.scales, **kw)
        torch.cuda.synchronize()

    def check(self, label="", **kw):
        n_q, n_kv, d = self.n_q, self.n_kv, self.d
        before = [values(self.k, 0), values(self.v, 1), f64(self.scales), self.k.clone(), self.v.clone()]
        self.run(**kw)
        x = f64(self.qkv).reshape(-1, n_q + 2 * n_kv, d)
        cs = self.rope.double().cpu().numpy()
        gains = [None if g is None else f64(g) for g in self.gains]
        pages = self.k.shape[0]
        got_q, got = f64(self.q_out).reshape(-1, n_q, d), [values(self.k, 0), values(self.v, 1)]
        scales = f64(self.scales)
        new = np.full((2, pages, PAGE, n_kv, d), np.nan)
        room = np.zeros((2, pages, PAGE, n_kv, d))
        wrote = np.zeros((pages, PAGE), dtype=bool)
        for r, slot in enumerate(self.slots):
            if not 0 <= slot < pages * PAGE:
                assert np.all(got_q[r] == 7.0)
                continue
            angle = cs[min(max(self.positions[r], 0), len(cs) - 1)]
            want, t = O.norm_rotate(x[r, :n_q], gains[0], self.eps, angle)
            with np.errstate(invalid="ignore"):
                off = np.abs(got_q[r] - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -19 * t)
            assert np.all((off <= 0) | (np.isnan(want) & np.isnan(got_q[r]))), (label, r)
            p, s = divmod(int(slot), PAGE)
            wrote[p, s] = True
            new[0, p, s], room[0, p, s] = O.norm_rotate(x[r, n_q:n_q + n_kv], gains[1], self.eps, angle)
            new[1, p, s] = x[r, n_q + n_kv:]
        for side in range(2):
            for p in range(pages):
                if not wrote[p].any():
                    continue
                first = int(np.argmax(wrote[p]))
                at = np.nonzero(wrote[p])[0]
                for h in range(n_kv):
                    y, t = new[side, p, at, h], room[side, p, at, h]
                    fin = np.isfinite(y)
                    most, slack = (np.abs(y[fin]).max() if fin.any() else 0.0), 2.0 ** -19 * (t[fin].max() if fin.any() else 0.0)
                    sc, old = scales[p, h, side], before[2][p, h, side]
                    if first == 0:
                        want = max(most / 448, O.LEAST)
                        assert abs(sc - want) <= 2.0 ** -23 * want + slack / 448, (label, p, h, side)
                        twice = 0
                    else:
                        if not (0 < old < np.inf):
                            old = O.LEAST
                        twice = np.log2(sc / old)
                        assert twice == int(twice) and twice >= 0
                        assert (most - slack) / 448 <= sc * (1 + 2.0 ** -23) and (twice == 0 or (most + slack) / 448 * (1 + 2.0 ** -23) > sc / 2), (label, p, h, side)
                        assert np.array_equal(got[side][p, :first, h], O.round_e4m3(before[side][p, :first, h] * 2.0 ** -twice), equal_nan=True), (label, p, h, side)
                    with np.errstate(invalid="ignore"):
                        z = got[side][p, at, h] * sc
                        tol = O.half_step(np.minimum(np.abs(y), 448 * sc) / sc) * sc * (1 + 2.0 ** -20) + 2.0 ** -19 * t + 2.0 ** -22 * np.abs(y)
                        assert np.all((np.abs(z - y) <= tol) | (~fin & np.isnan(z))), (label, p, h, side)
        still = torch.tensor(~wrote, device=DEV)                          # pages and slots that no row names: bit for bit
        gone = still & (torch.tensor(wrote, device=DEV).int().cumsum(1) == 0)
        left = still & ~(gone & torch.tensor(wrote.any(1), device=DEV)[:, None])
        for now, was, shape in ((self.k, before[3], lambda c: c.permute(0, 2, 4, 1, 3, 5).reshape(pages, PAGE, -1)), (self.v, before[4], lambda c: c.permute(0, 3, 1, 2).reshape(pages, PAGE, -1))):
            assert torch.equal(shape(now)[left], shape(was)[left]), label
        idle = ~wrote.any(1)
        assert np.array_equal(scales[idle], before[2][idle], equal_nan=True)


RUNS = [(0, 16), (0, 1), (15, 1), (3, 1), (5, 11), (1, 14), (0, 7), (8, 2), (0, 15), (12, 4)]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_norm_rope_store(heads, dtype, norm):
    print(f"store {heads} {dtype} norm {norm}", flush=True)
    Store(heads, RUNS, dtype, norm, seed=heads[0]).check(f"{heads}")


def test_store_rows_left_out_strides_and_many_rows():
    print("store: rows without slots, strided rows, many rows", flush=True)
    Store((10, 2, 128), RUNS, seed=1, skip=(0, 16, 17, 20, 71), pad=12).check("left out")
    Store((4, 2, 64), RUNS, torch.bfloat16, seed=2, skip=(3, 40), pad=4).check("left out, bf16")
    rng = np.random.default_rng(0)
    runs = [(f, int(rng.integers(1, 17 - f))) for f in rng.integers(0, 16, 300)]
    Store((8, 2, 64), runs, seed=3).check("many runs")
    Store((4, 1, 128), [(5, 1)], seed=4).check("one row")
    Store((2, 1, 64), [(0, 16)] * 200, seed=5).check("whole pages")


@pytest.mark.parametrize("pages", [10, 150, 520])
def test_store_of_rows_in_any_order_within_their_page(pages):
    """A page's rows in another order than their slots, with slots between them that nobody writes, and rows without slots between them.  Few rows, more
    than 1024, more than 4096."""
    print(f"store: rows in any order, {pages} pages", flush=True)
    rng = np.random.default_rng(pages)
    s = Store((2, 1, 64), [(0, int(rng.integers(5, 13))) for _ in range(pages)], seed=6)
    at = 0
    for p in range(pages):
        n = int((s.slots[at:] // PAGE == s.slots[at] // PAGE).sum())
        s.slots[at:at + n] = s.slots[at] // PAGE * PAGE + rng.permutation(PAGE)[:n]
        if p % 3 == 0:
            s.slots[at + n // 2] = -1
        at += n
    s.check("any order")


@pytest.mark.parametrize("norm", [True, False])
def test_store_takes_one_gain_without_the_other(norm):
    s = Store((4, 2, 128), RUNS, seed=6)
    s.gains[0 if norm else 1] = None
    s.check("one gain")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128)], ids=str)
def test_store_of_zeros_extremes_and_values_that_are_not_finite(heads, dtype):
    print(f"store: odd values {heads}", flush=True)
    d = heads[2]
    for what in ("zeros", "tiny", "huge", "nan", "inf", "all nan", "border"):
        s = Store(heads, RUNS, dtype, norm=False, seed=7)
        kv = s.qkv[:, heads[0] * d:]
        if what == "zeros":
            s.qkv.zero_()
        elif what == "tiny":
            kv.mul_(1e-33)
        elif what == "huge":
            kv.mul_(1e33)
        elif what == "nan":
            kv[::3, 5] = float("nan")
        elif what == "inf":
            kv[1::4, d + 3] = float("inf")
            kv[2::4, 2 * d + 9] = -float("inf")
        elif what == "all nan":
            kv.fill_(float("nan"))
        else:                                            # magnitudes at and next to the largest that a page's scale holds
            s.scales.fill_(1.0 / 1024)
            kv.clamp_(-0.4, 0.4)
            kv[:, ::7] = 0.4375
            kv[:, 3::7] = 0.44 if dtype is torch.float32 else 0.439453125
        s.positions[:] = 0                               # (cosine 1, sine 0)
        s.check(what)


def test_store_over_scales_that_are_none():
    print("store: kept pages whose scales are no scales", flush=True)
    s = Store((4, 2, 64), [(3, 2), (5, 1), (1, 15), (9, 7), (0, 3)], seed=8)
    s.scales.view(-1)[::5] = float("nan")
    s.scales.view(-1)[1::5] = 0.0
    s.scales.view(-1)[2::5] = -1.0
    s.scales.view(-1)[3::5] = float("inf")
    s.k.zero_()
    s.v.zero_()
    s.check("no scales")


def test_a_page_filled_token_by_token_is_as_one_filled_at_once_but_for_small_codes():
    """Scales that grow by powers of two do not round the kept codes again: what 16 calls of one row leave differs from the values by half
    a step at the final scale (a quarter more where a kept code became a small one: below 2^-6 it was rounded twice)."""
    print("store: token by token", flush=True)
    one = Store((4, 2, 64), [(0, 16)], seed=9, norm=False)
    one.positions[:] = 0
    x = f64(one.qkv).reshape(16, 8, 64)
    ramp = torch.linspace(0.05, 3.0, 16, device=DEV)[:, None]
    one.qkv.mul_(ramp)
    x = f64(one.qkv).reshape(16, 8, 64)
    for t in range(16):
        C8.gllm_op_norm_rope_store8(one.qkv[t:t + 1], None, None, 0.0, one.rope, dev_ints([0]), dev_ints(one.slots[t:t + 1]), one.q_out[t:t + 1], one.k, one.v, one.scales)
    page = int(one.slots[0]) // PAGE
    sc = f64(one.scales)[page]
    for side, pool in ((0, one.k), (1, one.v)):
        got = values(pool, side)[page]
        for h in range(2):
            y = x[:, 4 + 2 * side + h]
            most = np.abs(y).max()
            assert most / 448 * (1 - 2.0 ** -22) <= sc[h, side] and sc[h, side] <= max(2 * most / 448, np.abs(y[0]).max() / 448) * (1 + 2.0 ** -22)
            tol = O.half_step(y / sc[h, side]) * sc[h, side] * (1 + 2.0 ** -20) + 2.0 ** -10 * sc[h, side]
            assert (np.abs(got[:, h] * sc[h, side] - y) <= tol).all()


# ---- attention ---------------------------------------------------------------------------------------------------------------

def bound(ref, weight, mass, d):
    """How far an output may lie from the reference, with u = 2^-8, half a step of bf16, and weight = sum p |v|.  The weights are rounded to
    q = p (1 + e), |e| <= u, and divided by their own sum, rounded or not.  By the rounded one:
      |sum q v / sum q - ref| = |sum p e (v - ref)| / sum q <= u (weight + |ref|) / (1 - u),        as sum p (v - ref) = 0 and sum p = 1
    (by the other one u weight, which is less), and the output is rounded to bf16, by u of itself:
      u |ref| + (1 + u) u (weight + |ref|) / (1 - u) <= u |ref| + (u + 2^-15 + 2^-22) (weight + |ref|).
    Beside that scores and exponents in float: a score of magnitude `mass` is off by (d + 10) 2^-24 of that, its weight by as much, both in
    the weights and in their sum, and 2^-17 for what is left (exponential, scales' logarithms and reciprocals, sums)."""
    u = 2.0 ** -8
    return u * np.abs(ref) + (u + 2.0 ** -15 + 2.0 ** -22) * (weight + np.abs(ref)) + (2 * mass[..., None] * (d + 10) * 2.0 ** -24 + 2.0 ** -17) * weight


class Batch:
    """Inputs of one call of attention: sequences of given new and cached lengths over a pool in which nothing but their positions holds numbers."""

    def __init__(self, heads, new, cached, seed=0, spare=3, tail_rows=0, table_extra=0, perm_seed=None, q_pad=0, spread=4.0):
        self.n_q, self.n_kv, self.d = n_q, n_kv, d = heads
        self.new, self.cached = list(new), list(cached)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(self.starts[-1]) + tail_rows
        g = torch.Generator(device=DEV).manual_seed(seed)
        pages = [max(1, -(-(max(c, 0) + n) // PAGE)) for n, c in zip(new, cached)]
        total = sum(pages) + spare
        order = np.random.default_rng(seed if perm_seed is None else perm_seed).permutation(total)
        self.tables = np.zeros((len(self.new), max(pages) + table_extra), dtype=np.int32)
        self.k, self.v, self.scales = empty_pool(total, n_kv, d)
        at = 0
        for s, (p, n, c) in enumerate(zip(pages, new, cached)):
            ids = order[at:at + p]
            self.tables[s, :p] = ids
            at += p
            # contents by logical position, so that another order of the pages holds the same keys
            x = torch.randn(2, p, PAGE, n_kv, d, generator=g, device=DEV) * 100
            codes = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            used = (torch.arange(p * PAGE, device=DEV) < max(c, 0) + n).view(p, PAGE, 1, 1)
            codes = torch.where(used, codes, NAN_CODE)
            ids = torch.tensor(ids, device=DEV)
            self.k[ids] = codes[0].view(p, 4, 4, n_kv, d // 16, 16).permute(0, 3, 1, 4, 2, 5)
            self.v[ids] = codes[1].permute(0, 2, 3, 1)
            self.scales[ids] = 0.01 * spread ** (torch.rand(p, n_kv, 2, generator=g, device=DEV) - 0.5)
        q = torch.randn(rows, n_q * d + q_pad, generator=g, device=DEV).bfloat16()
        self.q = q[:, :n_q * d]
        self.out = torch.full((rows, n_q * d + q_pad), 7.0, dtype=torch.bfloat16, device=DEV)[:, :n_q * d]
        self.dev = [dev_ints(x) for x in (self.tables, self.cached, self.starts)]

    def slot(self, s, pos):
        return int(self.tables[s, pos // PAGE]), pos % PAGE

    def put(self, side, s, pos, code):
        """All codes of a position."""
        page, t = self.slot(s, pos)
        if side == 0:
            self.k[page, :, t // 4, :, t % 4] = code
        else:
            self.v[page, :, :, t] = code

    def run(self, window=0, sinks=0, max_new=None, scale=None, **kw):
        tables, cached, starts = self.dev
        C8.gllm_op_attention8(self.q, self.k, self.v, self.scales, tables, cached, starts, self.out, max_new or max(self.new), window, sinks, scale=scale, **kw)
        torch.cuda.synchronize()
        return self.out

    def check(self, window=0, sinks=0, max_new=None, scale=None, label="", skip_rows=()):
        sc = self.d ** -0.5 if scale is None else scale
        q = f64(self.q).reshape(-1, self.n_q, self.d)
        of = np.clip(np.nan_to_num(f64(self.scales), nan=O.LEAST, posinf=O.MOST), O.LEAST, O.MOST)
        with np.errstate(invalid="ignore"):
            k, v = values(self.k, 0) * of[:, None, :, None, 0], values(self.v, 1) * of[:, None, :, None, 1]
            ref, weight, mass = O.attention(q, k, v, self.tables, self.cached, self.starts, sc, window, sinks, max_new)
        got = f64(self.out).reshape(ref.shape)
        rows = np.ones(len(ref), dtype=bool)
        rows[self.starts[-1]:] = False
        rows[list(skip_rows)] = False
        assert np.all(got[self.starts[-1]:] == 7.0)                          # rows of no sequence stay as they were
        assert np.isfinite(got[rows]).all(), label
        tol = bound(ref, weight, mass, self.d)
        off = np.abs(got - ref)[rows]
        print(f"[parity] attention8 {label}: max abs {off.max():.3g}, of the bound {(off / (tol[rows] + 1e-30)).max():.2f}", flush=True)
        assert (off - tol[rows]).max() <= 1e-30, label
        return ref, got


NEW = [1, 5, 17, 1, 33, 1, 64, 1, 26, 1, 130]
CACHED = [0, 1, 15, 16, 31, 62, 33, 100, 517, 63, 95]


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (7, 3), (64, 0), (100, 70), (5000, 4)])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_attention(heads, window, sinks):
    print(f"attention8 {heads} window {window} sinks {sinks}", flush=True)
    b = Batch(heads, NEW, CACHED, seed=1)
    b.run(window, sinks)
    b.check(window, sinks, label=f"{heads} window {window} sinks {sinks}")


@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 5)])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_attention_of_single_tokens(heads, window, sinks):
    print(f"attention8 single tokens {heads}", flush=True)
    b = Batch(heads, [1] * 12, [0, 1, 14, 15, 16, 31, 62, 63, 64, 127, 128, 1000], seed=2)
    b.run(window, sinks)
    b.check(window, sinks, label=f"single tokens {heads}")


@pytest.mark.parametrize("n,c", [(1, 0), (2, 0), (2, 63), (4, 60), (8, 1000), (16, 48), (31, 1), (64, 0), (65, 64), (128, 77), (200, 1000), (255, 31), (300, 0), (513, 129)])
@pytest.mark.parametrize("heads", [(4, 2, 64), (40, 8, 128)], ids=str)
def test_chunk_sizes(heads, n, c):
    print(f"attention8 chunk of {n} behind {c}, {heads}", flush=True)
    b = Batch(heads, [n, 2, 1], [c, 5, 40], seed=n)
    for window, sinks in ((0, 0), (50, 2)):
        b.run(window, sinks)
        b.check(window, sinks, label=f"{heads} chunk of {n} behind {c} window {window}")


@pytest.mark.parametrize("seqs,c,n,heads", [(1, 20000, 1, (32, 8, 128)), (1, 9001, 40, (32, 8, 128)), (2, 6000, 64, (16, 2, 64)), (3, 4000, 1, (16, 1, 128)),
                                            (70, 300, 4, (4, 2, 64)), (300, 20, 2, (2, 1, 64)), (300, 90, 1, (8, 2, 128)), (1, 3000, 700, (8, 1, 128))])
def test_attention_long_and_many(seqs, c, n, heads):
    print(f"attention8 {seqs} sequences of {c} keys, {n} rows, {heads}", flush=True)
    rng = np.random.default_rng(seqs)
    cached = [max(0, c - int(rng.integers(0, c // 3 + 1))) for _ in range(seqs)]
    new = [int(rng.integers(1, n + 1)) if i else n for i in range(seqs)]
    b = Batch(heads, new, cached, seed=seqs)
    for window, sinks in ((0, 0), (777, 20)):
        b.run(window, sinks)
        b.check(window, sinks, label=f"{seqs} x {c} keys window {window}")


def test_scores_of_any_size_and_scale():
    print("attention8 large scores", flush=True)
    b = Batch((8, 2, 64), [20, 3, 1], [700, 40, 900], seed=3)
    b.q.mul_(30.0)
    # ascending scores along the keys, so that the reference of the softmax has to move again and again
    for s in (0, 2):
        for p in range(40):
            b.scales[b.tables[s, p]] *= 0.1 + 0.05 * p
    for scale in (0.5, 1e-4):
        b.run(scale=scale)
        b.check(scale=scale, label=f"scores times {scale}")


def test_scales_of_any_size():
    print("attention8 scales far apart", flush=True)
    b = Batch((8, 2, 64), [20, 1, 1], [300, 40, 500], seed=4)
    b.scales[:, :, 0] *= 1e-3
    b.q.mul_(100.0)
    b.scales[:, :, 1] *= 10.0 ** torch.linspace(-6, 6, len(b.scales), device=DEV)[:, None]
    b.run()
    b.check(label="values of 1e-6 to 1e6")
    b.scales[b.tables[0, 3], 0] = 0.0                       # counts as the least scale: keys of zero, values of nothing
    b.scales[b.tables[2, 5], 1, 1] = -3.0
    b.run()
    b.check(label="scales that are none")


def test_tables_windows_and_pages_that_were_given_back():
    print("attention8: entries that nobody sees", flush=True)
    b = Batch((10, 2, 128), [3, 1, 70], [1000, 2000, 700], seed=5, table_extra=2, tail_rows=4)
    window, sinks = 100, 20
    for s, (n, c) in enumerate(zip(b.new, b.cached)):
        low = c - window + 1
        for p in range(-(-sinks // PAGE), low // PAGE):
            b.tables[s, p] = -1 - p if p % 2 else 1 << 29
    b.tables[:, -2:] = 1 << 29
    b.dev[0] = dev_ints(b.tables)
    b.run(window, sinks)
    b.check(window, sinks, label="pages given back")


def test_sequences_that_break_a_rule_receive_zeros():
    print("attention8: broken sequences", flush=True)
    b = Batch((8, 2, 64), [4, 3, 2, 5, 1], [20, 30, 10, 50, 12], seed=6, tail_rows=3)
    b.cached = [20, -1, 1 << 20, 2 ** 31 - 2, 12]
    b.dev[1] = dev_ints(b.cached)
    b.run()
    ref, got = b.check(label="broken")
    assert not got[4:14].any() and got[:4].any()
    b.run(max_new=3)
    ref, got = b.check(max_new=3, label="more rows than said")
    assert not got[:14].any() and got[14].any()


@pytest.mark.parametrize("starts", [[0, 5, 3, 9], [-1, 2, 3, 9], [0, 2, 3, 10 ** 6]])
def test_rows_in_no_order_are_not_written(starts):
    b = Batch((8, 2, 64), [2, 1, 6], [5, 6, 7], seed=7)
    b.dev[2] = dev_ints(starts)
    b.run(max_new=9)
    assert bool((b.out == 7.0).all())


@pytest.mark.parametrize("heads", [(8, 2, 64), (8, 2, 128), (8, 8, 128)], ids=str)
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 3], [130, 70, 2]], ids=str)
def test_codes_that_are_no_numbers_spoil_the_rows_that_see_them_only(new, heads):
    print(f"attention8: NaN codes, {new} {heads}", flush=True)
    window, sinks = 48, 5
    new = new + [2]                                          # (a sequence without any)
    b = Batch(heads, new, [45, 100, 200, 70], seed=8)
    where = [(0, 0, 1), (0, 1, 40), (1, 0, 100), (2, 1, 150), (2, 0, 200)]
    where += [(0, 1, 45 + new[0] // 2), (1, 0, 100 + new[1] // 2)]
    for s, side, pos in where:
        b.put(side, s, pos, NAN_CODE)
    b.run(window, sinks)
    spoilt = []
    for s, (n, c) in enumerate(zip(new, b.cached)):
        for i in range(n):
            if any(t == s and pos <= c + i and (pos > c + i - window or pos < sinks) for t, _, pos in where):
                spoilt.append(int(b.starts[s]) + i)
    assert len(spoilt) not in (0, sum(new))
    got = f64(b.out)
    assert np.isnan(got[spoilt]).all(1).all()
    b.check(window, sinks, label="rows beside", skip_rows=spoilt)


def spoilt_by(b, s, pos, window, sinks):
    """The rows that see a position of sequence s."""
    c = b.cached[s]
    return [int(b.starts[s]) + i for i in range(b.new[s]) if pos <= c + i and (window == 0 or pos > c + i - window or pos < sinks)]


@pytest.mark.parametrize("side", [0, 1], ids=["key", "value"])
@pytest.mark.parametrize("heads", [(16, 4, 64), (16, 2, 128), (4, 2, 128), (6, 6, 64)], ids=str)
@pytest.mark.parametrize("new,cached,window,sinks,at", [
    ([64], [0], 0, 0, (5, 0, 31, 32, 63)), ([64], [1000], 0, 0, (970, 999, 1000, 1031, 1063)), ([130], [0], 0, 0, (10, 63, 64, 100, 129)),
    ([600, 3], [40, 7], 0, 0, (20, 90, 320, 600)), ([200], [300], 100, 0, (201, 230, 260, 300, 390)), ([150], [500], 64, 20, (0, 15, 19, 437, 455, 500, 600)),
    ([64] + [24] * 59, [330] + [300] * 59, 0, 0, (5, 320, 335, 350, 380)), ([70] + [24] * 80, [330] + [300] * 80, 90, 70, (66, 242, 280, 335, 399))], ids=str)
def test_one_code_that_is_no_number_spoils_all_rows_of_a_tile_that_see_it(new, cached, window, sinks, at, heads, side):
    """One position at a time, in blocks that some rows of a tile see and others do not: tiles that are cut, and (many sequences) tiles that are not."""
    print(f"attention8: one NaN {'value' if side else 'key'}, {len(new)} sequences, {new[0]} behind {cached[0]} {heads}", flush=True)
    b = Batch(heads, new, cached, seed=30)
    for pos in at:
        b.put(side, 0, pos, NAN_CODE)
        b.run(window, sinks)
        spoilt = spoilt_by(b, 0, pos, window, sinks)
        bad = np.isnan(f64(b.out))
        b.put(side, 0, pos, 0x30)                            # (what it is does not reach the other rows)
        assert np.nonzero(bad.any(1))[0].tolist() == spoilt and bad[spoilt].all(), pos
        if pos == at[-1]:
            b.check(window, sinks, label=f"rows beside position {pos}", skip_rows=spoilt)


def test_strides_page_order_and_repetition():
    print("attention8: strided rows, other page orders", flush=True)
    a = Batch((12, 4, 128), NEW, CACHED, seed=9, q_pad=24, tail_rows=2)
    a.run()
    a.check(label="strided")
    first = a.out.clone()
    for seed in (5, 6):
        c = Batch((12, 4, 128), NEW, CACHED, seed=9, q_pad=24, tail_rows=2, perm_seed=seed, spare=40)
        c.run()
        assert torch.equal(c.out, first)
    a.run()
    assert torch.equal(a.out, first)


def spoilt_workspace(b, max_new):
    """Of the size asked for, all bytes set: counts of -1, sums that are no numbers."""
    return torch.full((C8.gllm_op_attention8_workspace_bytes(b.n_q, b.n_kv, b.d, max_new),), 255, dtype=torch.uint8, device=DEV)


def test_scales_whose_product_with_the_scores_leaves_the_range():
    print("attention8 products out of range", flush=True)
    b = Batch((8, 2, 64), [20, 1, 3], [60, 70, 40], seed=14)
    b.scales[:, :, 0] = 1e-30
    b.run(scale=1e-30)
    b.check(scale=1e-30, label="scale 1e-30 over scales of 1e-30")
    b.scales[:, :, 0] = 1e30
    b.q.zero_()
    b.run(scale=2e38)
    b.check(scale=2e38, label="queries of zeros, scale 2e38 over scales of 1e30")


@pytest.mark.parametrize("n", [1, 20, 40])
def test_keys_of_low_weight_whose_values_are_all_zeros_count_in_the_sum(n):
    """One key of a score 27 above (in base 2) the 2^24 behind it, whose pages of zeros have the least scale: in the sum of the weights they are an
    eighth (and 16 of them, a lane's in a block, 2^-23, what float adds to 1 without rounding).  As many KV heads as compute units, so that the keys are
    cut into few parts; 1 column, 20, and a tile of 40."""
    print(f"attention8: 2^24 keys of zeros, {n} rows", flush=True)
    heads, keys = 256, 1 << 24
    b = Batch((heads, heads, 64), [n], [32], seed=31)
    first, rest = b.tables[0, 0], b.tables[0, 1]
    b.tables = np.full((1, keys // PAGE + 4), rest, dtype=np.int32)
    b.tables[0, 0] = first
    b.cached = [keys]
    b.dev[0], b.dev[1] = dev_ints(b.tables), dev_ints(b.cached)
    b.k.zero_()
    b.v.zero_()
    b.put(0, 0, 0, 0x38)                                     # code of 1
    b.put(1, 0, 0, 0x38)
    b.scales.fill_(1.0)
    b.scales[int(rest), :, 1] = O.LEAST
    b.q.fill_(1.0)
    above = 27.0
    b.run(scale=above * np.log(2) / 64)
    total = 1 + (keys + np.arange(n)) * 2.0 ** -above
    want = np.broadcast_to((1 / total)[:, None], (n, heads * 64))
    tol = bound(want, want, np.full(n, above * np.log(2)), 64)
    off = np.abs(f64(b.out) - want)
    print(f"[parity] attention8 keys of zeros: max abs {off.max():.3g}, of the bound {(off / tol).max():.2f}", flush=True)
    assert (off <= tol).all()


@pytest.mark.parametrize("heads", [(16, 4, 64), (8, 1, 128)], ids=str)
@pytest.mark.parametrize("new", [1, 3, 100])
def test_pages_of_zeros_under_large_scales(new, heads):
    """Keys of large scores whose values are zeros: their scale does not matter, and they count as any others."""
    print(f"attention8: zeros under scales of 2^100, {new} rows {heads}", flush=True)
    b = Batch(heads, [new], [300], seed=32)
    b.q.mul_(7.0)
    for page in range(18):
        b.scales[b.tables[0, page], :, 0] = 0.01 if page >= 4 else 1e-5
        if page >= 4:
            b.v[b.tables[0, page]] = 0
            b.scales[b.tables[0, page], :, 1] = float("inf") if page % 2 else 2.0 ** 100
    b.run()
    b.check(label=f"zeros under scales of 2^100 {heads}")


@pytest.mark.parametrize("seqs,n", [(17, 40), (70, 20)])
def test_shared_prefix_of_more_pages_than_a_tile_holds_ids_of(seqs, n):
    """One prefix for all sequences, whose tiles are too many to be cut."""
    print(f"attention8 {seqs} sequences over one prefix", flush=True)
    prefix = 562 * PAGE
    b = Batch((8, 8, 64), [n] * seqs, [prefix] + [0] * (seqs - 1), seed=15)
    own = -(-n // PAGE)
    for s in range(1, seqs):
        b.tables[s, 562:562 + own] = b.tables[s, :own]
        b.tables[s, :562] = b.tables[0, :562]
    b.cached = [prefix] * seqs
    b.dev[0], b.dev[1] = dev_ints(b.tables), dev_ints(b.cached)
    for window, sinks in ((0, 0), (8500, 100)):
        b.run(window, sinks)
        b.check(window, sinks, label=f"{seqs} sequences over one prefix, window {window}")


@pytest.mark.parametrize("window,sinks", [(0, 0), (8500, 100)])
def test_tiles_of_128_dims_over_more_pages_than_they_hold_ids_of(window, sinks):
    """One prefix for all sequences, whose tiles are too many to be cut: units of 142 blocks and, with a window, of 137."""
    print(f"attention8 one prefix, 128 dims, window {window}", flush=True)
    seqs, n, prefix = 34, 40, 562 * PAGE
    b = Batch((8, 8, 128), [n] * seqs, [prefix] + [0] * (seqs - 1), seed=34)
    for s in range(1, seqs):
        b.tables[s, 562:565] = b.tables[s, :3]
        b.tables[s, :562] = b.tables[0, :562]
    b.cached = [prefix] * seqs
    b.dev[0], b.dev[1] = dev_ints(b.tables), dev_ints(b.cached)
    b.run(window, sinks)
    b.check(window, sinks, label=f"one prefix, 128 dims, window {window}")


@pytest.mark.parametrize("new,cached", [([1], [400]), ([1, 40], [400, 10]), ([2, 30], [385, 3]), ([1, 1, 20], [383, 384, 500]), ([1, 1], [100, 449])], ids=str)
def test_streams_about_as_long_as_are_cut(new, cached):
    print(f"attention8 streams {new} {cached}", flush=True)
    b = Batch((16, 2, 64), new, cached, seed=16)
    b.run(workspace=spoilt_workspace(b, max(new)))
    b.check(label=f"streams {new} {cached}")


@pytest.mark.parametrize("heads,most", [((16, 1, 128), 1), ((4, 2, 64), 8), ((32, 8, 128), 4), ((8, 8, 64), 1)], ids=str)
@pytest.mark.parametrize("seqs", [40, 64, 65, 200, 256, 257])
def test_streams_of_very_different_lengths(seqs, heads, most):
    print(f"attention8 {seqs} streams, {heads}", flush=True)
    rng = np.random.default_rng(seqs)
    cached = [int(rng.choice([0, 1, 15, 63, 64, 320, 383, 384, 448, 1500])) for _ in range(seqs)]
    cached[3], cached[7] = 5000, 9000
    new = [int(rng.integers(0 if i % 3 else 1, most + 1)) for i in range(seqs)]
    new[3] = most
    b = Batch(heads, new, cached, seed=17)
    ws = spoilt_workspace(b, most)
    for window, sinks in ((0, 0), (1000, 130)):
        ws.fill_(255)
        b.run(window, sinks, max_new=most, workspace=ws)
        b.check(window, sinks, max_new=most, label=f"{seqs} streams {heads} window {window}")


@pytest.mark.parametrize("heads,most", [((32, 8, 128), 8), ((40, 8, 128), 6), ((16, 1, 128), 2), ((8, 8, 128), 32), ((7, 1, 64), 4), ((4, 2, 64), 16), ((8, 8, 64), 17)], ids=str)
@pytest.mark.parametrize("seqs", [1, 12, 65, 256, 257])
def test_a_few_rows_of_each_sequence(seqs, heads, most):
    """Between 17 and 32 columns."""
    print(f"attention8 {seqs} sequences of up to {most} rows, {heads}", flush=True)
    rng = np.random.default_rng(seqs)
    cached = [int(rng.choice([0, 1, 15, 48, 63, 320, 383, 384, 900])) for _ in range(seqs)]
    new = [int(rng.integers(1, most + 1)) for _ in range(seqs)]
    cached[0], new[0] = 7000, most
    b = Batch(heads, new, cached, seed=28, tail_rows=3)
    ws = spoilt_workspace(b, most)
    for window, sinks, broken in ((0, 0, False), (70, 10, False), (900, 130, True)):
        if broken and seqs > 4:
            b.cached[3] = -1
            b.dev[1] = dev_ints(b.cached)
        b.out.fill_(7.0)
        ws.fill_(255)
        b.run(window, sinks, workspace=ws)
        b.check(window, sinks, max_new=most, label=f"{seqs} of up to {most} rows {heads} window {window}")
    want = b.out.clone()
    b.run(900, 130, workspace=ws)
    assert torch.equal(b.out, want)


@pytest.mark.parametrize("heads,new", [((8, 2, 128), [8, 3, 5]), ((8, 2, 64), [7, 1, 8]), ((16, 1, 64), [2, 1, 2])], ids=str)
def test_no_numbers_among_a_few_rows(heads, new):
    print(f"attention8: NaN codes, {new} {heads}", flush=True)
    window, sinks = 48, 5
    b = Batch(heads, new, [45, 100, 200], seed=29)
    where = [(0, 0, 45 + new[0] // 2), (0, 1, 40), (1, 1, 100), (2, 0, 201), (2, 1, 3), (1, 0, 60)]
    for s, side, pos in where:
        b.put(side, s, pos, NAN_CODE)
    b.run(window, sinks)
    spoilt = [int(b.starts[s]) + i for s, (n, c) in enumerate(zip(new, b.cached)) for i in range(n)
              if any(t == s and pos <= c + i and (pos > c + i - window or pos < sinks) for t, _, pos in where)]
    got = f64(b.out)
    assert np.isnan(got[spoilt]).all(1).all()
    rest = [r for r in range(len(got)) if r not in spoilt]
    assert np.isfinite(got[rest]).all()
    if rest:
        b.check(window, sinks, label="rows beside", skip_rows=spoilt)


@pytest.mark.parametrize("heads", [(8, 2, 64), (12, 4, 128), (16, 1, 128)], ids=str)
@pytest.mark.parametrize("seqs", [30, 64, 65, 150, 256, 257, 400])
def test_hybrids_of_every_kind_of_sequence(seqs, heads):
    print(f"attention8 hybrid of {seqs}, {heads}", flush=True)
    rng = np.random.default_rng(seqs)
    new = [int(rng.choice([0, 1, 1, 1, 2, 5, 40, 130])) for _ in range(seqs)]
    cached = [int(rng.choice([0, 1, 16, 70, 383, 500, 1300])) for _ in range(seqs)]
    new[2], new[5], cached[5], new[seqs - 1], cached[seqs - 1] = 300, 1, 6000, 7, 2500
    b = Batch(heads, new, cached, seed=18, tail_rows=5)
    ws = spoilt_workspace(b, 300)
    for window, sinks, broken in ((0, 0, False), (200, 17, False), (0, 0, True)):
        if broken:
            for s in (0, 9, seqs - 2):
                b.cached[s] = [-3, 1 << 21, 2 ** 31 - 1][s % 3]
            b.dev[1] = dev_ints(b.cached)
        b.out.fill_(7.0)
        ws.fill_(255)
        b.run(window, sinks, max_new=300, workspace=ws)
        b.check(window, sinks, max_new=300, label=f"hybrid of {seqs} {heads} window {window}")
    b.out.fill_(7.0)
    ws.fill_(255)
    starts = b.starts.copy()
    starts[seqs // 2] += 10 ** 6
    b.dev[2] = dev_ints(starts)
    b.run(max_new=300, workspace=ws)
    assert bool((b.out == 7.0).all())


@pytest.mark.parametrize("most", [2, 12])
def test_more_sequences_than_runs_of_64(most):
    print("attention8 5000 sequences", flush=True)
    rng = np.random.default_rng(19)
    new, cached = rng.integers(0, most + 1, 5000).tolist(), rng.integers(0, 40, 5000).tolist()
    cached[4321] = 3000
    new[4321] = most
    b = Batch((4, 2, 64), new, cached, seed=19)
    b.run(workspace=spoilt_workspace(b, most))
    b.check(label=f"5000 sequences of up to {most}")


# ---- refusals, streams, graphs -----------------------------------------------------------------------------------------------

def test_binding_refuses_what_does_not_fit():
    b = Batch((8, 2, 64), [2, 1], [25, 46], seed=10)         # (tables of three entries, which every other one of is no table)
    tables, cached, starts = b.dev
    for change in (dict(q=b.q.float()), dict(q=b.q[:, :100]), dict(k=b.k.float()), dict(v=b.v[:, :1]), dict(scales=b.scales[:1]), dict(tables=tables.long()),
                   dict(starts=starts[:2]), dict(out=b.out[:1]), dict(scales=b.scales.double()), dict(k=b.k[:, ::2]), dict(tables=tables[:, ::2])):
        x = {**dict(q=b.q, k=b.k, v=b.v, scales=b.scales, tables=tables, cached=cached, starts=starts, out=b.out), **change}
        with pytest.raises(B.GllmError):
            C8.gllm_op_attention8(*x.values(), 2)
    with pytest.raises(B.GllmError):
        C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, tables, cached, starts, b.out, 2, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(B.GllmError):
        C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, tables, cached, starts, b.out, 2, stream=torch.cuda.current_stream().cuda_stream)
    assert bool((b.out == 7.0).all())
    s = Store((4, 2, 64), [(0, 3)], seed=1)
    with pytest.raises(B.GllmError):
        C8.gllm_op_norm_rope_store8(s.qkv, s.gains[0][:32], None, 1e-6, s.rope, dev_ints([0] * 3), dev_ints([0, 1, 2]), s.q_out, s.k, s.v, s.scales)
    with pytest.raises(B.GllmError):
        C8.gllm_op_norm_rope_store8(s.qkv.half(), None, None, 1e-6, s.rope, dev_ints([0] * 3), dev_ints([0, 1, 2]), s.q_out, s.k, s.v, s.scales)
    i = dev_ints([1, 2])
    with pytest.raises(B.GllmError):
        C8.gllm_op_step_maps(i, i, i, i.view(2, 1), 5, i, i, i, i)


@pytest.mark.parametrize("max_new", [1, 8, 40])
def test_errors_of_the_runtime_are_no_lack_of_capacity(max_new):
    """An error of the runtime that nobody has read yet is returned by the next call that reads it, as one of the runtime."""
    b = Batch((8, 2, 64), [1, 1], [25, 46], seed=33)
    ws = spoilt_workspace(b, max_new)
    torch.cuda.synchronize()
    hip = C8._lib()
    hip.hipGetDeviceCount.argtypes = [C.c_void_p]
    hip.hipPeekAtLastError.argtypes = hip.hipGetLastError.argtypes = []
    try:
        assert hip.hipGetDeviceCount(None) == INVALID_VALUE and hip.hipPeekAtLastError() == INVALID_VALUE
        with pytest.raises(B.GllmError) as e:
            C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, *b.dev, b.out, max_new, workspace=ws)
        assert e.value.status == HIP
    finally:
        hip.hipGetLastError()
    b.run(max_new=max_new)
    b.check(max_new=max_new, label="behind an error")


def test_codes_may_be_given_as_float8():
    b = Batch((8, 2, 64), [2, 1], [50, 60], seed=11)
    first = b.run().clone()
    b.k, b.v = b.k.view(torch.float8_e4m3fn), b.v.view(torch.float8_e4m3fn)
    assert torch.equal(b.run(), first)


def test_two_calls_at_once_on_streams_of_their_own():
    print("attention8 on two streams", flush=True)
    batches = [Batch((32, 8, 128), [1] * 8 + [100], [3000 + 100 * i for i in range(8)] + [500], seed=s) for s in (1, 2)]
    alone = [b.run().clone() for b in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    for b in batches:
        b.out.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(5):
        for b, st in zip(batches, streams):
            C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, *b.dev, b.out, 100, stream=st)
    torch.cuda.synchronize()
    for b, want in zip(batches, alone):
        assert torch.equal(b.out, want)


def test_a_step_captured_and_replayed_grows_its_sequences():
    """Maps, store and attention of decode steps in one graph; the lengths, the list of free pages and the rows change between replays.  Every
    replay against the eager calls on a second set of buffers."""
    print("a step from a graph", flush=True)
    n_q, n_kv, d = heads = (8, 2, 64)
    seqs, pages, entries, pad = 5, 60, 8, 3
    g = torch.Generator(device=DEV).manual_seed(3)
    rope = rope_table(256, d)
    gain = (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).bfloat16()

    class Side:
        def __init__(self):
            self.k, self.v, self.scales = empty_pool(pages, n_kv, d)
            self.tables = torch.full((seqs, entries), -1, dtype=torch.int32, device=DEV)
            self.new, self.cached, self.free = dev_ints([1] * seqs), dev_ints([0] * seqs), dev_ints(range(12))
            self.maps = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (seqs + 1, rows, rows, 2)]
            self.qkv = torch.zeros(rows, (n_q + 2 * n_kv) * d, device=DEV)
            self.q, self.out = (torch.full((rows, n_q * d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            self.ws = torch.empty(C8.gllm_op_attention8_workspace_bytes(n_q, n_kv, d, 20), dtype=torch.uint8, device=DEV)

        def step(self):
            C8.gllm_op_step_maps(self.new, self.cached, self.free, self.tables, pages, *self.maps)
            C8.gllm_op_norm_rope_store8(self.qkv, gain, gain, 1e-6, rope, self.maps[1], self.maps[2], self.q, self.k, self.v, self.scales)
            C8.gllm_op_attention8(self.q, self.k, self.v, self.scales, self.tables, self.cached, self.maps[0], self.out, 20, 40, 3, workspace=self.ws)

    rows = seqs * 20 + pad
    eager, graphed = Side(), Side()
    graphed.step()
    torch.cuda.synchronize()
    fresh = Side()
    for name in ("k", "v", "scales", "tables", "q", "out"):
        getattr(graphed, name).copy_(getattr(fresh, name))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    rng = np.random.default_rng(0)
    cached, used = np.zeros(seqs, dtype=np.int64), 0
    for step in range(6):
        new = rng.integers(1, 20, seqs) if step % 2 == 0 else np.ones(seqs, dtype=np.int64)
        need = int((-(-(cached + new) // PAGE) - -(-cached // PAGE)).sum())
        free = list(range(used, used + need)) + [pages + 5] * (12 - need)
        used += need
        x = torch.randn(rows, (n_q + 2 * n_kv) * d, generator=g, device=DEV)
        for side in (eager, graphed):
            side.new.copy_(dev_ints(new))
            side.cached.copy_(dev_ints(cached))
            side.free.copy_(dev_ints(free))
            side.qkv.copy_(x)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("k", "v", "scales", "tables", "q", "out"):
            a, b = getattr(eager, name), getattr(graphed, name)
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (step, name)
        total = int(new.sum())
        assert graphed.maps[3].tolist() == [total, need]
        # the outputs against the oracle, on what the pool holds
        of = f64(eager.scales)
        with np.errstate(invalid="ignore"):
            k, v = values(eager.k, 0) * of[:, None, :, None, 0], values(eager.v, 1) * of[:, None, :, None, 1]
        q = f64(eager.q).reshape(rows, n_q, d)
        ref, weight, mass = O.attention(q, k, v, eager.tables.cpu().numpy(), cached, eager.maps[0].cpu().numpy(), d ** -0.5, 40, 3)
        got = f64(eager.out).reshape(ref.shape)[:total]
        ref, weight, mass = ref[:total], weight[:total], mass[:total]
        assert (np.abs(got - ref) <= bound(ref, weight, mass, d)).all(), step
        cached += new


@pytest.mark.parametrize("seqs", [20, 100])
def test_attention_captured_and_replayed_with_other_lengths(seqs):
    """Streams, tiles and broken sequences change places between replays, in a workspace that something else has written to."""
    print(f"attention8 of {seqs} from a graph", flush=True)
    heads, most = (12, 4, 128), 200
    rng = np.random.default_rng(seqs)
    b = Batch(heads, [most] + [4] * (seqs - 1), [4000] + [600] * (seqs - 1), seed=20, tail_rows=1500)
    ws = spoilt_workspace(b, most)
    tables, cached, starts = b.dev

    def call(workspace, out):
        C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, tables, cached, starts, out, most, workspace=workspace)

    b.k.copy_(torch.where(b.k & 0x7F == NAN_CODE, 0x20, b.k))            # (all slots and pages hold numbers)
    b.v.copy_(torch.where(b.v & 0x7F == NAN_CODE, 0x20, b.v))
    b.scales.nan_to_num_(nan=0.01)
    eager = torch.empty_like(b.out)
    call(None, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ws, b.out)
    for step in range(6):
        new = rng.choice([0, 1, 2, 5, 30], seqs)
        new[step] = [most, 1, 150, 4, 33, most][step]
        c = rng.integers(0, 580, seqs)
        c[0] = 3900 if step % 2 else 100
        if step % 3 == 2:
            c[step + 4] = -1
        cached.copy_(dev_ints(c))
        starts.copy_(dev_ints(np.concatenate([[0], np.cumsum(new)])))
        eager.fill_(7.0)
        b.out.fill_(7.0)
        ws.fill_(255)
        call(None, eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, b.out), step
        # and against the oracle
        b.new, b.cached, b.tables = new.tolist(), c.tolist(), tables.cpu().numpy()
        b.starts = starts.cpu().numpy()
        b.check(max_new=most, label=f"replay {step}")


def test_binding_refuses_lengths_that_do_not_fit_32_bits():
    b = Batch((8, 2, 64), [2, 1], [25, 46], seed=21)
    for change in (dict(max_new=(1 << 32) + 2), dict(window=1 << 32), dict(window=40, sinks=1 << 32), dict(window=-1), dict(max_new=-(1 << 32) + 2)):
        with pytest.raises(B.GllmError):
            C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, *b.dev, b.out, **{"max_new": 2, **change})
    assert bool((b.out == 7.0).all())


def test_binding_refuses_arrays_that_do_not_fit_32_bits():
    """Arrays of 2^32 and a few entries (not looked at), whose lengths have as many as a few in their lower half."""
    print("arrays beyond 32 bits", flush=True)
    far = torch.empty((1 << 32) + 48, dtype=torch.int32, device=DEV)
    few = far[:(1 << 32) + 2]
    one, two = dev_ints([1]), dev_ints([7, 7])
    out = [torch.full((n,), -99, dtype=torch.int32, device=DEV) for n in (2, 5, 5, 2)]
    tables = torch.full((1, 4), -5, dtype=torch.int32, device=DEV)
    with pytest.raises(B.GllmError):
        C8.gllm_op_step_maps(one, one, few, tables, 9, *out)
    with pytest.raises(B.GllmError):
        C8.gllm_op_step_maps(one, one, two, far.view(1, -1), 9, *out)
    with pytest.raises(B.GllmError):
        C8.gllm_op_step_maps(one, one, two, tables, 9, out[0], few, few, out[3])
    b = Batch((8, 2, 64), [2], [25], seed=35)
    with pytest.raises(B.GllmError):
        C8.gllm_op_attention8(b.q, b.k, b.v, b.scales, far.view(1, -1), *b.dev[1:], b.out, 2)
    torch.cuda.synchronize()
    assert all(bool((t == -99).all()) for t in out) and bool((b.out == 7.0).all())


def test_pools_beyond_4_gib():
    """The same pages at the far end of a large pool: the same bits."""
    print("a pool beyond 4 GiB", flush=True)
    heads, pages = (16, 8, 128), 270000
    k, v = (torch.zeros(pages, *shape, dtype=torch.uint8, device=DEV) for shape in ((8, 4, 8, 4, 16), (8, 128, 16)))
    scales = torch.ones(pages, 8, 2, device=DEV)
    assert k.numel() > 2 ** 32 and v.numel() > 2 ** 32
    b = Batch(heads, [1, 2, 60, 5], [500, 30, 700, 2000], seed=22)
    want = b.run().clone()
    few = b.k.shape[0]
    small = [x.clone() for x in (b.k, b.v, b.scales)]
    for big, x in zip((k, v, scales), small):
        big[pages - few:] = x
    b.k, b.v, b.scales = k, v, scales
    b.dev[0] = dev_ints(b.tables + (pages - few))
    b.out.fill_(7.0)
    assert torch.equal(b.run(), want)
    s = Store(heads, RUNS, seed=23)
    few = s.k.shape[0]
    for big, x in zip((k, v, scales), (s.k, s.v, s.scales)):
        big[pages - few:] = x
    s.run()
    want = [x.clone() for x in (s.q_out, s.k, s.v, s.scales)]
    s.q_out.fill_(7.0)
    s.k, s.v, s.scales = k, v, scales
    s.slots = s.slots + (pages - few) * PAGE
    s.run()
    assert torch.equal(s.q_out, want[0])
    for big, x in zip((k, v, scales), want[1:]):
        assert torch.equal(big[pages - few:].view(torch.uint8), x.view(torch.uint8))


def test_rows_whose_offsets_pass_32_bits():
    print("rows far apart", flush=True)
    far = 1 << 28
    b = Batch((8, 2, 128), [1, 20, 3], [100, 200, 50], seed=24)
    want = b.run().clone()
    rows, width = b.q.shape
    wide = torch.empty(rows, far, dtype=torch.bfloat16, device=DEV)
    assert rows * far > 2 ** 32
    wide[:, :width] = b.q
    b.q, b.out = wide[:, :width], wide[:, 4096:4096 + width]
    b.out.fill_(7.0)
    assert torch.equal(b.run(), want)
    s = Store((8, 2, 128), [(0, 16), (3, 4), (5, 1)], torch.bfloat16, seed=25)
    first = [x.clone() for x in (s.k, s.v, s.scales)]
    s.run()
    want = [x.clone() for x in (s.q_out, s.k, s.v, s.scales)]
    rows, width = s.qkv.shape
    wide[:rows, :width] = s.qkv
    s.qkv, s.q_out = wide[:rows, :width], wide[:rows, 4096:4096 + s.q_out.shape[1]]
    s.k, s.v, s.scales = first
    s.run()
    for a, x in zip((s.q_out, s.k, s.v, s.scales), want):
        assert torch.equal(a, x)


def test_binding_looks_at_every_tensor():
    """Each argument in turn of another type, on the CPU, with gaps or of another shape; nothing is written."""
    b = Batch((8, 2, 64), [2, 1], [25, 46], seed=26)
    s = Store((8, 2, 64), [(0, 3)], seed=27)
    row, entry = dev_ints([0] * 3), dev_ints([0, 1, 2])
    maps = [dev_ints(x) for x in ([2, 1], [25, 46], [1, 2], np.zeros((2, 3)), [0] * 3, [0] * 3, [0] * 3, [0] * 2)]
    calls = [(lambda *t: C8.gllm_op_attention8(*t, 2), [b.q, b.k, b.v, b.scales, *b.dev, b.out]),
             (lambda *t: C8.gllm_op_attention8(*t[:-1], 2, workspace=t[-1]), [b.q, b.k, b.v, b.scales, *b.dev, b.out, spoilt_workspace(b, 2)]),
             (lambda qkv, g, h, *t: C8.gllm_op_norm_rope_store8(qkv, g, h, 1e-6, *t), [s.qkv, *s.gains, s.rope, row, entry, s.q_out, s.k, s.v, s.scales]),
             (lambda *t: C8.gllm_op_step_maps(*t[:4], 9, *t[4:]), maps)]
    for call, tensors in calls:
        written = [t.clone() for t in tensors]
        for i, t in enumerate(tensors):
            gaps = torch.zeros(*t.shape, 2, dtype=t.dtype, device=DEV)[..., 0]
            for other in (t.double(), t.cpu(), gaps, t.new_zeros(()), t.new_zeros((2, 3, 5, 7))):
                with pytest.raises(B.GllmError):
                    call(*tensors[:i], other, *tensors[i + 1:])
        for t, was in zip(tensors, written):
            assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
        call(*tensors)
    torch.cuda.synchronize()
