"""Plain float64 statements of the operators over a KV cache held in 8 bits (include/gllm_cache8.h), written from the formulas: test
infrastructure, slow on purpose, independent of the library."""
from __future__ import annotations

import numpy as np

PAGE = 16
TOP = 448.0
LEAST, MOST = 2.0 ** -100, 2.0 ** 100
LAST = 2 ** 31 - 64
# The value of every code: sign, 4 bits of exponent (bias 7), 3 of mantissa; all seven lower bits set: not a number.
VALUES = np.array([np.nan if c & 0x7F == 0x7F else (-1.0 if c >> 7 else 1.0) * ((c & 7) * 2.0 ** -9 if c >> 3 & 15 == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                   for c in range(256)])


def round_e4m3(x):
    """The nearest values of the type, even where two are as near; |x| <= 448, not-a-numbers stay."""
    x = np.asarray(x, dtype=np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.clip(np.rint(x / step) * step, -TOP, TOP)


def half_step(x):
    """Half the distance of neighbouring values at |x|."""
    return 0.5 * 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)


def step_maps(new, cached, free, tables, num_blocks, rows):
    """Returns row_start, positions, slots, needed, tables."""
    tables = np.array(tables, dtype=np.int64)
    start, positions, slots = [0], np.zeros(rows, dtype=np.int64), np.full(rows, -1, dtype=np.int64)
    asked, pages, full = 0, 0, False
    for s, (n, c) in enumerate(zip(new, cached)):
        n, c = max(int(n), 0), int(c)
        good = c >= 0 and c + n <= min(tables.shape[1] * PAGE, LAST)
        held = -(-c // PAGE)
        need = -(-(c + n) // PAGE) - held if good else 0
        asked += n
        full = full or asked > rows
        r0 = start[-1]
        start.append(r0 if full else r0 + n)
        if good and not full:
            for i in range(need):
                tables[s, held + i] = free[pages + i] if pages + i < len(free) else -1
            for i in range(n):
                page = tables[s, (c + i) // PAGE]
                positions[r0 + i] = c + i
                if 0 <= page < num_blocks:
                    slots[r0 + i] = page * PAGE + (c + i) % PAGE
        pages += need
    return np.array(start), positions, slots, np.minimum([asked, pages], 2 ** 31 - 1), tables


def norm_rotate(x, gain, eps, cs):
    """x [..., d], cs [d/2][2]; returns the result and what roundings of the rotation are relative to."""
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    h = x.shape[-1] // 2
    a, b, co, si = x[..., :h], x[..., h:], cs[:, 0], cs[:, 1]
    with np.errstate(invalid="ignore"):                         # (infinities)
        return (np.concatenate([a * co - b * si, b * co + a * si], -1),
                np.concatenate([np.abs(a * co) + np.abs(b * si), np.abs(b * co) + np.abs(a * si)], -1))


def slots_of_k(k):
    """[pages][n_kv][4][d/16][4][16] -> [pages][16][n_kv][d]."""
    p, n_kv, d = k.shape[0], k.shape[1], 16 * k.shape[3]
    return k.transpose(0, 2, 4, 1, 3, 5).reshape(p, PAGE, n_kv, d)


def slots_of_v(v):
    """[pages][n_kv][d][16] -> [pages][16][n_kv][d]."""
    return v.transpose(0, 3, 1, 2)


def attention(q, k, v, tables, cached, starts, scale, window=0, sinks=0, max_new=None):
    """q [R][n_q][d]; k, v [pages][16][n_kv][d] values.  Returns out [R][n_q][d] with NaN in the rows of no sequence, the weights' sum of
    p |v| (what roundings of p are relative to), and the largest sum of |q_i k_i| * scale of a row and head."""
    rows, n_q, d = q.shape
    n_kv = k.shape[2]
    out, weight, mass = np.full((rows, n_q, d), np.nan), np.zeros((rows, n_q, d)), np.zeros((rows, n_q))
    for s in range(len(cached)):
        r0, r1, c = int(starts[s]), int(starts[s + 1]), int(cached[s])
        n = r1 - r0
        if n <= 0:
            continue
        out[r0:r1] = 0.0
        if (max_new is not None and n > max_new) or c < 0 or c + n > min(len(tables[s]) * PAGE, LAST):
            continue
        pos, j = np.arange(c, c + n)[:, None], np.arange(c + n)[None, :]
        seen = j <= pos
        if window:
            seen &= (j > pos - window) | (j < sinks)
        at = np.nonzero(seen.any(0))[0]                         # positions that some row sees: no others are looked up
        page = np.asarray(tables[s])[at // PAGE]
        kk, vv, seen = k[page, at % PAGE], v[page, at % PAGE], seen[:, at]
        for h in range(n_q):
            kv = h // (n_q // n_kv)
            with np.errstate(invalid="ignore"):
                x = np.where(seen, q[r0:r1, h] @ kk[:, kv].T * scale, -np.inf)
                mass[r0:r1, h] = np.where(seen, np.abs(q[r0:r1, h]) @ np.abs(kk[:, kv]).T * scale, 0).max(1)
                p = np.exp(x - x.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[r0:r1, h] = p @ vv[:, kv]
                weight[r0:r1, h] = p @ np.abs(vv[:, kv])
    return out, weight, mass
