"""Plain float64 statements of the operators for several continuations of one sequence (include/gllm_branch.h), written from the
formulas: test infrastructure, slow on purpose, independent of the library."""
from __future__ import annotations

import numpy as np

PAGE = 16
MAX_NODES = 256


def chain(parents, i):
    """The nodes from a root down to node i, or None where node i is unused."""
    up = []
    while True:
        up.append(i)
        p = int(parents[i])
        if p == -1:
            return up[::-1]
        if not 0 <= p < i:
            return None
        i = p


def gather_k(k_pool, table, positions):
    """k_pool [pages][n_kv][d/8][16][8] -> [positions][n_kv][d]."""
    pages, slots = np.asarray(table)[positions // PAGE], positions % PAGE
    k = k_pool[pages, :, :, slots, :]
    return k.reshape(k.shape[0], k.shape[1], -1)


def gather_v(v_pool, table, positions):
    """v_pool [pages][n_kv][d][16] -> [positions][n_kv][d]."""
    pages, slots = np.asarray(table)[positions // PAGE], positions % PAGE
    return v_pool[pages, :, :, slots]


def tree_attention(q, k_pool, v_pool, tables, cached, starts, parents, scale, max_nodes=MAX_NODES):
    """float64 arrays; q [R][n_q][d].  Returns (out, weight): out [R][n_q][d] with NaN in the rows of no sequence, weight the sum
    of p |v| (what roundings of p are relative to), and the largest sum of |q_i k_i| * scale of a row and head."""
    rows, n_q, d = q.shape
    n_kv = k_pool.shape[1]
    out = np.full((rows, n_q, d), np.nan)
    weight = np.zeros((rows, n_q, d))
    mass = np.zeros((rows, n_q))
    for s in range(len(cached)):
        r0, r1, c = int(starts[s]), int(starts[s + 1]), int(cached[s])
        n = r1 - r0
        if n <= 0:
            continue
        out[r0:r1] = 0.0
        if n > max_nodes or c < 0 or c + n > len(tables[s]) * PAGE:
            continue
        for i in range(n):
            seen = chain(parents[r0:r1], i)
            if seen is None:
                continue
            at = np.concatenate([np.arange(c), c + np.asarray(seen)]).astype(np.int64)
            k, v = gather_k(k_pool, tables[s], at), gather_v(v_pool, tables[s], at)
            for h in range(n_q):
                kv = h // (n_q // n_kv)
                x = k[:, kv] @ q[r0 + i, h] * scale
                mass[r0 + i, h] = (np.abs(k[:, kv]) @ np.abs(q[r0 + i, h])).max() * scale
                p = np.exp(x - x.max())
                p /= p.sum()
                out[r0 + i, h] = p @ v[:, kv]
                weight[r0 + i, h] = p @ np.abs(v[:, kv])
    return out, weight, mass


def tree_commit(tokens, parents, sampled, starts, cached, tables, k_pool=None, v_pool=None):
    """Pools [layers][pages][n_kv]..., changed in place.  Returns path, count, next."""
    path = np.full(len(tokens), -7, dtype=np.int32)
    count, follow = np.zeros(len(cached), dtype=np.int32), np.full(len(cached), -1, dtype=np.int32)
    for s in range(len(cached)):
        r0, r1, c = int(starts[s]), int(starts[s + 1]), int(cached[s])
        n = r1 - r0
        path[r0:r1] = -1
        if n < 1 or n > MAX_NODES or c < 0 or c + n > len(tables[s]) * PAGE or parents[r0] != -1:
            continue
        walk = [0]
        while True:
            here = walk[-1]
            kids = [i for i in range(here + 1, n) if parents[r0 + i] == here and tokens[r0 + i] == sampled[r0 + here]]
            if not kids:
                break
            walk.append(kids[0])
        path[r0:r0 + len(walk)] = walk
        count[s], follow[s] = len(walk), sampled[r0 + walk[-1]]
        if k_pool is None:
            continue
        pages = k_pool.shape[1]
        for i, j in enumerate(walk):
            src, dst = int(tables[s][(c + j) // PAGE]), int(tables[s][(c + i) // PAGE])
            if i == j or not (0 <= src < pages and 0 <= dst < pages):
                continue
            k_pool[:, dst, :, :, (c + i) % PAGE] = k_pool[:, src, :, :, (c + j) % PAGE]
            v_pool[:, dst, :, :, (c + i) % PAGE] = v_pool[:, src, :, :, (c + j) % PAGE]
    return path, count, follow


def log_softmax(x):
    """Of one row; not-a-number counts as -infinity, +infinities share the probability."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    m = x.max()
    if m == -np.inf:
        return np.full_like(x, -np.inf)
    if m == np.inf:
        return np.where(x == np.inf, -np.log(np.sum(x == np.inf)), -np.inf)
    with np.errstate(over="ignore"):
        return x - m - np.log(np.exp(x - m).sum())


def beam_select(logits, scores, keep):
    """logits [S*W][V], scores [S][W].  Returns scores, beams, tokens [S][keep]: by the sum in 64 bits, equal ones by the beam, in a beam by
    the logit, then by the token."""
    seqs, beams = scores.shape
    vocab = logits.shape[1]
    out = np.full((seqs, keep), -np.inf), np.full((seqs, keep), -1, np.int32), np.full((seqs, keep), -1, np.int32)
    for s in range(seqs):
        total = np.full((beams, vocab), -np.inf)
        for b in range(beams):
            if np.isfinite(scores[s, b]):
                total[b] = np.float64(scores[s, b]) + log_softmax(logits[s * beams + b])
        flat, x = total.reshape(-1), logits[s * beams:(s + 1) * beams].reshape(-1)
        there = np.flatnonzero(flat > -np.inf)
        if len(there) > keep:                                                    # those that reach the keep-th best sum
            there = there[flat[there] >= np.partition(flat[there], -keep)[-keep]]
        order = there[np.lexsort((there % vocab, -x[there].astype(np.float64), there // vocab, -flat[there]))][:keep]
        out[0][s, :len(order)] = flat[order]
        out[1][s, :len(order)] = order // vocab
        out[2][s, :len(order)] = order % vocab
    return out
