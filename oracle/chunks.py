"""fp64 restatement of the caller's paged cache: ragged chunks of new tokens, rotation, append, attention.

Test infrastructure: numpy, a loop over sequences and rows, nothing shared with the library.  Arrays as the header has
them: pool [n_pages][Hkv][2][page][hd], rows [n_rows][heads][hd].
"""
from __future__ import annotations

import numpy as np


def positions(row_starts, kv_lens):
    """[(sequence, row, position)] of every row that belongs to a sequence."""
    out = []
    for s in range(len(kv_lens)):
        n = int(row_starts[s + 1]) - int(row_starts[s])
        out += [(s, int(row_starts[s]) + i, int(kv_lens[s]) - n + i) for i in range(n)]
    return out


def rotate(x, position, theta):
    """One row [heads][hd] turned by its position: pairs (j, j + hd/2), angle position theta^(-2j/hd)."""
    hd = x.shape[-1]
    angle = np.float64(position) * np.float64(theta) ** (-2.0 * np.arange(hd // 2) / hd)
    c, s = np.cos(angle), np.sin(angle)
    a, b = x[..., : hd // 2].astype(np.float64), x[..., hd // 2:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def append(pool, q, k, v, row_starts, kv_lens, page_table, theta):
    """(pool, q) after the append, fp64; rows of no sequence keep what q holds."""
    pool, turned, page = pool.astype(np.float64), q.astype(np.float64), pool.shape[3]
    for s, row, t in positions(row_starts, kv_lens):
        at = int(page_table[s, t // page])
        pool[at, :, 0, t % page] = rotate(k[row], t, theta)
        pool[at, :, 1, t % page] = v[row].astype(np.float64)
        turned[row] = rotate(q[row], t, theta)
    return pool, turned


def attend(pool, q, row_starts, kv_lens, page_table, out):
    """(outputs fp64, per output sum p |v|, per row and head the largest sum |q| |k| / sqrt(hd)); rows of no sequence keep
    `out`, and have 0 in the other two."""
    out, spread, scores = out.astype(np.float64), np.zeros(out.shape), np.zeros(out.shape[:2])
    Hkv, page, hd = pool.shape[1], pool.shape[3], pool.shape[4]
    group = q.shape[1] // Hkv
    gathered = {}
    for s, row, t in positions(row_starts, kv_lens):
        if t < 0:
            out[row] = 0.0
            continue
        if s not in gathered:
            kv = pool[page_table[s, : -(-int(kv_lens[s]) // page)].astype(np.int64)].astype(np.float64)
            gathered = {s: kv.transpose(1, 2, 0, 3, 4).reshape(Hkv, 2, -1, hd)}
        k, v = gathered[s][:, 0, : t + 1], gathered[s][:, 1, : t + 1]
        z = np.matmul(q[row].astype(np.float64).reshape(Hkv, group, hd), k.transpose(0, 2, 1)) / np.sqrt(hd)
        with np.errstate(invalid="ignore"):
            p = np.exp(z - z.max(axis=2, keepdims=True))
            p /= p.sum(axis=2, keepdims=True)
            out[row] = np.matmul(p, v).reshape(-1, hd)
            spread[row] = np.matmul(p, np.abs(v)).reshape(-1, hd)
            qa = np.abs(q[row].astype(np.float64)).reshape(Hkv, group, hd)
            scores[row] = (np.matmul(qa, np.abs(k).transpose(0, 2, 1)) / np.sqrt(hd)).max(axis=2).reshape(-1)
    return out, spread, scores
