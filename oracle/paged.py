"""Oracle for the paged key/value cache (test infrastructure only): float64 numpy, request by request.

The cache is [n_pages][n_kv][page][head_dim]; request i's key j is slot j % page of page
table[i][j // page].  Rows are packed request by request (cu); row r of request i sits at
position L_i + r and sees keys 0 .. L_i + r.
"""
from __future__ import annotations

import numpy as np


def keys_of(pool: np.ndarray, pages: np.ndarray, n: int) -> np.ndarray:
    """The first n keys that `pages` list: [n_kv][n][head_dim]."""
    x = pool[pages]                                            # [pages][n_kv][page][hd]
    return np.moveaxis(x, 1, 0).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """One row q [n_q][hd] over keys k, v [n_kv][n][hd]: out [n_q][hd], ln sum exp [n_q], sum_j p_j |v_j| [n_q][hd],
    max_j sum_d |q_d k_jd| / sqrt(hd) [n_q] (the scale of rounding in the values and in the scores)."""
    n_q, hd = q.shape
    G = n_q // k.shape[0]
    out, lse, mag, big = np.empty((n_q, hd)), np.empty(n_q), np.empty((n_q, hd)), np.empty(n_q)
    for h in range(n_q):
        kg, vg = k[h // G], v[h // G]
        s = kg @ q[h] / np.sqrt(hd)
        p = np.exp(s - s.max())
        out[h], lse[h], mag[h] = p @ vg / p.sum(), s.max() + np.log(p.sum()), p @ np.abs(vg) / p.sum()
        big[h] = (np.abs(kg) @ np.abs(q[h])).max() / np.sqrt(hd)
    return out, lse, mag, big


def paged_attn(q, kp, vp, table, cu, ctx, page):
    """All live rows; rows of requests without any are absent.  Arrays are float64 (values of the bf16 bits)."""
    M, n_q, hd = int(cu[-1]), q.shape[1], q.shape[2]
    out, lse, mag, big = np.zeros((M, n_q, hd)), np.zeros((M, n_q)), np.zeros((M, n_q, hd)), np.zeros((M, n_q))
    for i in range(len(ctx)):
        n = int(ctx[i] + cu[i + 1] - cu[i])
        if cu[i + 1] == cu[i]:
            continue
        pg = table[i, : -(-n // page)]
        k, v = keys_of(kp, pg, n), keys_of(vp, pg, n)
        for t in range(cu[i], cu[i + 1]):
            m = int(ctx[i] + t - cu[i] + 1)
            out[t], lse[t], mag[t], big[t] = attend(q[t], k[:, :m], v[:, :m])
    return dict(out=out, lse=lse, mag=mag, big=big)


def select_pages(q, kmin, kmax, n_sel, n_sink, n_local):
    """Pages one row reads for one kv head: q [G][hd]; kmin, kmax [pages][hd] of the pages it sees."""
    n = len(kmin)
    with np.errstate(invalid="ignore"):
        score = np.maximum(q, 0).sum(0) @ kmax.T + np.minimum(q, 0).sum(0) @ kmin.T
    forced = [j for j in range(n) if j < n_sink or j >= n - n_local]
    if n <= n_sel:
        return list(range(n))
    rest = [j for j in range(n) if j not in set(forced)]
    rest.sort(key=lambda j: (np.isnan(score[j]), -score[j] if not np.isnan(score[j]) else 0.0, j))
    return sorted((forced + rest)[:n_sel])


def paged_attn_sparse(q, kp, vp, kmin, kmax, table, cu, ctx, page, n_sel, n_sink, n_local):
    M, n_q, hd = int(cu[-1]), q.shape[1], q.shape[2]
    n_kv = kp.shape[1]
    G = n_q // n_kv
    out, lse, mag, big = np.zeros((M, n_q, hd)), np.zeros((M, n_q)), np.zeros((M, n_q, hd)), np.zeros((M, n_q))
    blocks = np.full((M, n_kv, n_sel), -1, dtype=np.int32)
    for i in range(len(ctx)):
        for t in range(cu[i], cu[i + 1]):
            p = int(ctx[i] + t - cu[i])
            seen = table[i, : p // page + 1]
            for g in range(n_kv):
                qs = slice(g * G, g * G + G)
                pick = select_pages(q[t, qs], kmin[seen, g], kmax[seen, g], n_sel, n_sink, n_local)
                blocks[t, g, : len(pick)] = pick
                m = (len(pick) - 1) * page + p % page + 1
                k, v = (x[seen[pick], g].reshape(1, -1, hd)[:, :m] for x in (kp, vp))
                out[t, qs], lse[t, qs], mag[t, qs], big[t, qs] = attend(q[t, qs], k, v)
    return dict(out=out, lse=lse, mag=mag, big=big, blocks=blocks)


def rotate(x: np.ndarray, pos: np.ndarray, theta: float) -> np.ndarray:
    """Rows x [rows][heads][hd] at positions pos: the complex rotation of pairs (j, j + hd/2)."""
    half = x.shape[-1] // 2
    ang = pos[:, None].astype(np.float64) * theta ** (-np.arange(half) / half)
    z = (x[..., :half] + 1j * x[..., half:]) * np.exp(1j * ang)[:, None]
    return np.concatenate([z.real, z.imag], axis=-1)
