"""Plain 64-bit reference of the latent operators: appending, the products of the absorbed form, attention over the cache of latents,
compaction; and the attention of the model itself, with keys and values of every head.  numpy only, request by request, written from the
definitions; shares no code with the product.

TEST INFRASTRUCTURE ONLY.  The pool is [pages, 16 tokens, latent + rope].
"""
from __future__ import annotations

import numpy as np

from .cache import PAGE, chains, page_of, rotate, token_rows


def append(c, latent, key, pool, norm=None, eps=0.0):
    """The pool after the call, in 64 bits (unrounded)."""
    pool = np.array(pool, dtype=np.float64)
    C = latent.shape[1]
    for b, _, row, slot, pos in token_rows(c):
        pg = page_of(c["table"][b], slot // PAGE, pool.shape[0])
        if pg < 0:
            continue
        z = np.asarray(latent[row], dtype=np.float64)
        if norm is not None:
            z = z / np.sqrt((z * z).mean() + eps) * np.asarray(norm, dtype=np.float64)
        pool[pg, slot % PAGE, :C] = z
        pool[pg, slot % PAGE, C:] = rotate(key[row][None], pos, c["inv_freq"], c["interleaved"], c["scale"])[0]
    return pool


def absorb(c, q, w_key):
    """[rows, heads, latent + rope] in 64 bits; rows behind the last request: zeros."""
    H, N, C = w_key.shape
    got = np.zeros((q.shape[0], H, C + q.shape[2] - N))
    for _, _, row, _, pos in token_rows(c):
        for h in range(H):
            got[row, h, :C] = np.asarray(q[row, h, :N], dtype=np.float64) @ np.asarray(w_key[h], dtype=np.float64)
        got[row, :, C:] = rotate(q[row, :, N:], pos, c["inv_freq"], c["interleaved"], c["scale"])
    return got


def expand(x, w_value):
    return np.stack([np.asarray(x[:, h], dtype=np.float64) @ np.asarray(w_value[h], dtype=np.float64).T for h in range(w_value.shape[0])], 1)


def visible(c, b, num_pages):
    """(pool row of every position of request b (0 where there is none), [nodes, positions]: which are seen)."""
    o, e, ctx = int(c["offsets"][b]), int(c["offsets"][b + 1]), int(c["ctx"][b])
    n = e - o
    up = chains(None if c["parent"] is None else c["parent"][o:e], n)
    pg = np.array([page_of(c["table"][b], t // PAGE, num_pages) for t in range(ctx + n)], dtype=np.int64)
    sees = np.zeros((n, ctx + n), dtype=bool)
    sees[:, :ctx] = True
    for j in range(n):
        sees[j, [ctx + a for a in up[j]]] = True
    return np.where(pg >= 0, pg, 0) * PAGE + np.arange(ctx + n) % PAGE, sees & (pg >= 0)


def attend(c, q, pool, C, scale):
    """(out, lse, size, most, seen) in 64 bits: size = sum w |c|, most = the largest scale sum |q k| of the positions a row sees, seen = how many."""
    total, H, W = q.shape
    rows = np.asarray(pool, dtype=np.float64).reshape(-1, W)
    out, lse, size = np.zeros((total, H, C)), np.full((total, H), -np.inf), np.zeros((total, H, C))
    most, seen = np.zeros((total, H)), np.zeros((total, H))
    for b in range(len(c["ctx"])):
        o = int(c["offsets"][b])
        at, sees = visible(c, b, pool.shape[0])
        k = rows[at]
        for j in range(len(sees)):
            if not sees[j].any():
                continue
            kj, qj = k[sees[j]], np.asarray(q[o + j], dtype=np.float64)
            with np.errstate(invalid="ignore"):
                s = qj @ kj.T * scale
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                z = p.sum(-1, keepdims=True)
                out[o + j] = (p / z) @ kj[:, :C]
                lse[o + j] = (m + np.log(z))[:, 0]
                size[o + j] = (p / z) @ np.abs(kj[:, :C])
                most[o + j] = (np.abs(qj) @ np.abs(kj).T * scale).max(-1)
                seen[o + j] = sees[j].sum()
    return out, lse, size, most, seen


def compact(c, pool, stop):
    """(pool, new_len) after the call."""
    before, pool = np.array(pool), np.array(pool)
    new_len = np.array(c["ctx"], dtype=np.int32)
    for b in range(len(c["ctx"])):
        o, e, ctx = int(c["offsets"][b]), int(c["offsets"][b + 1]), int(c["ctx"][b])
        if not 0 <= int(stop[b]) < e - o:
            continue
        path = chains(None if c["parent"] is None else c["parent"][o:e], e - o)[int(stop[b])]
        new_len[b] = ctx + len(path)
        if c["parent"] is None:
            continue
        for d, j in enumerate(path):
            src, dst = (page_of(c["table"][b], (ctx + x) // PAGE, pool.shape[0]) for x in (j, d))
            if src >= 0 and dst >= 0:
                pool[dst, (ctx + d) % PAGE] = before[src, (ctx + j) % PAGE]
    return pool, new_len


def model(c, q, pool, w_key, w_value, scale):
    """The layer as the model defines it, keys and values of every head made from the latents: [total, heads, value] in 64 bits, queries unrotated as the
    step has them.  pool: rows with rotated shared keys."""
    H, N, C = w_key.shape
    rows = np.asarray(pool, dtype=np.float64).reshape(-1, pool.shape[-1])
    q = np.array(q, dtype=np.float64)
    for _, _, row, _, pos in token_rows(c):
        q[row, :, N:] = rotate(q[row, :, N:], pos, c["inv_freq"], c["interleaved"], c["scale"])
    out = np.zeros((q.shape[0], H, w_value.shape[1]))
    for b in range(len(c["ctx"])):
        o = int(c["offsets"][b])
        at, sees = visible(c, b, pool.shape[0])
        latent, shared = rows[at, :C], rows[at, C:]
        for h in range(H):
            k = np.concatenate([latent @ np.asarray(w_key[h], dtype=np.float64).T, shared], 1)
            v = latent @ np.asarray(w_value[h], dtype=np.float64).T
            for j in range(len(sees)):
                s = k[sees[j]] @ q[o + j, h] * scale
                p = np.exp(s - s.max())
                out[o + j, h] = p @ v[sees[j]] / p.sum()
    return out
