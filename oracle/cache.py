"""Plain 64-bit reference of the cache operators: appending with position rotation, the 8-bit pages, attention over
them, compaction.  numpy only, request by request and entry by entry, written from the definitions; shares no code
with the product.

TEST INFRASTRUCTURE ONLY.  8-bit pools are held as the product lays them out - keys [pages, heads, D / 16, 16 tokens,
16], values [pages, heads, D, 16 tokens], uint8 codes - with fp32 scales [pages, heads].
"""
from __future__ import annotations

import numpy as np

PAGE = 16
LEAST_EXP, MOST_EXP = -100, 119


def _decode_table() -> np.ndarray:
    code = np.arange(256)
    sign, e, m = np.where(code & 0x80, -1.0, 1.0), (code >> 3) & 15, code & 7
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    x = np.where((code & 0x7f) == 0x7f, np.nan, x)
    return sign * x


E4M3 = _decode_table()


def e4m3_step(x) -> np.ndarray:
    """Distance of neighbouring e4m3 values around |x| (largest binade below 448 included)."""
    _, e = np.frexp(np.abs(np.asarray(x, dtype=np.float64)))
    return 2.0 ** (np.maximum(e - 1, -6) - 3.0)


def encode_e4m3(x) -> np.ndarray:
    """Nearest e4m3 codes (even on ties); beyond +-448 saturates, NaN stays NaN."""
    x = np.asarray(x, dtype=np.float64)
    step = e4m3_step(np.minimum(np.abs(x), 448.0))
    a = np.minimum(np.rint(np.minimum(np.abs(x), 448.0) / step) * step, 448.0)
    positive = E4M3[:127]
    code = np.searchsorted(positive, np.where(np.isnan(a), 0.0, a)).astype(np.uint8)
    code = np.where(np.signbit(x), code | 0x80, code)
    return np.where(np.isnan(x), 0x7f, code).astype(np.uint8)


def page_scale(amax: float) -> float:
    """Least power of two in range with amax <= 448 * scale."""
    e = LEAST_EXP
    while e < MOST_EXP and amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def chains(parent, n):
    """Ancestors-or-self of every node, root first.  A parent outside [-1, own index) makes a root."""
    got = []
    for j in range(n):
        up, a = [], j
        while a >= 0:
            up.append(a)
            p = a - 1 if parent is None else int(parent[a])
            a = p if p < a else -1
        got.append(up[::-1])
    return got


def rotate(x, pos, inv_freq, interleaved=False, scale=1.0):
    """x [heads, D] in 64 bits, rotated by one position."""
    x = np.array(x, dtype=np.float64)
    h = 0 if inv_freq is None else len(inv_freq)
    a = float(pos) * np.asarray(inv_freq if h else [], dtype=np.float64)
    for i in range(h):
        u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = scale * np.cos(a[i]), scale * np.sin(a[i])
        x1, x2 = x[:, u].copy(), x[:, w].copy()
        x[:, u], x[:, w] = x1 * c - x2 * s, x2 * c + x1 * s
    return x


def page_of(table_row, lp, num_pages):
    p = int(table_row[lp]) if lp < len(table_row) else -1
    return p if 0 <= p < num_pages else -1


def token_rows(c):
    """(request, index, row, slot, rotation position) of every new token of a case (a dict, see tests)."""
    for b in range(len(c["ctx"])):
        o, e = int(c["offsets"][b]), int(c["offsets"][b + 1])
        up = chains(None if c["parent"] is None else c["parent"][o:e], e - o) if c["parent"] is not None else None
        for i in range(e - o):
            depth = i if up is None else len(up[i]) - 1
            pos = int(c["positions"][o + i]) if c.get("positions") is not None else int(c["ctx"][b]) + depth
            yield b, i, o + i, int(c["ctx"][b]) + i, pos


def append(c, k_pool, v_pool):
    """Rotated queries [total, Hq, D] and pools [pages, heads, 16, D] after the call, all in 64 bits (unrounded)."""
    q = np.array(c["q"], dtype=np.float64)
    k_pool, v_pool = np.array(k_pool, dtype=np.float64), np.array(v_pool, dtype=np.float64)
    for b, _, row, slot, pos in token_rows(c):
        q[row] = rotate(c["q"][row], pos, c["inv_freq"], c["interleaved"], c["scale"])
        pg = page_of(c["table"][b], slot // PAGE, k_pool.shape[0])
        if pg >= 0:
            k_pool[pg, :, slot % PAGE] = rotate(c["k"][row], pos, c["inv_freq"], c["interleaved"], c["scale"])
            v_pool[pg, :, slot % PAGE] = c["v"][row]
    return q, k_pool, v_pool


def _put(pool, scale, pg, h, keys, entries, kept, least):
    """Slots {t: D entries (64 bits)} of one (page, head); `kept` committed slots before; least: scale that the entries need."""
    own = float(scale[pg, h])
    new = max(own, least) if kept else least
    view = pool[pg, h]
    if kept and new > own:
        part = view[:, :kept]                                     # (slots are the second axis of either layout)
        part[...] = encode_e4m3(E4M3[part] * (own / new))
    for t, x in entries.items():
        code = encode_e4m3(x / new)
        if keys:
            view[:, t] = code.reshape(-1, 16)
        else:
            view[:, t] = code
    scale[pg, h] = new


def append_quant(c, k_pool, v_pool, k_scale, v_scale):
    """(q, k_pool, v_pool, k_scale, v_scale, k_true): pools and scales after the call; k_true the unrounded keys by (page, head, slot)."""
    q = np.array(c["q"], dtype=np.float64)
    k_pool, v_pool, k_scale, v_scale = (np.array(x) for x in (k_pool, v_pool, k_scale, v_scale))
    fresh, truth = {}, {}
    for b, _, row, slot, pos in token_rows(c):
        q[row] = rotate(c["q"][row], pos, c["inv_freq"], c["interleaved"], c["scale"])
        pg = page_of(c["table"][b], slot // PAGE, k_pool.shape[0])
        if pg < 0:
            continue
        kept = max(int(c["ctx"][b]) - slot // PAGE * PAGE, 0)
        k = rotate(c["k"][row], pos, c["inv_freq"], c["interleaved"], c["scale"])
        for h in range(k.shape[0]):
            fresh.setdefault((pg, h), (kept, {}, {}))[1][slot % PAGE] = k[h]
            fresh[pg, h][2][slot % PAGE] = np.asarray(c["v"][row, h], dtype=np.float64)
            truth[pg, h, slot % PAGE] = k[h]
    for (pg, h), (kept, ks, vs) in fresh.items():
        for pool, scale, keys, entries in ((k_pool, k_scale, True, ks), (v_pool, v_scale, False, vs)):
            every = np.concatenate(list(entries.values()))
            amax = np.abs(every[np.isfinite(every)]).max(initial=0.0)
            _put(pool, scale, pg, h, keys, entries, kept, page_scale(amax))
    return q, k_pool, v_pool, k_scale, v_scale, truth


def attend(c, q, k_pool, v_pool, k_scale, v_scale, scale=None):
    """(out, lse) in 64 bits over 8-bit pools."""
    total, Hq, D = q.shape
    pages, Hkv = k_scale.shape
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    out, lse = np.zeros((total, Hq, D)), np.full((total, Hq), -np.inf)
    for b in range(len(c["ctx"])):
        o, e, ctx = int(c["offsets"][b]), int(c["offsets"][b + 1]), int(c["ctx"][b])
        n = e - o
        if n == 0:
            continue
        up = chains(None if c["parent"] is None else c["parent"][o:e], n)
        L = ctx + n
        pg = np.array([page_of(c["table"][b], t // PAGE, pages) for t in range(L)])
        there = pg >= 0
        sees = np.zeros((n, L), dtype=bool)
        sees[:, :ctx] = True
        for j in range(n):
            sees[j, [ctx + a for a in up[j]]] = True
        sees &= there
        slot = np.arange(L) % PAGE
        p0 = np.where(there, pg, 0)
        for h in range(Hkv):
            k = E4M3[k_pool[p0, h, :, slot, :].reshape(L, D)] * k_scale[p0, h, None].astype(np.float64)
            v = E4M3[v_pool[p0, h, :, slot]] * v_scale[p0, h, None].astype(np.float64)
            for j in range(n):
                if not sees[j].any():
                    continue
                for g in range(G):
                    with np.errstate(invalid="ignore"):
                        s = (k[sees[j]] @ np.asarray(q[o + j, h * G + g], dtype=np.float64)) * scale
                        m = s.max()
                        p = np.exp(s - m)
                        z = p.sum()
                        out[o + j, h * G + g] = (p / z) @ v[sees[j]]
                        lse[o + j, h * G + g] = m + np.log(z)
    return out, lse


def compact_quant(c, k_pool, v_pool, k_scale, v_scale, stop):
    """(k_pool, v_pool, k_scale, v_scale, new_len) after the call."""
    k_pool, v_pool, k_scale, v_scale = (np.array(x) for x in (k_pool, v_pool, k_scale, v_scale))
    before = [np.array(x) for x in (k_pool, v_pool, k_scale, v_scale)]
    new_len = np.array(c["ctx"], dtype=np.int32)
    pages, Hkv = k_scale.shape
    for b in range(len(c["ctx"])):
        o, e, ctx = int(c["offsets"][b]), int(c["offsets"][b + 1]), int(c["ctx"][b])
        if not 0 <= int(stop[b]) < e - o:
            continue
        path = chains(None if c["parent"] is None else c["parent"][o:e], e - o)[int(stop[b])]
        new_len[b] = ctx + len(path)
        if c["parent"] is None:
            continue
        for to_page in sorted({(ctx + d) // PAGE for d in range(len(path))}):
            dst = page_of(c["table"][b], to_page, pages)
            moves = {}
            for d, j in enumerate(path):
                src = page_of(c["table"][b], (ctx + j) // PAGE, pages)
                if (ctx + d) // PAGE == to_page and src >= 0:
                    moves[(ctx + d) % PAGE] = (src, (ctx + j) % PAGE)
            if dst < 0 or not moves:
                continue
            kept = max(ctx - to_page * PAGE, 0)
            for h in range(Hkv):
                for pool, scale, old, old_scale, keys in ((k_pool, k_scale, before[0], before[2], True),
                                                          (v_pool, v_scale, before[1], before[3], False)):
                    entries = {t: E4M3[old[p, h, :, s] if keys else old[p, h, :, s]].reshape(-1) * float(old_scale[p, h])
                               for t, (p, s) in moves.items()}
                    _put(pool, scale, dst, h, keys, entries, kept, max(float(old_scale[p, h]) for p, _ in moves.values()))
    return k_pool, v_pool, k_scale, v_scale, new_len
