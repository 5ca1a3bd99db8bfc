"""Plain forms of the operators around the paged cache, in numpy with 64-bit integers and floats: what the GPU tests compare with.
One row of one head at a time, from the definitions in include/intattn.h."""
import math

import numpy as np


def lut(bits=5, clip=6.6):
    top = (1 << bits) - 1
    return np.array([math.floor(255 * math.exp(-clip * i / top) + 0.5) for i in range(top)] + [0], dtype=np.int64)


def turned(x, pos, freq, axis, halves, inverse=False):
    """x [B, H, L, d] in 64 bits with pair i of the first 2 len(freq) channels turned by pos[axis[i]] freq[i] (pos [axes, B, L])."""
    y = x.astype(np.float64).copy()
    n = len(freq)
    for i in range(n):
        a, b = (i, i + n) if halves else (2 * i, 2 * i + 1)
        t = pos[axis[i]].astype(np.float64) * freq[i] * (-1 if inverse else 1)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def int8(x, scale):
    """rint(fl32(x / scale)), ties to even, clamped; x and scale float32."""
    return np.clip(np.rint((x.astype(np.float32) / np.asarray(scale, dtype=np.float32)).astype(np.float32)), -127, 127).astype(np.int8)


def page_of(table_row, slot, page_size, n_pages):
    p = int(table_row[slot // page_size])
    return p if 0 <= p < n_pages else None


def gather(pages, table_row, length, head):
    """(rows [length, d], there [length]) of one head of a sequence; rows of pages that are not there are 0."""
    n_pages, _, ps, d = pages.shape
    rows, there = np.zeros((length, d), dtype=np.int64), np.zeros(length, dtype=bool)
    for j in range(length):
        p = page_of(table_row, j, ps, n_pages)
        if p is not None:
            rows[j], there[j] = pages[p, head, j % ps], True
    return rows, there


def requantize(acc, s_v, s_o):
    m, e = math.frexp(float(s_v) / (255.0 * float(s_o)))
    M = math.floor(m * 2.0 ** 31 + 0.5)
    if M == 1 << 31:
        M, e = 1 << 30, e + 1
    sh = 31 - e
    return np.clip((acc * M + (1 << (sh - 1))) >> sh, -127, 127)


def good(s):
    return math.isfinite(float(s)) and float(s) > 0


def attend(q, scale_q, k_pages, v_pages, table, lens, scale_k, scale_v, scale_out=None, n_new=None, weight=None, decay=1.0, bits=5, clip=6.6,
           capacity=None):
    """(accumulators, int8 output, output in real numbers, new weights) of cache_forward."""
    B, Hq, L, d = q.shape
    Hkv = k_pages.shape[1]
    G, top, table8 = Hq // Hkv, (1 << bits) - 1, lut(bits, clip)
    acc = np.zeros((B, Hq, L, d), dtype=np.int64)
    out8, real = np.zeros_like(q), np.zeros((B, Hq, L, d))
    new_weight = None if weight is None else weight.astype(np.float64).copy()
    capacity = capacity or table.shape[1] * k_pages.shape[2]
    one = lambda s, i: s[i] if len(s) > 1 else s[0]
    for b in range(B):
        n = min(max(int(lens[b]), 0), capacity)
        fresh = min(L, n) if n_new is None else min(max(int(n_new[b]), 0), min(L, n))
        for h in range(Hkv):
            keys, there = gather(k_pages, table[b], n, h)
            values, _ = gather(v_pages, table[b], n, h)
            if new_weight is not None:
                new_weight[b, h, :n] *= decay
            for head in range(h * G, (h + 1) * G):
                for t in range(fresh):
                    sq, sk, sv = scale_q[b, head, t], one(scale_k, h), one(scale_v, h)
                    so = sv if scale_out is None else one(scale_out, head)
                    sees = there & (np.arange(n) <= n - fresh + t)
                    if not (good(sq) and good(sk) and good(sv) and good(so)) or not sees.any():
                        continue
                    a = keys @ q[b, head, t].astype(np.int64)
                    c = math.floor(clip / ((float(sq) * float(sk)) / math.sqrt(d)) + 0.5)
                    c = min(max(c, 1), 1 << 30)
                    away = np.minimum(a[sees].max() - a, c)
                    e = np.where(sees, table8[np.clip((2 * top * away + c) // (2 * c), 0, top)], 0)
                    p = (510 * e + e.sum()) // (2 * e.sum())
                    acc[b, head, t] = p @ values
                    out8[b, head, t] = requantize(acc[b, head, t], sv, so)
                    real[b, head, t] = acc[b, head, t] * (float(sv) / 255.0)
                    if new_weight is not None:
                        new_weight[b, h, :n] += e / e.sum()
    return acc, out8, real, new_weight


def evict(k_pages, v_pages, table, lens, weight, order, keep, total=None, sink=0, recent=0, capacity=None):
    """Copies of (k_pages, v_pages, weight, order, lens) after cache_evict; order None: slots."""
    k_pages, v_pages, weight, lens = k_pages.copy(), v_pages.copy(), weight.copy(), lens.copy()
    slots = np.broadcast_to(np.arange(weight.shape[2], dtype=np.int32), weight.shape).copy()
    order = slots if order is None else order.copy()
    n_pages, Hkv, ps, _ = k_pages.shape
    capacity = capacity or table.shape[1] * ps
    for b in range(len(lens)):
        n = min(max(int(lens[b]), 0), capacity)
        lens[b] = n
        if n <= keep or any(page_of(table[b], j, ps, n_pages) is None for j in range(n)):
            continue
        lens[b] = keep
        seen = n if total is None else int(total[b])
        for h in range(Hkv):
            w, o = weight[b, h, :n].astype(np.float64), order[b, h, :n].astype(np.int64)
            held = (o < sink) | (o >= seen - recent)
            rank = np.lexsort((np.arange(n), o, np.where(np.isnan(w), np.inf, w), np.isnan(w), held))
            leaves = np.zeros(n, dtype=bool)
            leaves[rank[:n - keep]] = True
            gaps, behind = np.flatnonzero(leaves[:keep]), keep + np.flatnonzero(~leaves[keep:])
            for to, src in zip(gaps, behind):
                for pages in (k_pages, v_pages):
                    pages[table[b, to // ps], h, to % ps] = pages[table[b, src // ps], h, src % ps]
                weight[b, h, to], order[b, h, to] = weight[b, h, src], order[b, h, src]
    return k_pages, v_pages, weight, order, lens
