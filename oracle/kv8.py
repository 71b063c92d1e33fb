"""Oracle of serving from the 8-bit cache, in numpy and 64 bits: the e4m3
quantiser with a power-of-two scale for 16 tokens, cache writes, attention and
the weights it gives, eviction, and the norm and rotation of queries and keys.
Written from the definitions in include/fastcoder.h, sharing no code with the
GPU path."""
from __future__ import annotations

import numpy as np

BLOCK = 16

# what the 256 e4m3 bytes stand for
_E, _M = (np.arange(256) >> 3) & 15, np.arange(256) & 7
VALUES = np.where(_E > 0, (8 + _M) * 2.0 ** (_E - 10), _M * 2.0 ** -9) * np.where(np.arange(256) < 128, 1.0, -1.0)
VALUES[[0x7F, 0xFF]] = np.nan
_POS = VALUES[:127]


def encode(x):
    """The bytes of the nearest e4m3 numbers of |x| <= 448 (ties to the even byte)."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    i = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo, hi = a - _POS[i - 1], _POS[i] - a
    up = (hi < lo) | ((hi == lo) & (i % 2 == 0))
    b = np.where(up, i, i - 1).astype(np.uint8)
    return np.where(np.signbit(x), b | 0x80, b).astype(np.uint8)


def decode(b):
    return VALUES[b]


def scale_for(top):
    e = -120
    while 448.0 * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def place(slot, page):
    return slot // page, slot % page


def write(cache, k, v, slot, src=None, track=None, pos=None):
    """cache: [k_codes, v_codes, k_scale, v_scale] as numpy (changed in place);
    k, v [rows, H, D] float64, slot [rows]; track: [weight, born]."""
    page = cache[0].shape[2]
    rows = {}
    for r, s in enumerate(slot):
        at = r if src is None else int(src[r])
        if s >= 0 and 0 <= at < len(k) and s < cache[0].shape[0] * page:
            rows.setdefault(int(s) // BLOCK, []).append((int(s) % BLOCK, at, r))
    for block, new in rows.items():
        p, t = block * BLOCK // page, block * BLOCK % page // BLOCK
        first = min(o for o, _, _ in new)
        for x, codes, scales in ((k, cache[0], cache[2]), (v, cache[1], cache[3])):
            for h in range(codes.shape[1]):
                vals = np.stack([x[at, h] for _, at, _ in new])
                old = float(scales[p, h, t])
                if not np.isfinite(vals).all() or (first > 0 and np.isnan(old)):
                    scales[p, h, t] = np.nan
                    for o, _, _ in new:
                        codes[p, h, t * BLOCK + o] = 0
                    continue
                s = scale_for(np.abs(vals).max())
                if first > 0:
                    s = max(s, old)
                    held = codes[p, h, t * BLOCK:t * BLOCK + first]
                    if s > old:
                        codes[p, h, t * BLOCK:t * BLOCK + first] = encode(decode(held) * old / s)
                scales[p, h, t] = s
                for (o, _, _), row in zip(new, vals):
                    codes[p, h, t * BLOCK + o] = encode(row / s)
        if track is not None:
            for o, _, r in new:
                track[0][p, :, t * BLOCK + o] = 0
                track[1][p, :, t * BLOCK + o] = pos[r]


def cached(cache, which, table, n, h):
    """The values [n, D] of one request's first n tokens for head h."""
    page = cache[0].shape[2]
    i = np.arange(n)
    p, o = table[i // page], i % page
    return decode(cache[which][p, h, o]) * cache[2 + which][p, h, o // BLOCK].astype(np.float64)[:, None]


def attend(q, k, v, sees, scale, new=0):
    """q [n, D], k, v [L, D], sees [n, L]: (out, weights [n, L], mean |v|, e): e
    bounds a score's error where sums of 128 products round to fp32 and queries,
    and the last `new` keys by 16, are sums of two e4m3 numbers: 2^-17 of the
    largest magnitude of their row, or 16 rows.  (That one is put at 2^7 to 2^8.
    The nearest e4m3 number of x leaves at most four significant bits, of x's
    last place or more; what is below 2^-9, e4m3's smallest step, is rounded to
    it, by 2^-10 at most: 2^-17 of 2^7.)"""
    z = np.where(sees, (q @ k.T) * scale, -np.inf)
    top = z.max(1, keepdims=True, initial=-np.inf)
    w = np.where(sees, np.exp(z - np.where(np.isfinite(top), top, 0)), 0)
    total = w.sum(1, keepdims=True)
    w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    e = scale * (2.0 ** -16 * (np.abs(q) @ np.abs(k).T) + 2.0 ** -17 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1)[None])
    for j in range(len(k) - new, len(k), BLOCK):
        e[:, j:j + BLOCK] += scale * 2.0 ** -17 * np.abs(k[j:j + BLOCK]).max() * np.abs(q).sum(1)[:, None]
    return w @ v, w, w @ np.abs(v), np.where(sees, e, 0).max(1, keepdims=True, initial=0.0)


def evict(cache, table, kv_len, keep, recent, track, track_out, cap):
    """In place; returns from [B, H, cap]."""
    page, H = cache[0].shape[2], cache[0].shape[1]
    B = len(kv_len)
    frm = np.full((B, H, cap), -1, np.int32)
    for b in range(B):
        L, K = int(kv_len[b]), int(keep[b])
        i = np.arange(L)
        p, o = table[b][i // page], i % page
        for h in range(H):
            w, born = track[0][p, h, o].astype(np.float64), track[1][p, h, o].astype(np.int64)
            if K < L:
                fresh = born > born.max() - recent
                rank = sorted(range(L), key=lambda j: (not fresh[j], -born[j] if fresh[j] else 0, 0 if fresh[j] or np.isnan(w[j]) else 1,
                                                      0 if fresh[j] or np.isnan(w[j]) else -w[j], j))
                stay = np.zeros(L, bool)
                stay[rank[:K]] = True
                holes, sources = np.nonzero(~stay[:K])[0], K + np.nonzero(stay[K:])[0]
            else:
                holes = sources = np.zeros(0, int)
            now = i.copy()
            now[holes] = sources
            frm[b, h, holes] = sources
            n = min(K, L)
            track_out[0][p[:n], h, o[:n]] = track[0][p[now[:n]], h, o[now[:n]]]
            track_out[1][p[:n], h, o[:n]] = track[1][p[now[:n]], h, o[now[:n]]]
            for codes, scales in ((cache[0], cache[2]), (cache[1], cache[3])):
                was, by = codes[p, h, o].copy(), scales[p, h, o // BLOCK].astype(np.float64)
                for t in sorted(set((holes // BLOCK).tolist())):
                    r = np.arange(t * BLOCK, min(L, (t + 1) * BLOCK))
                    val = decode(was[now[r]]) * by[now[r]][:, None]
                    s = np.nan if np.isnan(by[now[r]]).any() else scale_for(np.abs(val).max())
                    codes[p[r], h, o[r]] = was[now[r]] if np.isnan(s) else encode(val / s)
                    scales[p[r[0]], h, o[r[0]] // BLOCK] = s
    return frm


def norm_rope(x, w, pos, base, eps):
    """x [B, n, heads, D], pos [B, n] -> (y, its two terms' magnitude)."""
    D = x.shape[-1]
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    a = pos[:, :, None, None] * base ** (-2.0 * np.arange(D // 2) / D)
    a = np.where(pos[:, :, None, None] < 0, 0, a)
    c, s = np.cos(a), np.sin(a)
    lo, hi = y[..., :D // 2], y[..., D // 2:]
    mag = np.concatenate([np.abs(lo) + np.abs(hi)] * 2, -1)
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1), mag
