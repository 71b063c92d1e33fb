"""Oracle of serving in four bits, in numpy and 64 bits: the quantiser, the
paged cache's plans, the attention over it and the few-row product.  Written
from the definitions in include/fastcoder.h, sharing no code with the GPU path."""
from __future__ import annotations

import numpy as np


def bf16_round(x):
    """float64 -> the nearest bf16 value (ties to even), as float64."""
    f = np.asarray(x, np.float64).astype(np.float32)
    b = f.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16
    return np.where(np.isfinite(f), r.astype(np.uint32).view(np.float32), f).astype(np.float64)


def quantise(x, axis=-1):
    """(numbers as int, scales as float64) of x along axis."""
    x = np.asarray(x, np.float64)
    s = bf16_round(np.abs(x).max(axis, keepdims=True) / 7.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s > 0, np.clip(np.rint(x / s), -7, 7), 0)
    return c.astype(np.int64), np.squeeze(s, axis)


def pack(c):
    """Numbers along the last axis, two to a byte."""
    u = (c + 8).astype(np.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def unpack(b):
    out = np.empty(b.shape[:-1] + (2 * b.shape[-1],), np.int64)
    out[..., 0::2] = (b & 15).astype(np.int64) - 8
    out[..., 1::2] = (b >> 4).astype(np.int64) - 8
    return out


def pages_plan(kv_len, n_new, page, table, free, n_free, rows_cap, path=None, n_per_seq=0):
    """One request after another; returns the dict of fc_kv_pages_plan's outputs
    (table among them) and whether every request was served."""
    table, B = table.copy(), len(kv_len)
    ints = lambda n: np.full(n, -1, np.int32)
    o = dict(cu=np.zeros(B + 1, np.int32), seq=ints(rows_cap), pos=ints(rows_cap), slot=ints(rows_cap),
             src=ints(rows_cap), kv_len=np.maximum(np.asarray(kv_len, np.int32), 0))
    row, asked, taken, all_ok = 0, 0, 0, True
    for b in range(B):
        kv, n = max(int(kv_len[b]), 0), max(int(n_new[b]), 0)
        have, need = -(-kv // page), -(-(kv + n) // page)
        ok = kv_len[b] >= 0 and n_new[b] >= 0 and need <= table.shape[1]
        first = asked
        if ok:
            asked += need - have
        served = ok and row + n <= rows_cap and (need == have or asked <= n_free)
        if served:
            for j in range(have, need):
                table[b, j] = free[n_free - 1 - first - (j - have)]
            taken += need - have
            o["kv_len"][b] = kv + n
        all_ok = all_ok and served
        for j in range(n):
            r = row + j
            if r >= rows_cap:
                break
            p = kv + j
            o["seq"][r], o["pos"][r] = b, p
            o["slot"][r] = table[b, p // page] * page + p % page if served else -1
            if n_per_seq:
                node = j if path is None else (path[b][j] if j < len(path[b]) else -1)
                o["src"][r] = b * n_per_seq + node if 0 <= node < n_per_seq else -1
        row += n
        o["cu"][b + 1] = min(row, rows_cap)
    o["n_free"] = np.array([n_free - taken], np.int32)
    o["table"] = table
    return o, all_ok


def attn(q, k_codes, v_codes, k_scale, v_scale, table, kv_len, k_new, v_new, sees, n_nodes, scale):
    """(out, weight): out [B, n, H, D] and, per element, the mean of |v| under
    the same probabilities (what a relative error of the probabilities scales
    with).  sees [B, n, n] bool."""
    B, n, H, D = q.shape
    G, P = k_codes.shape[1], k_codes.shape[2]
    out, weight = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        L, m = int(kv_len[b]), int(n_nodes[b])
        page, off = table[b, np.arange(L) // P], np.arange(L) % P
        for h in range(H):
            g = h // (H // G)
            k = unpack(k_codes[page, g, off]) * k_scale[page, g, off][:, None]
            v = unpack(v_codes[page, g, off]) * v_scale[page, g, off][:, None]
            new = k_new is not None
            for i in range(m):
                vis = np.flatnonzero(sees[b, i, :m]) if new else []
                kk = np.concatenate([k, k_new[b, g, vis]]) if new else k
                vv = np.concatenate([v, v_new[b, g, vis]]) if new else v
                if not len(kk):
                    continue
                z = kk @ q[b, i, h] * scale
                p = np.exp(z - z.max())
                p /= p.sum()
                out[b, i, h], weight[b, i, h] = p @ vv, p @ np.abs(vv)
    return out, weight


def matvec(x, w, group):
    """(y, size): x times the weights that w [K, N] is held as, and the sum of
    |x| s per element, the size of a rounding unit of its terms."""
    K, N = w.shape
    c, s = quantise(np.asarray(w, np.float64).reshape(K // group, group, N), 1)
    xg = np.asarray(x, np.float64).reshape(len(x), K // group, group)
    y = np.einsum("mtk,tkn,tn->mn", xg, c.astype(np.float64), s)
    return y, np.einsum("mtk,tn->mn", np.abs(xg), s)
