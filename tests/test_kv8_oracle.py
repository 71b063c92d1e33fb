"""The 8-bit oracle against brute force, and the refusals of the calls that
need no GPU (nothing here launches a kernel)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8 as o8


@pytest.fixture(scope="module")
def fc():
    from paper_2502_17139_gb300 import build
    build.build()
    import paper_2502_17139_gb300.fastcoder as m
    return m


def test_e4m3_is_torchs():
    b = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(b).view(torch.float8_e4m3fn)
    assert np.array_equal(o8.decode(b), t.double().numpy(), equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.clip(rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 9, 20000), -448, 448).astype(np.float32)
    x[:256] = np.nan_to_num(o8.decode(b))
    x[256:508] = (o8.VALUES[:126].repeat(2).reshape(-1, 2) + np.diff(o8.VALUES[:127])[:, None] / 2).reshape(-1)  # ties
    assert np.array_equal(o8.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_scale_is_the_smallest_power_that_fits():
    for top in (1e-40, 1.0, 448.0, 448.1, 449.0, 3.0e38, 2.0 ** -30 * 448):
        s = o8.scale_for(top)
        assert 448 * s >= top and (448 * s / 2 < top or s == 2.0 ** -120)
    assert o8.scale_for(0.0) == 2.0 ** -120


def test_write_keeps_what_a_block_holds():
    rng = np.random.default_rng(2)
    cache = [o8.encode(rng.standard_normal((2, 1, 16, 128))) for _ in range(2)] + [np.ones((2, 1, 1), np.float32) for _ in range(2)]
    was = o8.decode(cache[0][1, 0, :4]).copy()
    x = rng.standard_normal((3, 1, 128)) * 1e4
    o8.write(cache, x, x, [20, 21, 22])
    s = float(cache[2][1, 0, 0])
    assert s == o8.scale_for(np.abs(x).max()) and s > 1
    assert np.all(np.abs(o8.decode(cache[0][1, 0, :4]) * s - was) <= np.maximum(2.0 ** -10 * s, 0))  # half the smallest step
    assert np.all(np.abs(o8.decode(cache[0][1, 0, 4:7]) * s - x[:, 0]) <= np.maximum(2.0 ** -4 * np.abs(x[:, 0]), 2.0 ** -10 * s))


def test_evict_keeps_the_heaviest_and_the_newest():
    rng = np.random.default_rng(3)
    L, K = 40, 20
    cache = [o8.encode(rng.standard_normal((3, 1, 16, 128)) * 30) for _ in range(2)] + [(2.0 ** rng.integers(-2, 3, (3, 1, 1))).astype(np.float32) for _ in range(2)]
    table = np.array([[2, 0, 1]], np.int32)
    w, born = rng.random((3, 1, 16)).astype(np.float32), rng.permutation(48).reshape(3, 1, 16).astype(np.int32)
    before = o8.cached(cache, 0, table[0], L, 0)
    i = np.arange(L)
    wl, bl = w[table[0][i // 16], 0, i % 16], born[table[0][i // 16], 0, i % 16]
    outs = [np.zeros_like(w), np.zeros_like(born)]
    frm = o8.evict(cache, table, [L], [K], 5, [w, born], outs, K)
    fresh = bl > bl.max() - 5
    best = set(np.nonzero(fresh)[0]) | set(sorted(np.nonzero(~fresh)[0], key=lambda j: -wl[j])[:K - fresh.sum()])
    now = np.where(frm[0, 0] >= 0, frm[0, 0], np.arange(K))
    assert set(now) == best and np.all((frm[0, 0] < 0) | (frm[0, 0] >= K))
    after = o8.cached(cache, 0, table[0], K, 0)
    top = np.abs(np.concatenate((before[now], before[K:32]))).max()
    assert np.all(np.abs(after - before[now]) <= 2.0 ** -9 * top / 100)
    assert np.array_equal(outs[0][table[0][i[:K] // 16], 0, i[:K] % 16], wl[now])


def test_host_refusals(fc):
    L, nul, f = fc.LIB, None, C.c_float
    good = fc.fc_kv8_cache(256, 256, 256, 256, 10, 64, 8, 128)
    bad = lambda **kw: C.byref(fc.fc_kv8_cache(*[kw.get(n, getattr(good, n)) for n, _ in fc.fc_kv8_cache._fields_]))
    ok = C.byref(good)
    INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3

    def write(cache=ok, k=256, v=256, n_seq=4, n_per=1, st=(0, 1024, 128), src=nul, slot=256, rows=4, pos=nul, weight=nul, born=nul):
        return L.fc_kv8_write(cache, k, v, n_seq, n_per, *st, src, slot, rows, pos, weight, born, nul)

    assert write(rows=0) == 0
    for kw, want in ((dict(cache=nul), INVALID), (dict(cache=bad(D=64)), UNSUPPORTED), (dict(cache=bad(page_size=48)), UNSUPPORTED),
                     (dict(cache=bad(page_size=512)), UNSUPPORTED), (dict(cache=bad(n_pages=0)), INVALID), (dict(cache=bad(k_codes=8)), INVALID),
                     (dict(cache=bad(v_scale=nul)), INVALID), (dict(cache=bad(n_pages=1 << 30)), UNSUPPORTED), (dict(k=nul), INVALID),
                     (dict(v=8), INVALID), (dict(st=(0, 4, 128)), INVALID), (dict(st=(0, -8, 128)), INVALID), (dict(rows=5), INVALID),
                     (dict(rows=-1), INVALID), (dict(slot=nul), INVALID), (dict(weight=256), INVALID), (dict(weight=256, born=256), INVALID),
                     (dict(born=256, pos=256), INVALID)):
        assert write(**kw) == want, kw
    assert L.fc_kv8_read(ok, nul, 0, nul, nul, nul) == 0
    assert L.fc_kv8_read(ok, nul, 1, 256, 256, nul) == INVALID
    assert L.fc_kv8_read(ok, 256, 1, 264, 256, nul) == INVALID

    def attn(q=256, cache=ok, table=256, pages=4, kv=256, k=256, v=256, mask=nul, nodes=nul, B=2, n=1, H=8, scale=0.1, weight=nul, decay=1.0,
             out=256, ws=nul, wsb=0):
        return L.fc_kv8_attn(q, cache, table, pages, kv, k, v, mask, nodes, B, n, H, f(scale), weight, f(decay), out, ws, wsb, nul)

    assert attn(B=0) == 0
    for kw, want in ((dict(q=nul), INVALID), (dict(q=8), INVALID), (dict(table=nul), INVALID), (dict(k=nul), INVALID), (dict(v=nul), INVALID),
                     (dict(n=0), UNSUPPORTED), (dict(n=129), UNSUPPORTED), (dict(H=9), UNSUPPORTED), (dict(H=8 * 17), UNSUPPORTED),
                     (dict(scale=0.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(B=-1), INVALID), (dict(pages=0), INVALID),
                     (dict(mask=4), INVALID), (dict(ws=16, wsb=99), INVALID), (dict(weight=256), WORKSPACE),
                     (dict(weight=256, ws=256, wsb=256), WORKSPACE), (dict(weight=256, n=17), UNSUPPORTED),
                     (dict(weight=256, decay=float("nan")), INVALID), (dict(out=nul), INVALID), (dict(kv=nul), INVALID)):
        assert attn(**kw) == want, kw
    assert L.fc_kv8_attn_workspace(1, 0, 8, 8, 0) == 0 and L.fc_kv8_attn_workspace(1, 17, 8, 8, 64) == 0
    assert L.fc_kv8_attn_workspace(2, 1, 8, 8, 1000) >= 2 * 8 * 1000 * 4

    def evict(cache=ok, table=256, pages=4, kv=256, keep=256, B=2, recent=5, wi=256, bi=256, wo=512, bo=512, frm=256, cap=10, ws=256, wsb=1 << 20):
        return L.fc_kv8_evict(cache, table, pages, kv, keep, B, recent, wi, bi, wo, bo, frm, cap, ws, wsb, nul)

    assert evict(B=0) == 0
    for kw, want in ((dict(cache=nul), INVALID), (dict(table=nul), INVALID), (dict(keep=nul), INVALID), (dict(wo=256), INVALID),
                     (dict(bo=256), INVALID), (dict(frm=nul), INVALID), (dict(recent=-1), INVALID), (dict(recent=(1 << 22) + 1), UNSUPPORTED),
                     (dict(cap=-1), INVALID), (dict(ws=nul), WORKSPACE), (dict(wsb=10), WORKSPACE), (dict(pages=0), INVALID)):
        assert evict(**kw) == want, kw

    def norm(q=256, qs=(0, 1024, 128), k=256, v=256, ks=(0, 1024, 128), wq=256, wk=256, pos=256, B=1, n=4, H=8, Hkv=8, dim=128, base=1e4, eps=1e-6,
             qo=512, ko=512, vo=512):
        return L.fc_qk_norm_rope(q, *qs, k, v, *ks, wq, wk, pos, B, n, H, Hkv, dim, f(base), f(eps), qo, ko, vo, nul)

    assert norm(B=0) == 0 and norm(n=0) == 0
    for kw, want in ((dict(q=nul), INVALID), (dict(q=8), INVALID), (dict(dim=24), INVALID), (dict(dim=528), UNSUPPORTED), (dict(base=0.0), INVALID),
                     (dict(base=float("inf")), INVALID), (dict(eps=-1.0), INVALID), (dict(v=nul), INVALID), (dict(vo=nul), INVALID),
                     (dict(qs=(0, 1028, 128)), INVALID), (dict(ks=(0, -8, 128)), INVALID), (dict(wk=nul), INVALID), (dict(pos=nul), INVALID),
                     (dict(H=0), INVALID)):
        assert norm(**kw) == want, kw


def test_binding_refusals(fc):
    """The checks of the Python calls that come before any pointer is used."""
    x = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fc.fc_qk_norm_rope(x, x, x, x, x, x)  # not on a GPU
    with pytest.raises(TypeError):
        fc.fc_qk_norm_rope(x.float(), x, x, x, x, x)
    with pytest.raises(ValueError):
        fc.Kv8Cache.empty(2, 8, 64, device="cpu")


def test_evict_refuses_more_places_than_it_counts(fc):
    """d_from's places are counted in 32 bits: above 2^30 neither a workspace nor a call."""
    L, nul = fc.LIB, None
    cache = C.byref(fc.fc_kv8_cache(256, 256, 256, 256, 4, 16, 2, 128))
    for cap in ((1 << 30) + 1, (1 << 31) - 16, (1 << 31) - 1):
        assert L.fc_kv8_evict_workspace(1, 2, cap) == 0
        assert L.fc_kv8_evict(cache, 256, 4, 256, 256, 1, 5, 256, 256, 512, 512, 256, cap, 256, 1 << 40, nul) == 2  # FC_ERR_UNSUPPORTED
    assert L.fc_kv8_evict_workspace(1, 2, 1 << 30) > 2 << 32


@pytest.mark.parametrize("field,offset", [("k_codes", 16), ("v_codes", 16), ("k_codes", 8), ("v_codes", 1), ("k_scale", 2), ("v_scale", 2)])
def test_a_cache_off_its_alignment_is_refused(fc, field, offset):
    """Numbers at multiples of 32 bytes, scales of 4: rows are read 32 bytes at a time."""
    at = dict(k_codes=256, v_codes=256, k_scale=256, v_scale=256)
    for shift, want in ((0, 0), (offset, 1)):
        c = dict(at)
        c[field] += shift
        cache = C.byref(fc.fc_kv8_cache(c["k_codes"], c["v_codes"], c["k_scale"], c["v_scale"], 4, 16, 2, 128))
        assert fc.LIB.fc_kv8_read(cache, None, 0, None, None, None) == want


def parts(x, largest):
    """x as the sum of two e4m3 numbers, `largest` put at 2^7 to 2^8."""
    by = 2.0 ** (7 - np.floor(np.log2(largest)))
    near = o8.decode(o8.encode(x * by))
    return (near + o8.decode(o8.encode(x * by - near))) / by


@pytest.mark.parametrize("largest", [1.0, 1.75, 255 / 128, 2.0 ** 60, 2.0 ** -100])
def test_two_parts_hold_what_the_header_says(largest):
    """bf16 values, 8 significant bits, beside the largest of their row: exact down to 2^-9 of it, else to 2^-17 of it."""
    x = np.arange(128, 256)[None] / 128 * 2.0 ** -np.arange(0.0, 30)[:, None] * 2.0 ** np.floor(np.log2(largest))
    x = x[x <= largest]
    err = np.abs(parts(x, largest) - x)
    assert np.all(err[x >= 2.0 ** -9 * largest] == 0)
    assert 0 < err.max() <= 2.0 ** -17 * largest


def test_scores_of_two_parts_are_within_the_oracles_bound():
    """Small numbers beside a large one that meets zeros: all of a score's error is the parts'."""
    rng = np.random.default_rng(4)
    small = lambda *s: rng.integers(128, 256, s) / 128 * 2.0 ** -12.0
    q, k = small(3, 128), rng.standard_normal((40, 128))
    q[0] = 129 / 128 * 2.0 ** -10  # just between two sums of parts, all on one side
    k[0] = np.abs(k[0])
    q[:, 0], k[:, 0] = 1, 0
    k[8:] = small(32, 128)  # the last 32 are new
    k[8::16, 1], q[:, 1] = 1, 0
    k[8:, 0] = 0
    qp = np.stack([parts(r, 1.0) for r in q])
    kp = np.concatenate((k[:8], parts(k[8:], 1.0)))
    sees = np.ones((3, 40), bool)
    bound = lambda keys, new: o8.attend(q, k[keys], k[keys], sees[:, keys], 1.0, new)[3]
    err = np.abs(qp @ kp.T - q @ k.T)
    for keys, new in ((slice(0, 8), 0), (slice(8, 40), 32)):
        assert np.all(err[:, keys] <= bound(keys, new))


def test_more_query_rows_than_are_counted_are_refused(fc):
    """2^30 over all heads; sizes whose product passes 64 bits among them."""
    L, nul, f = fc.LIB, None, C.c_float
    for Hkv, batch, n, H in ((1 << 26, 1 << 30, 16, 1 << 30), (1 << 26, (1 << 31) - 1, 128, 1 << 30), (8, 1 << 27, 1, 9 * 8), (8, (1 << 27) + 1, 1, 8),
                             (1 << 26, 1, 16, 1 << 30)):
        cache = C.byref(fc.fc_kv8_cache(256, 256, 256, 256, 1, 16, Hkv, 128))
        assert L.fc_kv8_attn(256, cache, 256, 4, 256, nul, nul, nul, nul, batch, n, H, f(0.1), nul, f(1.0), 256, nul, 0, nul) == 2  # FC_ERR_UNSUPPORTED
        assert L.fc_kv8_attn_workspace(batch, n, H, Hkv, 0) == 0
    assert L.fc_kv8_attn_workspace(1 << 26, 1, 16, 8, 0) > 0 and L.fc_kv8_attn_workspace(1, 1, 8, 8, 1 << 31) == 0
