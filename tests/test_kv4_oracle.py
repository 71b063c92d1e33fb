"""The four-bit oracle against brute force, and the refusals of the calls that
need no GPU (nothing here launches a kernel)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv4 as o4


@pytest.fixture(scope="module")
def fc():
    from paper_2502_17139_gb300 import build
    build.build()
    import paper_2502_17139_gb300.fastcoder as m
    return m


def test_bf16_round_is_torchs():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal(5000) * 10.0 ** rng.integers(-30, 30, 5000)).astype(np.float32)
    assert np.array_equal(o4.bf16_round(x), torch.from_numpy(x).bfloat16().double().numpy())


def test_quantise_picks_the_nearest_number():
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((50, 128)).astype(np.float32)).bfloat16().double().numpy()
    x[0] = 0
    c, s = o4.quantise(x)
    assert c.min() >= -7 and c.max() <= 7 and np.all(c[0] == 0) and s[0] == 0
    for r in range(1, 50):
        err = np.abs(x[r][:, None] - np.arange(-7, 8)[None, :] * s[r])
        assert np.allclose(np.abs(x[r] - c[r] * s[r]), err.min(1), rtol=0, atol=0)
    assert np.array_equal(o4.unpack(o4.pack(c)), c)


def test_plan_allots_every_page_once():
    rng = np.random.default_rng(3)
    B, page, most = 20, 16, 12
    kv, new = rng.integers(0, 60, B).astype(np.int32), rng.integers(0, 60, B).astype(np.int32)
    order = rng.permutation(400).astype(np.int32)
    table = np.full((B, most), -1, np.int32)
    at = 0
    for b in range(B):
        n = -(-int(kv[b]) // page)
        table[b, :n] = order[at:at + n]
        at += n
    free = order[at:]
    out, ok = o4.pages_plan(kv, new, page, table, free, len(free), int(new.sum()))
    assert ok and np.array_equal(out["kv_len"], kv + new)
    used = out["table"][out["table"] >= 0]
    assert len(set(used.tolist())) == len(used)
    assert out["n_free"][0] == len(free) - (len(used) - at)
    assert len(set(out["slot"].tolist())) == len(out["slot"])  # no two tokens share a place


def test_host_refusals(fc):
    L, nul, f = fc.LIB, None, C.c_float
    good = fc.fc_kv4_cache(256, 256, 256, 256, 10, 64, 8, 128)
    ref = C.byref(good)
    for bad, st in ((fc.fc_kv4_cache(256, 256, 256, 256, 0, 64, 8, 128), 1), (fc.fc_kv4_cache(256, 256, 256, 256, 10, 64, 0, 128), 1),
                    (fc.fc_kv4_cache(256, 256, 256, 256, 10, 48, 8, 128), 2), (fc.fc_kv4_cache(256, 256, 256, 256, 10, 512, 8, 128), 2),
                    (fc.fc_kv4_cache(256, 256, 256, 256, 10, 64, 8, 64), 2), (fc.fc_kv4_cache(256, 256, 256, 256, 1 << 26, 64, 8, 128), 2),
                    (fc.fc_kv4_cache(256, 264, 256, 256, 10, 64, 8, 128), 1), (fc.fc_kv4_cache(256, 256, None, 256, 10, 64, 8, 128), 1)):
        assert L.fc_kv4_read(C.byref(bad), 16, 4, 16, 16, nul) == st
        assert L.fc_kv4_write(C.byref(bad), 16, 16, 1, 4, 0, 1024, 128, nul, 16, 4, nul) == st
        assert L.fc_kv4_attn(16, C.byref(bad), 16, 4, 16, nul, nul, nul, nul, 1, 1, 8, f(0.1), 16, nul, 0, nul) == st
    assert L.fc_kv4_read(None, 16, 4, 16, 16, nul) == 1
    # read and write: no rows is a no-op, null and odd pointers, strides that break the 16-byte loads, too few rows
    assert L.fc_kv4_read(ref, nul, 0, nul, nul, nul) == 0
    assert L.fc_kv4_read(ref, 16, 4, 18, 16, nul) == 1
    assert L.fc_kv4_write(ref, nul, nul, 1, 4, 0, 1024, 128, nul, nul, 0, nul) == 0
    assert L.fc_kv4_write(ref, 16, 16, 1, 4, 0, 1027, 128, nul, 16, 4, nul) == 1
    assert L.fc_kv4_write(ref, 24, 16, 1, 4, 0, 1024, 128, nul, 16, 4, nul) == 1
    assert L.fc_kv4_write(ref, 16, 16, 1, 4, 0, 1024, 128, nul, 16, 5, nul) == 1
    assert L.fc_kv4_write(ref, 16, 16, 1, 0, 0, 1024, 128, nul, 16, 4, nul) == 1
    # attention: shapes, scale, half a pair of new keys, a misaligned workspace; an empty batch is a no-op
    att = lambda *a: L.fc_kv4_attn(16, ref, 16, 4, 16, *a, nul)
    assert att(nul, nul, nul, nul, 1, 129, 8, f(0.1), 16, nul, 0) == 2
    assert att(nul, nul, nul, nul, 1, 0, 8, f(0.1), 16, nul, 0) == 2
    assert att(nul, nul, nul, nul, 1, 1, 12, f(0.1), 16, nul, 0) == 2
    assert att(nul, nul, nul, nul, 1, 1, 136, f(0.1), 16, nul, 0) == 2
    assert att(nul, nul, nul, nul, 1, 1, 8, f(0.0), 16, nul, 0) == 1
    assert att(nul, nul, nul, nul, 1, 1, 8, f(float("inf")), 16, nul, 0) == 1
    assert att(16, nul, nul, nul, 1, 1, 8, f(0.1), 16, nul, 0) == 1
    assert att(nul, nul, nul, nul, 1, 1, 8, f(0.1), 16, 128, 4096) == 1
    assert att(nul, nul, nul, nul, 1, 1, 8, f(0.1), 24, nul, 0) == 1
    assert att(nul, nul, nul, nul, 0, 1, 8, f(0.1), 16, nul, 0) == 0
    assert L.fc_kv4_attn_workspace(1, 129, 8, 8) == 0 and L.fc_kv4_attn_workspace(1, 1, 8, 8) > 0
    # plan and release: page sizes, aliased lengths and counts, missing outputs, a src without its row length
    plan = lambda page=64, table=16, mp=4, free=32, npg=10, nf=48, path=nul, pc=0, nps=0, rows=8, kvo=64, nfo=80, src=nul: \
        L.fc_kv_pages_plan(16, 16, 2, page, table, mp, free, npg, nf, path, pc, nps, rows, 96, 112, 128, 144, src, kvo, nfo, nul)
    assert plan(page=65) == 2 and plan(page=8) == 2
    assert plan(kvo=16) == 1 and plan(nfo=48) == 1 and plan(table=nul) == 1 and plan(mp=0) == 1 and plan(npg=0) == 1
    assert plan(src=160) == 1 and plan(src=160, nps=4, path=176, pc=0) == 1 and plan(rows=-1) == 1
    assert L.fc_kv_pages_plan(*[nul] * 2, 0, 64, nul, 4, nul, 10, nul, nul, 0, 0, 0, *[nul] * 8) == 0
    rel = lambda page=64, kvo=64, nfo=80, b=2: L.fc_kv_pages_release(16, 32, b, page, 16, 4, 32, 10, 48, kvo, nfo, nul)
    assert rel(page=100) == 2 and rel(kvo=16) == 1 and rel(nfo=48) == 1 and rel(b=-1) == 1 and rel(b=0) == 0
    # weights: k not a multiple of 64 or of the group, odd groups, too many rows
    assert L.fc_w4_codes_bytes(128, 33) == 3 * 2 * 512 and L.fc_w4_codes_bytes(100, 33) == 0
    assert L.fc_w4_pack(16, 96, 64, 32, 16, 16, nul) == 2 and L.fc_w4_pack(16, 192, 64, 128, 16, 16, nul) == 2
    assert L.fc_w4_pack(16, 128, 64, 48, 16, 16, nul) == 2 and L.fc_w4_pack(16, 128, 64, 64, 24, 16, nul) == 1
    assert L.fc_w4_matvec(16, 16, 16, 17, 128, 64, 64, 16, nul) == 2
    assert L.fc_w4_matvec(16, 16, 16, -1, 128, 64, 64, 16, nul) == 1
    assert L.fc_w4_matvec(24, 16, 16, 4, 128, 64, 64, 16, nul) == 1
    assert L.fc_w4_matvec(nul, nul, nul, 0, 128, 64, 64, nul, nul) == 0


def test_host_refuses_pointers_that_a_wide_load_would_fault_on(fc):
    L, nul = fc.LIB, None
    ref = C.byref(fc.fc_kv4_cache(256, 256, 256, 256, 10, 64, 8, 128))
    for mask in (12, 20):  # masks are read as 64-bit words
        assert L.fc_kv4_attn(16, ref, 16, 4, 16, 16, 16, mask, nul, 1, 1, 8, C.c_float(0.1), 16, nul, 0, nul) == 1
    for scale in (18, 20, 24):  # scales are fetched two and more at a time
        assert L.fc_w4_matvec(16, 16, scale, 4, 128, 64, 64, 16, nul) == 1
    assert L.fc_w4_matvec(16, 16, 16, 4, 128, 64, 64, 17, nul) == 1


def test_binding_refusals(fc):
    t = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt)
    with pytest.raises((TypeError, ValueError)):
        fc.KvPages(64, t(2, 4), t(10))  # not on the GPU
    with pytest.raises(TypeError):
        fc.fc_w4_pack(t(128, 64, dt=torch.float32))
    with pytest.raises(TypeError):
        fc.fc_kv4_attn(t(1, 1, 8, 128, dt=torch.float16), None, None, None)
