"""Serving in four bits on the GPU against the 64-bit oracle (oracle/kv4.py).

Whole numbers (plans, numbers, scales) are equal.  bf16 has 8 significant
bits, so a rounding to it moves a value by at most 2^-8 of itself.  Floating
tolerances, per element:
* attention: the output's rounding, 2^-8 |out|; each p's rounding, 2^-8 of A =
  the mean of |v| under the same probabilities; and a score's fp32 error
  (numbers may enter the product with a surplus of up to 136, sums of 128
  terms: below 2^-22 * 136 * sum|q| * s * scale < 2^-12 here), which changes p
  by as much again relative to the row sum: 2^-10 A.
* product: the fp32 sums' error e, whose terms carry a surplus of 136, is
  below 2^-20 * 136 * sum |x| s; the output lies between the roundings of
  y - e and y + e.
"""
import numpy as np
import pytest
import torch

from oracle import kv4 as o4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fc():
    import paper_2502_17139_gb300.fastcoder as m
    assert m.fc_get_error() == "FC_OK"
    return m


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf(rng, *shape, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).bfloat16()


def num(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------ pages
def pool(rng, kv, new, page, spare):
    """Tables that hold kv, and a free list of what new needs plus spare pages."""
    held = [-(-int(max(k, 0)) // page) for k in kv]
    need = [-(-int(max(k, 0) + max(n, 0)) // page) for k, n in zip(kv, new)]
    n_free = max(0, sum(need) - sum(held) + spare)
    n_pages = sum(held) + n_free + 3
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(kv), max(need) + 1), -1, np.int32)
    at = n_free
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    free = np.full(n_pages, -1, np.int32)
    free[:n_free] = order[:n_free]
    return table, free, n_free


def check_plan(fc, kv, new, page, table, free, n_free, rows_cap, path=None, n_per_seq=0, status="FC_OK"):
    ref, _ = o4.pages_plan(kv, new, page, table, free, n_free, rows_cap, path, n_per_seq)
    pages = fc.KvPages(page, dev(table), dev(free))
    out = fc.fc_kv_pages_plan(pages, dev(kv), dev(new), dev(np.array([n_free], np.int32)), rows_cap=rows_cap,
                              path=None if path is None else dev(path), n_per_seq=n_per_seq)
    again = fc.fc_kv_pages_plan(pages, dev(kv), dev(new), dev(np.array([n_free], np.int32)), rows_cap=rows_cap,
                                path=None if path is None else dev(path), n_per_seq=n_per_seq)
    assert fc.fc_get_error() == status
    for k in out:
        assert np.array_equal(out[k].cpu().numpy(), ref[k]), k
        assert torch.equal(out[k], again[k])
    assert np.array_equal(pages.table.cpu().numpy(), ref["table"])
    return pages, out


@pytest.mark.parametrize("B,most_kv,most_new,page", [(1, 0, 1, 16), (1, 5000, 700, 64), (32, 16384, 1, 64), (33, 300, 40, 16),
                                                     (512, 200, 9, 128), (513, 100, 90, 32), (1500, 70, 5, 256),
                                                     (2, 100, 30000, 16)])
def test_plan(fc, B, most_kv, most_new, page):
    rng = np.random.default_rng(B + page)
    kv = rng.integers(0, most_kv + 1, B).astype(np.int32)
    new = rng.integers(0, most_new + 1, B).astype(np.int32)
    new[0] = most_new
    table, free, n_free = pool(rng, kv, new, page, 2)
    check_plan(fc, kv, new, page, table, free, n_free, int(new.sum()) + (B % 3) * 7)


def test_plan_paths_name_the_source_rows(fc):
    rng = np.random.default_rng(7)
    B, cap = 40, 12
    kv, new = rng.integers(0, 90, B).astype(np.int32), rng.integers(1, 11, B).astype(np.int32)
    path = np.full((B, cap), -1, np.int32)
    for b in range(B):
        path[b, :new[b]] = np.sort(rng.choice(64, new[b], replace=False))
    path[3, 0] = 64  # outside its tree
    table, free, n_free = pool(rng, kv, new, 16, 0)
    check_plan(fc, kv, new, 16, table, free, n_free, int(new.sum()), path, 64)
    check_plan(fc, kv, new, 16, table, free, n_free, int(new.sum()), None, 8)


@pytest.mark.parametrize("case", ["pool", "table", "rows", "negative"])
def test_plan_refuses_what_does_not_fit(fc, case):
    rng = np.random.default_rng(11)
    B, page = 700, 16
    kv, new = rng.integers(0, 60, B).astype(np.int32), rng.integers(0, 60, B).astype(np.int32)
    new[600:640] = 0
    if case == "negative":
        kv[5], new[650] = -3, -1
    table, free, n_free = pool(rng, kv, new, page, -40 if case == "pool" else 0)
    rows = int(np.maximum(new, 0).sum())
    if case == "table":
        table = np.ascontiguousarray(table[:, :6])
    if case == "rows":
        rows -= 100
    check_plan(fc, kv, new, page, table, free, n_free, rows,
               status="FC_ERR_INVALID_ARG" if case == "negative" else "FC_ERR_CAPACITY")


def test_release_gives_the_pages_back_in_order(fc):
    rng = np.random.default_rng(13)
    B, page = 900, 16
    kv, new = rng.integers(0, 80, B).astype(np.int32), np.zeros(B, np.int32)
    table, free, n_free = pool(rng, kv, new, page, 5)
    keep = np.where(rng.random(B) < 0.4, rng.integers(0, 90, B), kv).astype(np.int32)
    want, at = free.copy(), n_free
    for b in range(B):
        k = min(keep[b], kv[b])
        for j in range(-(-int(k) // page), -(-int(kv[b]) // page)):
            want[at] = table[b, j]
            at += 1
    pages = fc.KvPages(page, dev(table), dev(free))
    kv_out, free_out = fc.fc_kv_pages_release(pages, dev(kv), dev(keep), dev(np.array([n_free], np.int32)))
    assert fc.fc_get_error() == "FC_OK"
    assert np.array_equal(pages.free.cpu().numpy(), want) and free_out.item() == at
    assert np.array_equal(kv_out.cpu().numpy(), np.minimum(keep, kv))
    # a free count that leaves no room: nothing is written past the list
    full = dev(np.array([len(free) - 4], np.int32))
    pages = fc.KvPages(page, dev(table), dev(free))
    _, free_out = fc.fc_kv_pages_release(pages, dev(kv), dev(np.zeros(B, np.int32)), full)
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG" and len(free) - 4 <= free_out.item() <= len(free)


@pytest.mark.parametrize("rows_cap", [0, 3])
def test_an_empty_plan_and_an_empty_release_carry_the_free_count_over(fc, rows_cap):
    """No requests: the outputs say so, whatever they held."""
    i32 = dict(dtype=torch.int32, device="cuda")
    none, n_free = torch.empty(0, **i32), torch.full((1,), 7, **i32)
    pages = fc.KvPages(16, torch.empty((0, 4), **i32), torch.arange(9, **i32))
    out = fc.kv_pages_outputs(0, rows_cap, "cuda", src=True)
    for t in out.values():
        t.fill_(99)
    fc.fc_kv_pages_plan(pages, none, none, n_free, n_per_seq=4, out=out)
    assert out["n_free"].tolist() == [7] and out["cu"].tolist() == [0]
    for k in ("seq", "pos", "slot", "src"):
        assert out[k].tolist() == [-1] * rows_cap
    kept = (torch.empty(0, **i32), torch.full((1,), 99, **i32))
    kv, free = fc.fc_kv_pages_release(pages, none, none, n_free, out=kept)
    assert kv.numel() == 0 and free.tolist() == [7] and n_free.tolist() == [7]
    assert fc.fc_get_error() == "FC_OK"


# ------------------------------------------------------------- write, read
def rows_of(rng, kind, R, H):
    """(k, v) tensors of three layouts that hold the same kind of rows."""
    if kind == "fused":
        qkv = bf(rng, R, (2 * H + 2 * H) * 128).cuda()
        return qkv[:, 2 * H * 128:3 * H * 128].view(R, H, 128), qkv[:, 3 * H * 128:].view(R, H, 128)
    if kind == "heads":  # [B, Hkv, n, D], transposed in place
        n = -(-R // 3)
        k, v = bf(rng, 3, H, n, 128).cuda(), bf(rng, 3, H, n, 128).cuda()
        return k.transpose(1, 2), v.transpose(1, 2)
    return bf(rng, R, H, 128).cuda(), bf(rng, R, H, 128).cuda()


@pytest.mark.parametrize("kind", ["dense", "fused", "heads"])
@pytest.mark.parametrize("R,H,page", [(1, 1, 16), (7, 3, 16), (33, 8, 64), (300, 2, 256)])
def test_write_and_read(fc, kind, R, H, page):
    rng = np.random.default_rng(R * 7 + H)
    k, v = rows_of(rng, kind, R, H)
    k, v = k.clone(memory_format=torch.preserve_format) if kind == "dense" else k, v
    flat = lambda t: num(t.reshape(-1, H, 128))
    n_pages = -(-R // page) + 2
    slot = rng.permutation(n_pages * page)[:R].astype(np.int32)
    src = rng.permutation(flat(k).shape[0])[:R].astype(np.int32)
    slot[R // 2] = -1 if R > 2 else slot[R // 2]
    cache = fc.Kv4Cache.empty(n_pages, H, page)
    fc.fc_kv4_write(cache, k, v, dev(slot), src=dev(src))
    rk, rv = fc.fc_kv4_read(cache, dev(slot))
    assert fc.fc_get_error() == "FC_OK"
    for x, codes, scale, back in ((k, cache.k_codes, cache.k_scale, rk), (v, cache.v_codes, cache.v_scale, rv)):
        c, s = o4.quantise(flat(x)[src])
        want_c = np.zeros((n_pages, H, page, 64), np.uint8)
        want_s = np.zeros((n_pages, H, page))
        live = slot >= 0
        want_c[slot[live] // page, :, slot[live] % page] = o4.pack(c)[live]
        want_s[slot[live] // page, :, slot[live] % page] = s[live]
        assert np.array_equal(codes.cpu().numpy(), want_c)  # and nothing else is written
        assert np.array_equal(num(scale), want_s)
        want = np.where(live[:, None, None], o4.bf16_round(c * s[..., None]), 0)
        assert np.array_equal(num(back), want)


def test_quantiser_at_ties_and_extremes(fc):
    """Every bf16 mantissa against every scale mantissa: exact ties, values
    just beside them, tiny and huge rows, zeros, NaN and infinities."""
    rng = np.random.default_rng(17)
    m = np.arange(128, 256)
    rows = []
    for top in m:  # the row's maximum; the others sweep mantissas and exponents
        for e in (-1, -2, -3, -4):
            r = np.zeros(128)
            r[:128] = m * 2.0 ** e * rng.choice([-1, 1], 128)
            r = np.where(np.abs(r) > top, 0, r)
            r[rng.integers(128)] = top
            rows.append(r)
    rows = np.array(rows)
    rows = np.concatenate([rows, rows[:40] * 2.0 ** 118, rows[40:80] * 2.0 ** -110, rows[80:120] * 2.0 ** -130,
                           np.zeros((2, 128)), np.full((1, 128), 2.0 ** -133), rng.standard_normal((5, 128))])
    x = torch.from_numpy(rows.astype(np.float32)).bfloat16()[:, None].cuda()
    R = len(rows)
    cache = fc.Kv4Cache.empty(-(-R // 16), 1, 16)
    slot = torch.arange(R, dtype=torch.int32).cuda()
    fc.fc_kv4_write(cache, x, -x, slot)
    c, s = o4.quantise(num(x)[:, 0])
    got = o4.unpack(cache.k_codes.cpu().numpy()).reshape(-1, 128)[:R]
    assert np.array_equal(num(cache.k_scale).reshape(-1)[:R], s)
    assert np.array_equal(got, c)
    assert np.array_equal(o4.unpack(cache.v_codes.cpu().numpy()).reshape(-1, 128)[:R], -c)
    x[3, 0, 5], x[4, 0, 6], x[5, 0, 7] = float("nan"), float("inf"), -float("inf")
    fc.fc_kv4_write(cache, x, x, slot)
    rk, rv = fc.fc_kv4_read(cache, slot[:8])
    for t in (rk, rv):
        assert torch.isnan(t[3:6]).all() and torch.isfinite(t[:3]).all() and torch.isfinite(t[6:]).all()
    assert fc.fc_get_error() == "FC_OK"


def test_write_and_read_leave_out_what_is_out_of_range(fc):
    rng = np.random.default_rng(19)
    k = bf(rng, 6, 2, 128).cuda()
    cache = fc.Kv4Cache.empty(2, 2, 16)
    fc.fc_kv4_write(cache, k, k, dev(np.array([0, 32, 5], np.int32)))  # two pages of 16: slot 32 is past the pool
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    fc.fc_kv4_write(cache, k, k, dev(np.array([6, 7], np.int32)), src=dev(np.array([6, -1], np.int32)))
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    c = cache.k_codes.cpu().numpy().reshape(2, 2, 16, 64)
    assert c[0, :, [0, 5]].any() and not c[0, :, 6:].any() and not c[1].any()
    out, _ = fc.fc_kv4_read(cache, dev(np.array([0, 1 << 20], np.int32)))
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG" and not out[1].any()


def test_write_binding_checks(fc):
    cache = fc.Kv4Cache.empty(2, 2, 16)
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    slot = torch.arange(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        fc.fc_kv4_write(cache, k, k[:2], slot)
    with pytest.raises(ValueError):
        fc.fc_kv4_write(cache, k[:2], k[:2], slot)
    with pytest.raises(ValueError):
        fc.fc_kv4_write(cache, k[:, :1], k[:, :1], slot)
    with pytest.raises(TypeError):
        fc.fc_kv4_write(cache, k.float(), k.float(), slot)
    with pytest.raises(TypeError):
        fc.fc_kv4_write(cache, k, k, slot.long())


def test_write_looks_at_no_stride_of_a_dimension_of_one(fc):
    """One row, or one head: whatever stride its dimension has is never used."""
    rng = np.random.default_rng(23)
    flat = bf(rng, 40 * 128).cuda()
    one = lambda at, s: torch.as_strided(flat, (3, 1, 128), (256, s, 1), at)
    row = lambda at, s: torch.as_strided(flat, (1, 2, 128), (s, 128, 1), at)
    for k, v, H in ((row(0, 5), row(512, 768), 2), (one(0, 3), one(128, 77), 1), (one(0, 128)[None], one(128, 5)[None], 1)):
        rows = k.numel() // (128 * H)
        cache, slot = fc.Kv4Cache.empty(1, H, 16), torch.arange(rows, dtype=torch.int32, device="cuda")
        fc.fc_kv4_write(cache, k, v, slot)
        for x, codes, scale in ((k, cache.k_codes, cache.k_scale), (v, cache.v_codes, cache.v_scale)):
            c, s = o4.quantise(num(x).reshape(rows, H, 128))
            assert np.array_equal(codes.cpu().numpy()[0, :, :rows].swapaxes(0, 1), o4.pack(c))
            assert np.array_equal(num(scale)[0, :, :rows].T, s)
    assert fc.fc_get_error() == "FC_OK"


# --------------------------------------------------------------- attention
def random_cache(rng, n_pages, G, page):
    codes = [np.clip(np.rint(rng.standard_normal((n_pages, G, page, 128)) * 2.6), -7, 7).astype(np.int64) for _ in range(2)]
    scales = [o4.bf16_round(0.3 + 0.2 * rng.random((n_pages, G, page))) for _ in range(2)]
    return codes, scales


def tree_sees(rng, B, n):
    """Ancestors and itself, random parents."""
    s = np.zeros((B, n, n), bool)
    for b in range(B):
        for i in range(n):
            if i:
                s[b, i] = s[b, rng.integers(max(0, i - 6), i)]
            s[b, i, i] = True
    return s


def mask_words(sees):
    B, n, _ = sees.shape
    w = np.zeros((B, n, (n + 63) // 64), np.uint64)
    for j in range(n):
        w[..., j // 64] |= sees[..., j].astype(np.uint64) << np.uint64(j % 64)
    return w.view(np.int64)


def attn_case(seed, B, n, H, G, lens, page, nodes=None, kind="tree", scale=None, spare=1, stale=True, qscale=1.0):
    rng = np.random.default_rng(seed)
    held = [-(-L // page) for L in lens]
    n_pages, most = sum(held) + 1, max(held) + spare
    codes, scales = random_cache(rng, n_pages, G, page)
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, max(most, 1)), 0, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
        if stale and lens[b] % page:  # what stands past a request's end
            for s in scales:
                s[table[b, h - 1], :, lens[b] % page:] = np.nan
    sees = tree_sees(rng, B, n) if kind == "tree" else np.broadcast_to(np.tril(np.ones((n, n), bool)), (B, n, n)).copy()
    return dict(q=bf(rng, B, n, H, 128, scale=qscale), codes=codes, scales=scales, table=table, lens=np.asarray(lens, np.int32),
                k_new=bf(rng, B, G, n, 128), v_new=bf(rng, B, G, n, 128), sees=sees, kind=kind,
                nodes=np.asarray(nodes if nodes is not None else [n] * B, np.int32), scale=128 ** -0.5 if scale is None else scale)


def gpu_cache(fc, c):
    return fc.Kv4Cache(*(dev(o4.pack(x)) for x in c["codes"]),
                       *(torch.from_numpy(s).to(torch.bfloat16).cuda() for s in c["scales"]))


def run_attn(fc, c, new=True, ws=True, nodes=True, cache=None):
    B, n, H, _ = c["q"].shape
    cache = cache or gpu_cache(fc, c)
    return fc.fc_kv4_attn(c["q"].cuda(), cache, dev(c["table"]), dev(c["lens"]), c["k_new"].cuda() if new else None,
                          c["v_new"].cuda() if new else None, dev(mask_words(c["sees"])) if c["kind"] == "tree" else None,
                          dev(c["nodes"]) if nodes else None, scale=c["scale"],
                          workspace=fc.kv4_attn_workspace(B, n, H, cache.Hkv, "cuda") if ws else None)


def check_attn(fc, c, new=True, **kw):
    out = run_attn(fc, c, new=new, **kw)
    assert fc.fc_get_error() == "FC_OK"
    kn, vn = (num(c["k_new"]), num(c["v_new"])) if new else (None, None)
    ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"], kn, vn,
                        c["sees"], c["nodes"], c["scale"])
    got = num(out)
    assert np.isfinite(got).all()
    bad = np.abs(got - ref) - 2.0 ** -8 * np.abs(ref) - size * (2.0 ** -8 + 2.0 ** -10)
    assert bad.max() <= 0, (bad.max(), np.unravel_index(bad.argmax(), bad.shape))
    return out


@pytest.mark.parametrize("lens", [[0], [1], [15, 16, 17], [63, 64, 65], [500, 0, 1, 129], [127, 128, 257]])
@pytest.mark.parametrize("G,rep", [(1, 1), (2, 4), (1, 8), (1, 16)])
def test_attn_one_token(fc, lens, G, rep):
    check_attn(fc, attn_case(len(lens) + rep, len(lens), 1, G * rep, G, lens, 16 if len(lens) % 2 else 64))


@pytest.mark.parametrize("n,H,G,page", [(2, 8, 2, 16), (5, 4, 4, 64), (8, 2, 1, 32), (9, 8, 2, 128), (16, 1, 1, 16),
                                        (17, 4, 1, 64), (33, 2, 2, 256), (64, 4, 1, 64), (65, 6, 2, 16), (100, 4, 2, 32),
                                        (127, 4, 1, 64), (128, 4, 1, 128), (128, 16, 1, 64)])
@pytest.mark.parametrize("kind", ["tree", "causal"])
def test_attn_trees(fc, n, H, G, page, kind):
    lens = [300, 0, 131]
    check_attn(fc, attn_case(n * 3 + H, 3, n, H, G, lens, page, nodes=[n, max(1, n // 2), max(1, n - 1)], kind=kind))


@pytest.mark.parametrize("n,H,G", [(1, 8, 2), (3, 4, 4), (40, 4, 2), (128, 4, 1)])
def test_attn_without_new_keys_and_without_any(fc, n, H, G):
    """The cache alone; a request with no cache then has rows that see nothing."""
    c = attn_case(n, 3, n, H, G, [200, 0, 33], 16)
    out = check_attn(fc, c, new=False)
    assert not out[1].any()


@pytest.mark.parametrize("n,H,G", [(1, 8, 2), (12, 4, 4), (128, 4, 1)])
def test_attn_masks_that_leave_a_row_empty(fc, n, H, G):
    c = attn_case(n + 50, 2, n, H, G, [0, 40], 16, nodes=[max(1, n - 1), n])
    c["sees"][:, 0] = False
    out = check_attn(fc, c)
    assert not out[0, 0].any() and out[1, 0].any()


def test_attn_rows_past_the_nodes_and_a_request_without_nodes(fc):
    c = attn_case(61, 3, 20, 4, 2, [70, 64, 5], 16, nodes=[0, 20, 3])
    out = check_attn(fc, c)
    assert not out[0].any() and not out[2, 3:].any() and out[1].any()


@pytest.mark.parametrize("n,H,G", [(3, 4, 2), (7, 4, 2), (40, 4, 2), (70, 4, 2), (128, 4, 2)])
def test_attn_what_is_not_finite_stays_with_the_rows_that_see_it(fc, n, H, G):
    """New tokens with a NaN or an infinity among their keys or values: rows
    that see them are NaN, the others what they are without them."""
    c = attn_case(n + 9, 2, n, H, G, [300, 9000], 64)
    c["v_new"][0, 0, n - 1, 5] = float("nan")
    c["v_new"][1, :, n // 2, 77] = -float("inf")
    c["k_new"][1, 0, 1, 3] = float("nan")
    hit = np.zeros((2, n, H), bool)
    hit[0, :, :H // G] = c["sees"][0, :, n - 1, None]
    hit[1] = c["sees"][1, :, n // 2, None]
    hit[1, :, :H // G] |= c["sees"][1, :, 1, None]
    assert hit.any() and not hit.all()
    for ws in (True, False):
        got = num(run_attn(fc, c, ws=ws))
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
        d = dict(c, v_new=torch.where(c["v_new"].isfinite(), c["v_new"], 0), k_new=torch.where(c["k_new"].isfinite(), c["k_new"], 0))
        ref, size = o4.attn(num(d["q"]), *(o4.pack(x) for x in d["codes"]), *d["scales"], d["table"], d["lens"],
                            num(d["k_new"]), num(d["v_new"]), d["sees"], d["nodes"], d["scale"])
        bad = np.abs(got - ref) - 2.0 ** -8 * np.abs(ref) - size * (2.0 ** -8 + 2.0 ** -10)
        assert bad[~hit].max() <= 0
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,L", [(1, 40000), (4, 20000), (70, 6000)])
def test_attn_long_and_split(fc, n, L):
    """Few requests with many keys: the keys are split and the parts joined,
    the same way every time, and alike without a workspace."""
    c = attn_case(L, 2, n, 4, 1, [L, L // 3 + 1], 64)
    if n > 1:
        c["q"], c["nodes"] = c["q"], c["nodes"]
    cache = gpu_cache(fc, c)
    out = check_attn(fc, c, cache=cache)
    for _ in range(4):
        assert torch.equal(run_attn(fc, c, cache=cache), out)
    one = run_attn(fc, c, cache=cache, ws=False)
    assert (one.float() - out.float()).abs().max() <= 2 ** -6 * out.float().abs().max()


@pytest.mark.parametrize("n", [1, 30])
def test_attn_sharp_and_shifted_scores(fc, n):
    """Queries that put all weight on few keys, late ones among them: the
    running maximum has to move."""
    c = attn_case(71 + n, 2, n, 4, 2, [700, 333], 32, qscale=12.0)
    c["lens"] = np.asarray([700, 333], np.int32)
    out = run_attn(fc, c)
    ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"],
                        num(c["k_new"]), num(c["v_new"]), c["sees"], c["nodes"], c["scale"])
    # scores reach 60: their fp32 errors (2^-22 * 136 * sum|q| s scale < 2^-8) are relative errors of p
    assert np.all(np.abs(num(out) - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -7))


def test_attn_one_workspace_for_every_shape(fc):
    """A workspace as large as any of them needs, zeroed once, for calls of
    different batches, heads and nodes in turn."""
    cases = [attn_case(300 + i, B, n, H, G, lens, 64) for i, (B, n, H, G, lens) in enumerate([
        (2, 40, 8, 2, [3000, 9000]), (1, 1, 8, 2, [20000]), (8, 1, 32, 8, [5000, 1, 0, 7000, 12000, 64, 300, 9000]),
        (1, 128, 8, 8, [4000]), (3, 5, 8, 2, [9000, 100, 4000]), (1, 1, 8, 8, [30000])])]
    shapes = [tuple(c["q"].shape[:3]) + (c["codes"][0].shape[1],) for c in cases]
    ws = torch.zeros(max(int(fc.LIB.fc_kv4_attn_workspace(*s)) for s in shapes), dtype=torch.uint8, device="cuda")
    want = [check_attn(fc, c) for c in cases]
    for i in [0, 1, 2, 3, 4, 5, 2, 0, 5, 4, 3, 2, 1]:
        c = cases[i]
        got = fc.fc_kv4_attn(c["q"].cuda(), gpu_cache(fc, c), dev(c["table"]), dev(c["lens"]), c["k_new"].cuda(),
                             c["v_new"].cuda(), dev(mask_words(c["sees"])), dev(c["nodes"]), scale=c["scale"], workspace=ws)
        assert torch.equal(got, want[i]), i
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n", [1, 8, 90])
def test_attn_refuses_bad_lengths_and_pages(fc, n):
    c = attn_case(81, 3, n, 4, 2, [64, 64, 64], 16, spare=0)
    good = run_attn(fc, c)
    bad = dict(c, lens=np.asarray([64, 65, -1], np.int32))  # tables of four pages
    out = run_attn(fc, bad)
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    assert torch.equal(out[0], good[0]) and not out[1:].any()
    bad = dict(c, nodes=np.asarray([n, n + 1, -1], np.int32))
    out = run_attn(fc, bad)
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    assert torch.equal(out[0], good[0]) and not out[1:].any()
    # a page outside the pool: its keys are left out
    t = c["table"].copy()
    t[1, 3], t[2, 3] = 13, -5
    out = run_attn(fc, dict(c, table=t))
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    short = run_attn(fc, dict(c, lens=np.asarray([64, 48, 48], np.int32)))
    assert (out.float() - short.float()).abs().max() <= 2 ** -6 * short.float().abs().max()
    assert fc.fc_get_error() == "FC_OK"


def test_attn_on_another_stream_and_in_a_graph(fc):
    c = attn_case(91, 2, 3, 8, 2, [3000, 1000], 64)
    cache, want = gpu_cache(fc, c), run_attn(fc, c)
    args = [c["q"].cuda(), cache, dev(c["table"]), dev(c["lens"]), c["k_new"].cuda(), c["v_new"].cuda(),
            dev(mask_words(c["sees"])), dev(c["nodes"])]
    kw = dict(scale=c["scale"], out=torch.empty_like(args[0]), workspace=fc.kv4_attn_workspace(2, 3, 8, 2, "cuda"))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert torch.equal(fc.fc_kv4_attn(*args, **kw), want)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fc.fc_kv4_attn(*args, **kw)
    for _ in range(3):
        kw["out"].zero_()
        g.replay()
        assert torch.equal(kw["out"], want)


def zero_values(c, which):
    """Value rows of zeros as a write leaves them: numbers 0, scale 0."""
    page = c["codes"][1].shape[2]
    for b, L in enumerate(c["lens"]):
        at = {"all": np.arange(L), "first": np.arange(1), "first 32": np.arange(min(L, 32)), "every fourth": np.arange(0, L, 4),
              "last": np.arange(L - 1, L)}[which]
        c["codes"][1][c["table"][b, at // page], :, at % page] = 0
        c["scales"][1][c["table"][b, at // page], :, at % page] = 0


@pytest.mark.parametrize("which", ["all", "first", "first 32", "every fourth", "last"])
@pytest.mark.parametrize("n,H,G", [(1, 8, 2), (3, 8, 2), (20, 4, 2)])
def test_attn_value_rows_of_zeros(fc, which, n, H, G):
    """Scale 0 is how a row of zeros is held: such keys count in the row sum
    and add nothing.  33 keys end in a step of one key, 1000 are cut in parts."""
    c = attn_case(n + len(which), 4, n, H, G, [1, 33, 300, 1000], 16)
    zero_values(c, which)
    for ws in (True, False):
        check_attn(fc, c, ws=ws)
    out = check_attn(fc, c, new=False)
    assert bool(out.any()) == (which != "all")


@pytest.mark.parametrize("n,H,G", [(1, 2, 1), (1, 16, 2), (2, 16, 2), (20, 4, 2)])
def test_attn_a_query_with_a_nan_is_alone_with_it(fc, n, H, G):
    """Rows share lanes and steps with a row of NaN while their own scores grow
    tenfold after 256 keys, so that their references have to move.  Scores'
    fp32 errors, 2^-22 * 136 * sum|q| * 2 * scale < 2^-10, are relative errors of
    p, and of the row sum once more."""
    c = attn_case(5 * n + H, 2, n, H, G, [2000, 700], 64)
    c["scales"][0][...] = 0.2
    for b in range(2):
        c["scales"][0][c["table"][b, 4:-(-c["lens"][b] // 64)]] = 2.0
    hit = np.zeros(c["q"].shape[:3], bool)
    hit[:, 0, ::H // G] = True
    ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"], num(c["k_new"]),
                        num(c["v_new"]), c["sees"], c["nodes"], c["scale"])
    c["q"][torch.from_numpy(hit)] = float("nan")
    for ws in (True, False):
        got = num(run_attn(fc, c, ws=ws))
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
        assert np.all((np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -9))[~hit])
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,G", [(1, 8, 2), (4, 16, 4), (20, 4, 2), (128, 4, 2)])
def test_attn_scales_far_apart(fc, n, H, G):
    """Value scales of 2^-60 to 2^20 and key scales of 2^-60 to 2^-1 side by
    side, some of them 0.  Beside the usual tolerance: weights are held
    relative to the largest, in fp16 at 2^11 or more, so that those below
    fp16's normal range are off by up to 2^-25: 2^-36 of that key's |c| s (at
    most 7 times its largest weight's) for each key.  Keys lose 2^-34 of their 16
    neighbours' largest (2^-1), less than what a score is off by anyway."""
    rng = np.random.default_rng(n)
    c = attn_case(n + 7, 3, n, H, G, [300, 37, 1000], 32, stale=False)
    for i, hi in ((0, -1), (1, 20)):
        s = o4.bf16_round(2.0 ** rng.uniform(-60, hi, c["scales"][i].shape))
        s[rng.random(s.shape) < 0.05] = 0
        c["scales"][i][...] = s
    for ws in (True, False):
        for new in (True, False):
            got = num(run_attn(fc, c, ws=ws, new=new))
            kn, vn = (num(c["k_new"]), num(c["v_new"])) if new else (None, None)
            ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"], kn, vn,
                                c["sees"], c["nodes"], c["scale"])
            floor = (c["lens"].max() + n) * 2.0 ** -33 * size.max(-1, keepdims=True)
            assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -10) + floor)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,G", [(1, 8, 2), (4, 16, 4), (20, 4, 2)])
def test_attn_key_rows_of_zeros_and_a_cache_never_written(fc, n, H, G):
    c = attn_case(n + 8, 2, n, H, G, [70, 333], 16, stale=False)
    c["codes"][0][...] = 0
    c["scales"][0][...] = 0
    check_attn(fc, c)  # every cached key scores 0: the mean of the values
    check_attn(fc, c, new=False)
    n_pages = c["codes"][0].shape[0]
    cache = fc.Kv4Cache.empty(n_pages, G, 16)
    assert not run_attn(fc, c, new=False, cache=cache).any()
    c["codes"][1][...] = 0
    c["scales"][1][...] = 0
    check_attn(fc, c, cache=cache)  # zeros weigh as much as the new tokens' scores leave them


@pytest.mark.parametrize("n,H,G", [(4, 8, 4), (4, 16, 4), (20, 4, 2)])
def test_attn_queries_of_other_sizes_beside_each_other(fc, n, H, G):
    """A head's queries 2^20 times the others': it keeps to its own rows."""
    c = attn_case(n + 11, 2, n, H, G, [200, 33], 16)
    big = np.zeros(c["q"].shape[:3], bool)
    big[:, 0] = True
    ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"], num(c["k_new"]),
                        num(c["v_new"]), c["sees"], c["nodes"], c["scale"])
    c["q"][:, 0] *= 2.0 ** 20
    got = num(run_attn(fc, c))
    assert np.isfinite(got).all()
    assert np.all((np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -10))[~big])
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n,H,G", [(3, 4, 2), (7, 4, 2), (40, 4, 2), (128, 4, 2)])
def test_attn_an_infinite_key_counts_as_its_product(fc, n, H, G, sign):
    """Where the product with the query is +inf the row is NaN, where it is
    -inf the key has no weight; rows that do not see it are untouched."""
    c = attn_case(n + 13, 2, n, H, G, [300, 0], 64)
    c["k_new"][:, :, 1, 3] = sign * float("inf")
    up = num(c["q"])[..., 3] * sign > 0
    sees = np.broadcast_to(c["sees"][:, :, 1, None], up.shape)
    assert (up & sees).any() and (~up & sees).any() and (~sees).any()
    with np.errstate(invalid="ignore"):
        ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"],
                            num(c["k_new"]), num(c["v_new"]), c["sees"], c["nodes"], c["scale"])
    hit = up & sees
    for ws in (True, False):
        got = num(run_attn(fc, c, ws=ws))
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
        assert np.all(np.abs(got - ref)[~hit] <= (2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -10))[~hit])
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("L", [2 ** 31 - 1, 2 ** 31 - 200, 2 ** 31 - 40])
@pytest.mark.parametrize("n,tol", [(1, 2.0 ** -7 + 2.0 ** -7), (20, 2.0 ** -7 + 0.053)])
def test_attn_of_a_length_just_below_32_bits(fc, L, n, tol):
    """One page again and again: all keys score alike, so that the result is
    the page's mean.  Roundings of two bf16 (2^-7), and of the fp32 sums: 56,000
    (of one token's warps) or 442,000 (of a tile) products one after another, each
    off by up to 2^-23 of the sum so far."""
    rng = np.random.default_rng(n)
    v = rng.integers(1, 8, (256, 128))
    cache = fc.Kv4Cache.empty(1, 1, 256)
    cache.k_codes.copy_(dev(o4.pack(np.zeros((1, 1, 256, 128), np.int64))))
    cache.v_codes.copy_(dev(o4.pack(v)[None, None]))
    cache.k_scale.fill_(1)
    cache.v_scale.fill_(1)
    q = bf(rng, 1, n, 1, 128).cuda()
    table = torch.zeros((1, 2 ** 23), dtype=torch.int32, device="cuda")
    out = fc.fc_kv4_attn(q, cache, table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                         workspace=fc.kv4_attn_workspace(1, n, 1, 1, "cuda"))
    assert fc.fc_get_error() == "FC_OK"
    want = v.mean(0)
    assert np.all(np.abs(num(out) - want) <= tol * want)


@pytest.mark.parametrize("n,H,G,lens", [(1, 8, 2, [9000, 1]), (4, 16, 4, [5000, 0, 3000]), (20, 4, 2, [3000, 5000]),
                                        (128, 4, 2, [2000, 700])])
def test_attn_with_less_workspace(fc, n, H, G, lens):
    """Any smaller workspace serves, zeroed once, with nothing written past its
    end, and the next call may have another size."""
    c = attn_case(n + 401, len(lens), n, H, G, lens, 64)
    cache = gpu_cache(fc, c)
    want = check_attn(fc, c, cache=cache)
    full = int(fc.LIB.fc_kv4_attn_workspace(len(lens), n, H, G))
    args = (c["q"].cuda(), cache, dev(c["table"]), dev(c["lens"]), c["k_new"].cuda(), c["v_new"].cuda(),
            dev(mask_words(c["sees"])), dev(c["nodes"]))
    ref, size = o4.attn(num(c["q"]), *(o4.pack(x) for x in c["codes"]), *c["scales"], c["table"], c["lens"], num(c["k_new"]),
                        num(c["v_new"]), c["sees"], c["nodes"], c["scale"])
    buf = torch.zeros(full + 4096, dtype=torch.uint8, device="cuda")
    for size_now in (full, full // 2, 1, 256, 1280, 1281, full // 50, full // 7 + 13, full - 1, full):
        buf[size_now:] = 0xA5
        out = fc.fc_kv4_attn(*args, scale=c["scale"], workspace=buf[:size_now])
        assert fc.fc_get_error() == "FC_OK"
        assert np.all(np.abs(num(out) - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -8 + 2.0 ** -10)), size_now
        assert bool((buf[size_now:] == 0xA5).all()), size_now
        if size_now == full:
            assert torch.equal(out, want)
        buf[size_now:min(1280, full)] = 0  # its counters, for a larger one


@pytest.mark.parametrize("n,H,G,L", [(1, 32, 8, 8000), (4, 32, 8, 4000), (32, 32, 8, 2000)])
def test_attn_a_small_workspace_is_no_slower_than_none(fc, n, H, G, L):
    """A workspace with room for the parts of two CTAs: whole units then, on
    all of the GPU (two CTAs for everything would take tens of times as long)."""
    c = attn_case(n + 77, 1, n, H, G, [L], 64)
    q, kn, vn = (c[k].cuda().repeat_interleave(16, 0) for k in ("q", "k_new", "v_new"))
    table, lens = dev(c["table"]).repeat(16, 1), dev(c["lens"]).repeat(16)
    cache, out = gpu_cache(fc, c), torch.empty_like(q)
    full = fc.kv4_attn_workspace(16, n, H, G, "cuda")
    few = 1280 + 2 * 2 * 16 * 130 * 4 if n * H // G <= 16 else 1280 + 256 + 2 * 2 * min(256, n * H // G) * 520

    def ms(ws):
        call = lambda: fc.fc_kv4_attn(q, cache, table, lens, kn, vn, out=out, workspace=ws)
        call()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(5):
            call()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / 5

    none, some = ms(None), ms(full[:few])
    assert some < 3 * none, (none, some)
    assert fc.fc_get_error() == "FC_OK"


# ------------------------------------------------------------------ product
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16])
@pytest.mark.parametrize("K,N,group", [(64, 1, 32), (64, 16, 64), (128, 33, 128), (320, 100, 64), (2048, 50, 32),
                                       (448, 2500, 64), (1024, 2049, 128)])
def test_matvec(fc, M, K, N, group):
    rng = np.random.default_rng(M * K + N)
    w, x = bf(rng, K, N, scale=K ** -0.5), bf(rng, M, K)
    h = fc.fc_w4_pack(w.cuda(), group)
    c, s = o4.quantise(num(w).reshape(K // group, group, N), 1)
    assert np.array_equal(num(h.scale), s)
    out = fc.fc_w4_matvec(x.cuda(), h)
    assert fc.fc_get_error() == "FC_OK"
    y, size = o4.matvec(num(x), num(w), group)
    e = 2.0 ** -20 * 136 * size
    got = num(out)
    assert np.all((o4.bf16_round(y - e) <= got) & (got <= o4.bf16_round(y + e)))


@pytest.mark.parametrize("M", [1, 8, 9, 16])
@pytest.mark.parametrize("K,N,group", [(64, 4865, 32), (320, 4900, 64), (256, 9728, 128), (192, 19457, 32), (576, 19500, 64),
                                       (128, 20001, 128), (128, 32256, 32)])
def test_matvec_of_wide_weights(fc, M, K, N, group):
    """Widths on either side of where a warp takes two and four column tiles,
    odd ones and such that end inside a tile."""
    test_matvec(fc, M, K, N, group)


def test_matvec_of_unit_rows_reads_the_weights_back(fc):
    """x = a unit row: the product is one row of the weights, so every number
    of the packed layout is checked by itself."""
    rng = np.random.default_rng(5)
    K, N, group = 192, 37, 64
    w = bf(rng, K, N)
    c, s = o4.quantise(num(w).reshape(K // group, group, N), 1)
    want = o4.bf16_round((c * s[:, None]).reshape(K, N))
    h = fc.fc_w4_pack(w.cuda(), group)
    eye = torch.eye(K, dtype=torch.bfloat16, device="cuda")
    got = torch.cat([fc.fc_w4_matvec(eye[i:i + 16].contiguous(), h) for i in range(0, K, 16)])
    assert np.array_equal(num(got), want)


def test_matvec_extremes_and_refusals(fc):
    K, N = 128, 40
    w = torch.zeros((K, N), dtype=torch.bfloat16, device="cuda")
    w[:, 1], w[3, 2], w[4, 3] = 2.0 ** -120, float("nan"), float("inf")
    out = fc.fc_w4_matvec(torch.ones((2, K), dtype=torch.bfloat16, device="cuda"), fc.fc_w4_pack(w, 64))
    assert not out[:, 0].any() and torch.isnan(out[:, 2:4]).all() and not out[:, 4:].any()
    assert (out[:, 1].double() / (128 * 2.0 ** -120) - 1).abs().max() < 0.01
    with pytest.raises(fc.FastCoderError):
        fc.fc_w4_matvec(torch.ones((17, K), dtype=torch.bfloat16, device="cuda"), fc.fc_w4_pack(w, 64))
    with pytest.raises(ValueError):
        fc.fc_w4_matvec(torch.ones((2, 64), dtype=torch.bfloat16, device="cuda"), fc.fc_w4_pack(w, 64))
    with pytest.raises(ValueError):
        fc.fc_w4_pack(torch.zeros((100, 8), dtype=torch.bfloat16, device="cuda"), 32)
    with pytest.raises(fc.FastCoderError):
        fc.fc_w4_pack(w, 48)


@pytest.mark.parametrize("M", [1, 8, 9, 16])
@pytest.mark.parametrize("K,N,group", [(64, 40, 32), (256, 100, 128), (192, 4900, 64), (128, 20000, 32)])
def test_matvec_of_large_x(fc, M, K, N, group):
    """x up to 2^118: a group of 128 products stays below 2^128, whatever the
    signs.  (A finite result is expected, with the usual tolerance.)"""
    rng = np.random.default_rng(M + K + N)
    w = bf(rng, K, N, scale=2.0 ** -100)
    x = (bf(rng, M, K).abs().clamp(max=2.0) * 2.0 ** 117).bfloat16()
    out = num(fc.fc_w4_matvec(x.cuda(), fc.fc_w4_pack(w.cuda(), group)))
    assert fc.fc_get_error() == "FC_OK" and np.isfinite(out).all()
    y, size = o4.matvec(num(x), num(w), group)
    e = 2.0 ** -20 * 136 * size
    assert np.all((o4.bf16_round(y - e) <= out) & (out <= o4.bf16_round(y + e)))


@pytest.mark.parametrize("M", [1, 8, 9, 16])
@pytest.mark.parametrize("K,N,group", [(1024, 40, 32), (1024, 100, 128), (512, 4900, 64), (256, 20000, 128)])
def test_matvec_of_columns_that_cancel(fc, M, K, N, group):
    """Columns whose products cancel pair by pair next to columns of one sign:
    the result is off by roundings of sums of c x s alone.  |c| <= 7; a sum
    has at most 32 groups (a rounding of 2^-24 each) of at most 8 matrix
    products (2^-23 each): below (32 + 16) 2^-24 * 7 sum|x| s."""
    rng = np.random.default_rng(M + K + N)
    w = bf(rng, K, N).abs()
    w[1::2] = -w[0::2]
    w[:, ::3] = w[:, ::3].abs()
    x = bf(rng, M, K).abs()
    x[:, 1::2] = x[:, 0::2]
    out = num(fc.fc_w4_matvec(x.cuda(), fc.fc_w4_pack(w.cuda(), group)))
    y, size = o4.matvec(num(x), num(w), group)
    e = 48 * 2.0 ** -24 * 7 * size
    assert np.all((o4.bf16_round(y - e) <= out) & (out <= o4.bf16_round(y + e)))
    assert fc.fc_get_error() == "FC_OK"


def test_matvec_of_x_that_is_not_finite(fc):
    """An infinity counts as its product with the weight, a NaN makes the row
    NaN; the other rows are what they are without them."""
    rng = np.random.default_rng(29)
    K, N, group = 128, 333, 64
    w, x = bf(rng, K, N), bf(rng, 9, K)
    c, _ = o4.quantise(num(w).reshape(K // group, group, N), 1)
    row = c.reshape(K, N)[70]
    h = fc.fc_w4_pack(w.cuda(), group)
    want = num(fc.fc_w4_matvec(x.cuda(), h))
    x[1, 70], x[4, 70], x[8, 3] = float("inf"), -float("inf"), float("nan")
    got = num(fc.fc_w4_matvec(x.cuda(), h))
    assert (row == 0).any() and (row != 0).any() and np.isnan(got[8]).all()
    for r, sign in ((1, 1), (4, -1)):
        assert np.isnan(got[r][row == 0]).all() and np.all(got[r][row != 0] == np.sign(row[row != 0]) * sign * np.inf)
    keep = [0, 2, 3, 5, 6, 7]
    assert np.array_equal(got[keep], want[keep])
    assert fc.fc_get_error() == "FC_OK"


def test_binding_refuses_outputs_that_are_too_small(fc):
    """Nothing is launched: a call would write past their ends, or read what is
    no device memory."""
    i32 = dict(dtype=torch.int32, device="cuda")
    B, rows = 3, 8
    pages = fc.KvPages(16, torch.zeros((B, 4), **i32), torch.arange(12, **i32))
    kv, new, n_free = torch.zeros(B, **i32), torch.full((B,), 2, **i32), torch.full((1,), 12, **i32)
    for k, n in (("pos", rows - 1), ("slot", rows + 1), ("src", rows - 1), ("cu", B), ("kv_len", B - 1), ("n_free", 0)):
        out = fc.kv_pages_outputs(B, rows, "cuda", src=True)
        out[k] = torch.empty(n, **i32)
        with pytest.raises(ValueError):
            fc.fc_kv_pages_plan(pages, kv, new, n_free, n_per_seq=2, out=out)
    for k, bad in (("seq", torch.empty(rows, dtype=torch.int64, device="cuda")), ("slot", torch.empty(rows, dtype=torch.int16, device="cuda")),
                   ("pos", torch.empty(rows, dtype=torch.int32)), ("cu", torch.empty(2 * (B + 1), **i32)[::2])):
        with pytest.raises((TypeError, ValueError)):
            fc.fc_kv_pages_plan(pages, kv, new, n_free, out=dict(fc.kv_pages_outputs(B, rows, "cuda"), **{k: bad}))
    with pytest.raises(ValueError):
        fc.fc_kv_pages_plan(pages, kv, new, n_free, rows_cap=rows, path=torch.empty((B, 0), **i32), n_per_seq=2)
    for bad in ((torch.empty(B - 1, **i32), torch.empty(1, **i32)), (torch.empty(B, **i32), torch.empty(0, **i32)),
                (torch.empty(B, dtype=torch.int64, device="cuda"), torch.empty(1, **i32))):
        with pytest.raises((TypeError, ValueError)):
            fc.fc_kv_pages_release(pages, kv, kv, n_free, out=bad)
    cache = fc.Kv4Cache.empty(12, 2, 16)
    q = torch.zeros((B, 1, 4, 128), dtype=torch.bfloat16, device="cuda")
    ws = fc.kv4_attn_workspace(B, 1, 4, 2, "cuda")
    for bad in (ws.cpu(), ws[::2]):
        with pytest.raises(ValueError):
            fc.fc_kv4_attn(q, cache, pages.table, kv, workspace=bad)
    h = fc.fc_w4_pack(torch.zeros((128, 40), dtype=torch.bfloat16, device="cuda"), 64)
    fc.W4Weight(h.codes, h.scale, 128, 40, 64)
    for bad in ((h.codes[:-1], h.scale, 128, 40, 64), (h.codes, h.scale, 128, 56, 64), (h.codes, h.scale, 128, 40, 32),
                (h.codes.cpu(), h.scale, 128, 40, 64), (h.codes, h.scale.float(), 128, 40, 64), (h.codes, h.scale, 128, 40, 0)):
        with pytest.raises((TypeError, ValueError)):
            fc.W4Weight(*bad)
    with pytest.raises(ValueError):
        fc.fc_w4_pack(torch.zeros((128, 40), dtype=torch.bfloat16, device="cuda"), 0)
    assert fc.fc_get_error() == "FC_OK"
