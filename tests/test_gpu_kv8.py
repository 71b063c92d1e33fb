"""Serving from the 8-bit cache on the GPU against the 64-bit oracle (oracle/kv8.py).

Codes, scales, positions and indexes are equal.  bf16 has 8 significant bits,
so a rounding to it moves a value by at most 2^-8 of itself.  Floating
tolerances, per element:
* attention: the output's rounding, 2^-8 |out|; each probability's rounding to
  16 bits, 2^-8 of A = the mean of |v| under the same probabilities; and a
  score's error e (oracle.attend), which changes a probability and the row sum
  by e of themselves: 2 e A.  fp32 sums of up to 2^17 probabilities in pieces:
  2^-16 A.
* weights: the scores' error on probability and row sum, 2 e, and fp32's
  arithmetic (exp2's 2^-22, sums), 2^-18, of each.
* norm and rotation: y's rounding, 2^-8 |y|; sine and cosine are good to 2^-20
  and the angle to 1e-6 (absolute), fp32's arithmetic to 2^-20: 2^-18 of |a| + |b|.
"""
import numpy as np
import pytest
import torch

from oracle import kv8 as o8

pytestmark = pytest.mark.gpu
D = 128


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


def random_cache(rng, n_pages, H, page, stale=False):
    codes = [o8.encode(np.clip(rng.standard_normal((n_pages, H, page, D)) * 100, -448, 448)) for _ in range(2)]
    scales = [(2.0 ** rng.integers(-8, -5, (n_pages, H, page // 16))).astype(np.float32) for _ in range(2)]
    return codes + scales


def on_gpu(fc, cache):
    return fc.Kv8Cache(*(dev(c) for c in cache))


def same_cache(got, want):
    for name, g, w in zip(("k_codes", "v_codes", "k_scale", "v_scale"), (got.k_codes, got.v_codes, got.k_scale, got.v_scale), want):
        assert np.array_equal(g.cpu().numpy(), w, equal_nan=w.dtype.kind == "f"), name


# ------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("B,n,H,Hkv,dim", [(1, 1, 1, 1, 128), (32, 1, 32, 8, 128), (3, 7, 5, 2, 64), (2, 130, 16, 16, 128),
                                           (1, 3, 6, 3, 16), (2, 5, 4, 1, 80), (1, 9, 8, 2, 256), (1, 2, 2, 2, 512), (700, 3, 40, 8, 128)])
def test_norm_rope(fc, B, n, H, Hkv, dim):
    rng = np.random.default_rng(B + n + dim)
    q, kv = bf(rng, B, n, H + 3, dim, scale=3.0), bf(rng, B, n, 2, Hkv, dim)
    q[0, 0, 0] = 0
    wq, wk = (bf(rng, dim) for _ in range(2))
    pos = rng.integers(0, 1 << 20, (B, n)).astype(np.int32)
    pos[-1, -1] = -1  # not turned
    pos[0, 0] = (1 << 24) - 1
    qg, kvg = q.cuda()[:, :, 1:1 + H], kv.cuda()
    out = fc.fc_qk_norm_rope(qg, kvg[:, :, 0], kvg[:, :, 1], wq.cuda(), wk.cuda(), dev(pos), 1e6, 1e-5)
    assert fc.fc_get_error() == "FC_OK"
    for x, w, got, turn in ((q[:, :, 1:1 + H], wq, out[0], False), (kv[:, :, 0], wk, out[1], True)):
        ref, mag = o8.norm_rope(num(x), num(w), pos.astype(np.float64), 1e6, 1e-5)
        if turn:
            ref, mag = ref.transpose(0, 2, 1, 3), mag.transpose(0, 2, 1, 3)
        assert np.all(np.abs(num(got) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * mag)
    assert torch.equal(out[2], kvg[:, :, 1].transpose(1, 2))
    two = fc.fc_qk_norm_rope(qg, kvg[:, :, 0], None, wq.cuda(), wk.cuda(), dev(pos), 1e6, 1e-5)
    assert two[2] is None and torch.equal(two[0], out[0]) and torch.equal(two[1], out[1])


def test_norm_rope_dimensions_of_one(fc):
    """One row, one head: their strides are not looked at."""
    rng = np.random.default_rng(4)
    x = bf(rng, 3, 64).cuda()
    odd = lambda r: torch.as_strided(x, (1, 1, 1, 64), (7, 3, 5, 1), 64 * r)
    w, pos = bf(rng, 64).cuda(), torch.full((1, 1), 9, dtype=torch.int32).cuda()
    out = fc.fc_qk_norm_rope(odd(0), odd(1), odd(2), w, w, pos)
    ref = fc.fc_qk_norm_rope(*(x[r].view(1, 1, 1, 64) for r in range(3)), w, w, pos)
    assert all(torch.equal(a, b) for a, b in zip(out, ref))
    got = fc.fc_qk_norm_rope(*(x[:0].view(0, 1, 1, 64) for _ in range(3)), w, w, pos[:0])
    assert got[0].shape == (0, 1, 1, 64)


def test_norm_rope_rows_that_are_not_finite_stay_alone(fc):
    rng = np.random.default_rng(3)
    q, k = bf(rng, 2, 4, 8, D).cuda(), bf(rng, 2, 4, 2, D).cuda()
    w, pos = bf(rng, D).cuda(), dev(np.arange(8).reshape(2, 4).astype(np.int32))
    clean = fc.fc_qk_norm_rope(q, k, k, w, w, pos)
    q[1, 2, 3, 5], k[0, 1, 1, 70] = float("nan"), float("inf")
    bad = fc.fc_qk_norm_rope(q, k, k, w, w, pos)
    assert bad[0][1, 2, 3].isnan().all() and bad[1][0, 1, 1].isnan().any()
    bad[0][1, 2, 3] = clean[0][1, 2, 3]
    bad[1][0, 1, 1] = clean[1][0, 1, 1]
    assert torch.equal(bad[0], clean[0]) and torch.equal(bad[1], clean[1])


# ------------------------------------------------------------------ writes
def plan(rng, kv, new, page, gaps=False):
    """Slots of new[b] tokens behind kv[b], pages in no order; n_pages, positions, tables."""
    held = [-(-int(k + n) // page) for k, n in zip(kv, new)]
    order = rng.permutation(sum(held) + 2).astype(np.int32)
    slot, pos, at = [], [], 0
    table = np.zeros((len(kv), max(max(held), 1)), np.int32)
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
        p = np.arange(kv[b], kv[b] + new[b])
        slot.append(table[b][p // page] * page + p % page)
        pos.append(p)
    slot = np.concatenate(slot).astype(np.int32)
    if gaps:
        slot[rng.random(len(slot)) < 0.1] = -1
    return slot, len(order), np.concatenate(pos).astype(np.int32), table


@pytest.mark.parametrize("kv,new,H,page,gaps", [([0], [1], 1, 16, False), ([5], [1], 2, 64, False), ([15, 16, 3], [1, 1, 1], 8, 32, False),
                                                ([7, 0, 100], [40, 16, 333], 3, 128, True), ([0] * 40, [9] * 40, 8, 16, True),
                                                ([3, 90], [2000, 777], 8, 256, True), ([11] * 5, [0, 1, 2, 3, 70], 32, 64, False)])
def test_write_and_read(fc, kv, new, H, page, gaps):
    rng = np.random.default_rng(len(kv) + H + page)
    slot, n_pages, pos, _ = plan(rng, kv, new, page, gaps)
    rows = len(slot)
    cache = random_cache(rng, n_pages, H, page)
    x = bf(rng, rows, 6 * H * D) * torch.exp(torch.from_numpy(rng.standard_normal((rows, 1)) * 2)).bfloat16()
    x[rows // 2] = 0
    xg = x.cuda()
    got = on_gpu(fc, cache)
    track = fc.Kv8Track(torch.full((n_pages, H, page), 3.5).cuda(), torch.full((n_pages, H, page), -7, dtype=torch.int32).cuda())
    rt = [track.weight.cpu().numpy(), track.born.cpu().numpy()]
    part = lambda t, i: t[:, i * H * D:(i + 1) * H * D].view(rows, H, D)
    fc.fc_kv8_write(got, part(xg, 4), part(xg, 5), dev(slot), track=track, pos=dev(pos))
    assert fc.fc_get_error() == "FC_OK"
    o8.write(cache, num(part(x, 4)), num(part(x, 5)), slot, None, rt, pos)
    same_cache(got, cache)
    assert np.array_equal(track.weight.cpu().numpy(), rt[0]) and np.array_equal(track.born.cpu().numpy(), rt[1])
    k, v = fc.fc_kv8_read(got, dev(slot))
    for t, i in ((k, 0), (v, 1)):
        p, o = slot // page, slot % page
        want = o8.decode(cache[i][p, :, o]) * cache[2 + i][p, :, o // 16].astype(np.float64)[..., None]
        want[slot < 0] = 0
        assert np.array_equal(num(t), want)
    again = on_gpu(fc, cache)  # the same rows once more change nothing
    fc.fc_kv8_write(again, part(xg, 4), part(xg, 5), dev(slot))
    same_cache(again, cache)


def test_write_one_by_one_and_head_major(fc):
    """Tokens appended singly, from head-major tensors by src, end as the oracle's do."""
    rng = np.random.default_rng(5)
    H, page, n = 4, 32, 45
    cache = random_cache(rng, 4, H, page)
    got = on_gpu(fc, cache)
    x = [bf(rng, 2, H, 8, D, scale=10.0 ** float(e)).cuda() for e in rng.integers(-3, 4, n)]
    for t in range(n):
        slot = np.array([2 * page + t if t < 32 else t - 32], np.int32)
        src = np.array([int(rng.integers(0, 16))], np.int32)
        rows = x[t].transpose(1, 2)
        fc.fc_kv8_write(got, rows, rows, dev(slot), src=dev(src))
        r = num(rows.reshape(16, H, D))
        o8.write(cache, r, r, slot, src)
    assert fc.fc_get_error() == "FC_OK"
    same_cache(got, cache)


def test_write_extremes(fc):
    """The largest and smallest bf16 numbers, zeros, NaN and infinities, and blocks begun anew."""
    H, page = 1, 16
    big, tiny = 3.3895313892515355e38, 9.183549615799121e-41
    x = torch.zeros(5, H, D)
    x[0, 0, :3] = torch.tensor([big, -1.0, tiny])
    x[1, 0, :2] = torch.tensor([tiny, -tiny])
    x[3, 0, 9] = float("nan")
    x[4, 0, 1] = float("-inf")
    x = x.bfloat16()
    slot = np.array([0, 16, 33, 52, 66], np.int32)
    rng = np.random.default_rng(1)
    cache = random_cache(rng, 6, H, page)
    got = on_gpu(fc, cache)
    fc.fc_kv8_write(got, x.cuda(), x.cuda(), dev(slot))
    o8.write(cache, num(x), num(x), slot)
    same_cache(got, cache)
    one = torch.ones(2, H, D).bfloat16()
    more = np.array([53, 64], np.int32)  # into a block that stands for NaN; into one from its start
    fc.fc_kv8_write(got, one.cuda(), one.cuda(), dev(more))
    o8.write(cache, num(one), num(one), more)
    same_cache(got, cache)
    k, _ = fc.fc_kv8_read(got, dev(np.array([52, 53, 64], np.int32)))
    assert k[:2].isnan().all() and (k[2] == 1).all() and fc.fc_get_error() == "FC_OK"


def test_write_leaves_out_what_is_out_of_range(fc):
    rng = np.random.default_rng(6)
    cache = random_cache(rng, 3, 2, 16)
    got = on_gpu(fc, cache)
    x = bf(rng, 4, 2, D)
    slot, src = np.array([0, 48, 17, 18], np.int32), np.array([0, 1, 4, 3], np.int32)  # slot 48 and row 4 are none
    fc.fc_kv8_write(got, x.cuda(), x.cuda(), dev(slot), src=dev(src))
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
    o8.write(cache, num(x), num(x), slot, src)
    same_cache(got, cache)
    k, v = fc.fc_kv8_read(got, dev(np.array([1 << 30, -1], np.int32)))
    assert fc.fc_get_error() == "FC_ERR_INVALID_ARG" and (k == 0).all() and (v == 0).all()


# ------------------------------------------------------------------ attention
def trees(rng, nodes, n):
    words = (n + 63) // 64
    m = np.zeros((len(nodes), n, words), np.uint64)
    for b, nn in enumerate(nodes):
        for i in range(nn):
            if i:
                m[b, i] = m[b, rng.integers(max(0, i - 8), i)]
            m[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m.view(np.int64)


def setup(rng, kv, n, H, Hkv, page, nodes=None, stale=True):
    B = len(kv)
    held = [-(-k // page) for k in kv]
    n_pages = sum(held) + 2
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, max(max(held), 1) + 1), -5, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    cache = random_cache(rng, n_pages, Hkv, page)
    if stale:  # what stands past a request's end is anything
        for b, k in enumerate(kv):
            for j in range(k, held[b] * page):
                for i in range(2):
                    cache[i][table[b, j // page], :, j % page] = 0x7F
                    if j % 16 == 0:
                        cache[2 + i][table[b, j // page], :, j % page // 16] = np.nan
    return dict(kv=np.array(kv, np.int32), nodes=np.array(nodes if nodes is not None else [n] * B, np.int32), table=table, cache=cache,
                q=bf(rng, B, n, H, D), k=bf(rng, B, Hkv, n, D), v=bf(rng, B, Hkv, n, D))


def reference(s, masks, scale, new=True, causal=False):
    B, n, H, _ = s["q"].shape
    Hkv = s["k"].shape[1]
    G = H // Hkv
    page = s["cache"][0].shape[2]
    out, mean, err = (np.zeros((B, n, H, m)) for m in (D, D, 1))
    weight, werr = np.zeros(s["cache"][0].shape[:3]), np.zeros(s["cache"][0].shape[:3])
    for b in range(B):
        L, m = int(s["kv"][b]), int(s["nodes"][b])
        i = np.arange(L)
        p, o = s["table"][b][i // page], i % page
        vis = np.zeros((m, m), bool)
        for x in range(m):
            for y in range(m):
                vis[x, y] = y <= x if causal else bool((int(masks[b, x, y // 64]) >> (y % 64)) & 1)
        if not new:
            vis = np.zeros((m, 0), bool)
        sees = np.concatenate((np.ones((m, L), bool), vis), 1)
        for g in range(Hkv):
            K, V = (np.concatenate((o8.cached(s["cache"], w, s["table"][b], L, g), num(s[x][b, g, :m if new else 0])))
                    for w, x in ((0, "k"), (1, "v")))
            for h in range(g * G, (g + 1) * G):
                out[b, :m, h], w, mean[b, :m, h], err[b, :m, h] = o8.attend(num(s["q"][b, :m, h]), K, V, sees, scale)
                weight[p, g, o] += w[:, :L].sum(0)
                werr[p, g, o] += ((2 * err[b, :m, h] + 2.0 ** -18) * w[:, :L]).sum(0)
    return out, (2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2.0 ** -16 + 2 * err) * mean), weight, werr


def call(fc, s, masks=None, new=True, **kw):
    c = on_gpu(fc, s["cache"])
    k, v = (s["k"].cuda(), s["v"].cuda()) if new else (None, None)
    return fc.fc_kv8_attn(s["q"].cuda(), c, dev(s["table"]), dev(s["kv"]), k, v, None if masks is None else dev(masks), dev(s["nodes"]), **kw)


SHAPES = [([0], 1, 1, 1, 16), ([1], 1, 8, 8, 16), ([17], 1, 4, 1, 16), ([500], 1, 32, 8, 64), ([31, 32, 33, 0], 1, 16, 2, 32),
          ([1000, 3, 257], 1, 8, 8, 128), ([700, 64], 2, 16, 8, 256), ([129, 5], 4, 8, 2, 64), ([300], 16, 2, 2, 16),
          ([2500], 3, 8, 2, 64), ([9000], 1, 2, 1, 64), ([100, 200], 2, 32, 2, 16),
          ([0, 130], 17, 4, 4, 16), ([127, 128, 129], 20, 8, 8, 32), ([600], 64, 8, 2, 64), ([1], 128, 4, 1, 128),
          ([700, 0, 31], 40, 16, 1, 16), ([2000], 128, 8, 2, 64), ([383, 900], 100, 3, 3, 256), ([260], 128, 32, 2, 64)]


@pytest.mark.parametrize("kv,n,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("workspace", [True, False])
def test_attention(fc, kv, n, H, Hkv, page, workspace):
    rng = np.random.default_rng(sum(kv) + n + H)
    nodes = [max(1, n - 3 * b) for b in range(len(kv))]
    s = setup(rng, kv, n, H, Hkv, page, nodes)
    masks = trees(rng, nodes, n)
    ws = fc.kv8_attn_workspace(len(kv), n, H, Hkv, "cuda") if workspace else None
    got = call(fc, s, masks, workspace=ws)
    assert fc.fc_get_error() == "FC_OK"
    ref, tol, _, _ = reference(s, masks.view(np.uint64), D ** -0.5)
    err = np.abs(num(got) - ref)
    assert np.all(err <= tol), (err - tol).max()
    for b, m in enumerate(nodes):
        assert (got[b, m:] == 0).all()
    if ws is not None:  # the workspace is fit for the next call, and results repeat
        assert torch.equal(call(fc, s, masks, workspace=ws), got)


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("new", [True, False])
def test_attention_of_many_requests_of_all_sizes(fc, new, workspace):
    """More units than CTAs: units of no rows, of 2 to 256, of no key, of new keys alone and of some blocks follow one another."""
    rng = np.random.default_rng(31 + new)
    nodes = [int(x) for x in rng.choice([0, 1, 8, 9, 31, 32, 33, 64, 65, 100, 128], 40)]
    kv = [int(x) for x in rng.choice([0, 1, 16, 40, 127, 128, 129, 256, 290], 40)]
    s = setup(rng, kv, 128, 16, 8, 16, nodes)
    masks = trees(rng, nodes, 128)
    ws = fc.kv8_attn_workspace(40, 128, 16, 8, "cuda") if workspace else None
    got = call(fc, s, masks, new=new, workspace=ws)
    assert fc.fc_get_error() == "FC_OK"
    ref, tol, _, _ = reference(s, masks.view(np.uint64), D ** -0.5, new=new)
    err = np.abs(num(got) - ref)
    assert np.all(err <= tol), (err - tol).max()
    for _ in range(3):
        assert torch.equal(call(fc, s, masks, new=new, workspace=ws), got)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (3, 4, 4), (64, 8, 2)])
def test_attention_without_new_tokens_and_causal(fc, n, H, Hkv):
    rng = np.random.default_rng(n)
    s = setup(rng, [300, 0, 45], n, H, Hkv, 32)
    got = call(fc, s, new=False, workspace=fc.kv8_attn_workspace(3, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, D ** -0.5, new=False, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol) and (got[1] == 0).all()  # no key at all: zeros
    got = call(fc, s, scale=0.05)
    ref, tol, _, _ = reference(s, None, 0.05, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)
    empty = np.zeros((3, n, (n + 63) // 64), np.int64)
    assert (call(fc, s, empty)[1] == 0).all()  # masks that leave a row nothing
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (4, 16, 4), (16, 1, 1), (2, 8, 8)])
@pytest.mark.parametrize("decay", [0.0, 1.0, 0.5])
def test_weights(fc, n, H, Hkv, decay):
    rng = np.random.default_rng(n + H)
    kv = [0, 5, 700, 64, 1500]
    nodes = [n, max(1, n - 1), n, 0, n]
    s = setup(rng, kv, n, H, Hkv, 64, nodes)
    masks = trees(rng, nodes, n)
    P = s["table"].shape[1] * 64
    ws = fc.kv8_attn_workspace(len(kv), n, H, Hkv, "cuda", P)
    before = rng.random(s["cache"][0].shape[:3]).astype(np.float32)
    weight = dev(np.full_like(before, np.nan) if decay == 0 else before)
    got = call(fc, s, masks, workspace=ws, weight=weight, decay=decay)
    assert fc.fc_get_error() == "FC_OK"
    assert torch.equal(got, call(fc, s, masks, workspace=ws))  # the output does not depend on them
    ref, tol, w, we = reference(s, masks.view(np.uint64), D ** -0.5)
    assert np.all(np.abs(num(got) - ref) <= tol)
    have, seen = num(weight), np.zeros(before.shape, bool)
    for b, k in enumerate(kv):
        i = np.arange(k)
        if nodes[b] or decay == 0:
            seen[s["table"][b][i // 64], :, i % 64] = True
        else:
            seen[s["table"][b][i // 64], :, i % 64] = True
    want = np.where(seen, decay * before.astype(np.float64) + w, before if decay else np.nan)
    bound = we + 2.0 ** -22 * np.abs(np.nan_to_num(want))
    assert np.array_equal(np.isnan(have), np.isnan(want))
    assert np.all(np.abs(np.nan_to_num(have) - np.nan_to_num(want)) <= bound)


def test_weights_need_their_workspace_and_few_rows(fc):
    rng = np.random.default_rng(2)
    s = setup(rng, [100], 1, 8, 2, 64)
    w = torch.zeros(s["cache"][0].shape[:3]).cuda()
    for ws in (None, fc.kv8_attn_workspace(1, 1, 8, 2, "cuda"), fc.kv8_attn_workspace(1, 1, 8, 2, "cuda", 64)):
        with pytest.raises(fc.FastCoderError) as e:
            call(fc, s, workspace=ws, weight=w)
        assert e.value.status == "FC_ERR_WORKSPACE"
    s = setup(rng, [100], 5, 8, 2, 64)
    with pytest.raises(fc.FastCoderError) as e:
        call(fc, s, workspace=torch.zeros(1 << 20, dtype=torch.uint8).cuda(), weight=w)
    assert e.value.status == "FC_ERR_UNSUPPORTED"


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (2, 16, 2), (40, 4, 2)])
def test_attention_scales_far_apart(fc, n, H, Hkv):
    """Blocks of very different size, zeros among them, and a row of large queries."""
    rng = np.random.default_rng(9)
    s = setup(rng, [400, 90], n, H, Hkv, 32, stale=False)
    s["cache"][3][:] = (2.0 ** rng.integers(-60, 60, s["cache"][3].shape)).astype(np.float32)
    s["cache"][2][:] = (2.0 ** rng.integers(-40, -6, s["cache"][2].shape)).astype(np.float32)
    s["cache"][1][3], s["cache"][0][4] = 0, 0
    s["q"][0, 0, 0] *= 64
    got = call(fc, s, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (4, 2, 2), (2, 16, 2), (40, 4, 2)])
@pytest.mark.parametrize("kv", [[300, 90], [3000, 17]])
def test_attention_scales_as_far_apart_as_they_may_be(fc, kv, n, H, Hkv):
    """Value scales of 2^-80 to 2^90 side by side: a row's sum and its output may be 2^170 apart."""
    rng = np.random.default_rng(19)
    s = setup(rng, kv, n, H, Hkv, 32, stale=False)
    s["cache"][3][:] = (2.0 ** rng.choice([-80, -79, 0, 60, 89, 90], s["cache"][3].shape)).astype(np.float32)
    got = call(fc, s, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
    # up to 16 rows: a weight times its value scale is fp16, its error at most 2^-36 of the row's largest (at
    # least 2^11 where a subnormal step is 2^-24), times numbers of up to 448
    for b, L in enumerate(s["kv"]):
        i = np.arange(L)
        for h in range(H):
            g = h // (H // Hkv)
            K = np.concatenate((o8.cached(s["cache"], 0, s["table"][b], L, g), num(s["k"][b, g])))
            scales = np.concatenate((s["cache"][3][s["table"][b][i // 32], g, i % 32 // 16], np.ones(n)))
            for r in range(n):
                z = K[:L + r + 1] @ num(s["q"][b, r, h]) * D ** -0.5
                p = np.exp(z - z.max())
                tol[b, r, h] += (p / p.sum() * scales[:L + r + 1]).max() * 448 * 2.0 ** -36 * (L + r + 1)
    assert np.all(np.abs(num(got) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (40, 4, 2)])
def test_attention_subnormal_and_largest_numbers(fc, n, H, Hkv):
    """Every e4m3 number: keys and values of each byte, e4m3's subnormal ones among them."""
    rng = np.random.default_rng(8)
    s = setup(rng, [400, 90], n, H, Hkv, 32, stale=False)
    for i in range(2):
        b = rng.integers(0, 254, s["cache"][i].shape).astype(np.uint8)
        b[b >= 127] += 1  # all but 0x7F and 0xFF
        b[:, 0] = (b[:, 0] & 0x80) | (b[:, 0] & 7)  # kv head 0: subnormal numbers alone
        s["cache"][i][:] = b
        s["cache"][2 + i][:] = 2.0 ** -8
        s["cache"][2 + i][:, 0] = 2.0 ** 6
    s["k"][:, 0] *= 0.1
    got = call(fc, s, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (4, 8, 2), (20, 4, 4), (128, 8, 2)])
@pytest.mark.parametrize("tiny", [0.0, 2.0 ** -40])
def test_attention_of_rows_and_keys_that_are_zero(fc, n, H, Hkv, tiny):
    """A padded batch: queries of zeros (or next to it) beside others, keys of zeros, whose blocks have the smallest
    scale, with places past the end in the same block."""
    rng = np.random.default_rng(12)
    s = setup(rng, [5, 40, 131, 300], n, H, Hkv, 16)
    for b, L in enumerate(s["kv"]):
        i = np.arange(L)
        p, o = s["table"][b][i // 16], i % 16
        zero = (i // 16) % 2 == 0
        s["cache"][0][p[zero], :, o[zero]] = 0
        s["cache"][2][p[zero], :, 0] = 2.0 ** -120
    s["q"][:, ::2] *= tiny
    s["k"][1:3] = 0
    got = call(fc, s, workspace=fc.kv8_attn_workspace(4, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (64, 4, 2)])
def test_attention_many_small_weights_beside_a_large_one(fc, n, H, Hkv):
    """One key 14 above thousands of others that together outweigh it."""
    rng = np.random.default_rng(10)
    L = 6000
    s = setup(rng, [L], n, H, Hkv, 64, stale=False)
    s["q"][:] = 0
    s["q"][..., 0] = 1
    for i in range(2):
        s["cache"][2 + i][:] = 1
    s["cache"][0][:] = 0
    page, off = s["table"][0][7], 5
    s["cache"][0][page, :, off, 0] = o8.encode(14.0)
    s["k"][:] = -30  # new tokens weigh nothing
    got = call(fc, s, scale=0.6, workspace=fc.kv8_attn_workspace(1, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, 0.6, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (64, 4, 2)])
def test_scores_that_grow_and_fall_along_the_cache(fc, n, H, Hkv):
    """Keys whose scores rise by 30 (base 2) a hundred tokens, then fall: the
    reference of a row moves many times, within blocks too."""
    rng = np.random.default_rng(13)
    L = 1500
    s = setup(rng, [L], n, H, Hkv, 64, stale=False)
    s["q"][:] = 0
    s["q"][..., 0] = 1
    s["q"][:, :, 1::2, 0] = -1  # every second head the other way round
    up = np.concatenate((np.linspace(-200, 200, 1000), np.linspace(200, 0, L - 1000)))
    i = np.arange(L)
    s["cache"][0][:] = 0
    s["cache"][2][:] = 2.0 ** 0
    s["cache"][0][s["table"][0][i // 64], :, i % 64, 0] = o8.encode(up)[:, None]
    got = call(fc, s, scale=1.0, workspace=fc.kv8_attn_workspace(1, n, H, Hkv, "cuda"))
    ref, tol, _, _ = reference(s, None, 1.0, causal=True)
    assert np.all(np.abs(num(got) - ref) <= tol)
    got = call(fc, s, scale=1.0)
    assert np.all(np.abs(num(got) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (64, 4, 2)])
def test_a_captured_call_is_good_for_other_lengths(fc, n, H, Hkv):
    """A graph of write and attention, replayed after lengths, tables and rows changed."""
    rng = np.random.default_rng(14)
    s = setup(rng, [200, 90], n, H, Hkv, 32, stale=False)
    cache = on_gpu(fc, s["cache"])
    table, kv, q, k, v = dev(s["table"]), dev(s["kv"]), s["q"].cuda(), s["k"].cuda(), s["v"].cuda()
    ws, out = fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"), torch.empty_like(q)
    slot = torch.full((2,), -1, dtype=torch.int32).cuda()
    rows = [torch.zeros(2, Hkv, D, dtype=torch.bfloat16).cuda() for _ in range(2)]

    def step():
        fc.fc_kv8_write(cache, rows[0], rows[1], slot)
        fc.fc_kv8_attn(q, cache, table, kv, k, v, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()  # captured on another stream than the tensors'
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for kv_new in ([37, 90], [0, 1], [199, 64]):
        s["kv"] = np.array(kv_new, np.int32)
        x = [bf(rng, 2, Hkv, D) for _ in range(2)]
        at = np.array([s["table"][b][L // 32] * 32 + L % 32 for b, L in enumerate(kv_new)], np.int32)
        for d, h in zip(rows + [slot, kv], x + [torch.from_numpy(at), torch.from_numpy(s["kv"] + 1)]):
            d.copy_(h)
        graph.replay()
        o8.write(s["cache"], num(x[0]), num(x[1]), at)
        s["kv"] = s["kv"] + 1
        ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
        assert np.all(np.abs(num(out) - ref) <= tol)
    assert fc.fc_get_error() == "FC_OK"


def test_attention_on_two_streams_at_once(fc):
    """Two calls that overlap, with a workspace each."""
    rng = np.random.default_rng(15)
    for n, H, Hkv in ((1, 16, 4), (48, 8, 4)):
        s = setup(rng, [3000, 700], n, H, Hkv, 64)
        ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
        cache, table, kv = on_gpu(fc, s["cache"]), dev(s["table"]), dev(s["kv"])
        q, k, v = s["q"].cuda(), s["k"].cuda(), s["v"].cuda()
        streams = [torch.cuda.Stream() for _ in range(2)]
        ws = [fc.kv8_attn_workspace(2, n, H, Hkv, "cuda") for _ in range(2)]
        outs = [torch.empty_like(q) for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(5):
            for st, w, o in zip(streams, ws, outs):
                with torch.cuda.stream(st):
                    fc.fc_kv8_attn(q, cache, table, kv, k, v, out=o, workspace=w)
        torch.cuda.synchronize()
        for o in outs:
            assert np.all(np.abs(num(o) - ref) <= tol)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (3, 4, 1), (64, 4, 2)])
def test_not_finite_values_reach_only_rows_that_see_them(fc, n, H, Hkv):
    rng = np.random.default_rng(11)
    s = setup(rng, [200, 70, 90], n, H, Hkv, 32)
    masks = trees(rng, [n] * 3, n)
    ws = fc.kv8_attn_workspace(3, n, H, Hkv, "cuda")
    clean = call(fc, s, masks, workspace=ws)
    s["cache"][2][s["table"][0][1], 0, 1] = np.nan  # request 0, kv head 0: keys that stand for NaN
    s["cache"][3][s["table"][1][0], Hkv - 1, 0] = np.nan  # request 1, the last kv head: values
    s["v"][2, 0, n - 1, 3] = float("inf")  # request 2, head 0: the last new token's value
    s["k"][2, 0, n - 1, 4] = float("nan")
    got = call(fc, s, masks, workspace=ws)
    G = H // Hkv
    want = torch.zeros(3, n, H, dtype=torch.bool)
    want[0, :, :G] = True
    want[1, :, -G:] = True
    want[2, :, :G] = torch.from_numpy((masks.view(np.uint64)[2, :, (n - 1) // 64] >> np.uint64((n - 1) % 64)) & np.uint64(1) == 1)[:, None]
    nan = got.isnan().all(-1).cpu()
    assert torch.equal(nan, want), (nan != want).nonzero()
    assert torch.equal(got[~want.cuda()], clean[~want.cuda()])


def test_bad_pages_and_lengths_are_recorded(fc):
    rng = np.random.default_rng(12)
    for n, H, Hkv in ((1, 8, 2), (40, 4, 2)):
        s = setup(rng, [100, 60, 80], n, H, Hkv, 32)
        ws = fc.kv8_attn_workspace(3, n, H, Hkv, "cuda")
        masks = trees(rng, [n] * 3, n)
        clean = call(fc, s, masks, workspace=ws)
        s["kv"][1] = 100000
        s["nodes"][2] = n + 1
        got = call(fc, s, masks, workspace=ws)
        assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
        assert (got[1:] == 0).all() and torch.equal(got[0], clean[0])
        s = setup(rng, [100, 60, 80], n, H, Hkv, 32, stale=False)
        whole = {k: v for k, v in s.items()}
        s["table"] = s["table"].copy()
        s["table"][0, 1] = 1 << 20  # its 32 keys are left out
        got = call(fc, s, masks, workspace=ws)
        assert fc.fc_get_error() == "FC_ERR_INVALID_ARG"
        short = dict(whole, table=np.concatenate((whole["table"][:, :1], whole["table"][:, 2:]), 1), kv=np.array([68, 0, 0], np.int32))
        ref, tol, _, _ = reference(short, masks.view(np.uint64), D ** -0.5)
        assert np.all(np.abs(num(got)[0] - ref[0]) <= tol[0])


# ------------------------------------------------------------------ eviction
@pytest.mark.parametrize("kv,keep,recent,H,page", [([20], [7], 0, 1, 16), ([64, 30], [40, 40], 8, 2, 32), ([1000, 333, 70], [500, 300, 1], 50, 3, 64),
                                                   ([100], [99], 100, 2, 16), ([300, 300], [16, 0], 5, 2, 128), ([2100], [2047], 64, 1, 256),
                                                   ([50, 0, 49], [48, 48, 48], 1000, 2, 16), ([4096, 4000], [4095, 2000], 0, 1, 256),
                                                   ([8192, 5], [4096, 5], 33, 1, 128), ([9000, 16384], [8999, 100], 64, 1, 64), ([17000], [8499], 100, 1, 256)])
def test_evict(fc, kv, keep, recent, H, page):
    rng = np.random.default_rng(sum(kv) + recent)
    s = setup(rng, kv, 1, H, H, page, stale=False)
    n_pages = len(s["cache"][0])
    w = np.where(rng.random((n_pages, H, page)) < 0.3, 0.25, np.exp(rng.standard_normal((n_pages, H, page)))).astype(np.float32)  # many ties
    w[rng.random(w.shape) < 0.01] = np.nan
    w[rng.random(w.shape) < 0.01] = np.inf
    w[rng.random(w.shape) < 0.02] = -0.0
    born = np.zeros((n_pages, H, page), np.int32)
    for b, k in enumerate(kv):
        for h in range(H):
            i = np.arange(k)
            born[s["table"][b][i // page], h, i % page] = rng.permutation(k) + 11
    w0 = np.full(w.shape, -5, np.float32)
    b0 = np.full(born.shape, -6, np.int32)
    cap = max([k for k, n in zip(keep, kv) if k < n] + [1]) + 3
    got = on_gpu(fc, s["cache"])
    t_in, t_out = fc.Kv8Track(dev(w), dev(born)), fc.Kv8Track(dev(w0), dev(b0))
    args = (dev(s["table"]), dev(s["kv"]), dev(np.array(keep, np.int32)), recent, t_in, t_out)
    frm = fc.fc_kv8_evict(got, *args, cap=cap)
    assert fc.fc_get_error() == "FC_OK"
    ref = o8.evict(s["cache"], s["table"], s["kv"], keep, recent, [w, born], [w0, b0], cap)
    assert np.array_equal(frm.cpu().numpy(), ref)
    same_cache(got, s["cache"])
    assert np.array_equal(t_out.weight.cpu().numpy(), w0, equal_nan=True) and np.array_equal(t_out.born.cpu().numpy(), b0)
    assert np.array_equal(t_in.weight.cpu().numpy(), w, equal_nan=True)


def test_a_captured_eviction_is_good_for_other_lengths(fc):
    """A graph of an eviction, captured on another stream, replayed over other caches, lengths and budgets, zero and nothing to do among them."""
    H, page, cap = 2, 32, 200
    kv = [500, 300]
    s = setup(np.random.default_rng(3), kv, 1, H, H, page, stale=False)
    got = on_gpu(fc, s["cache"])
    tracks = [fc.Kv8Track.empty(got) for _ in range(2)]
    table, lens, keep = dev(s["table"]), dev(s["kv"]), dev(np.array([200, 100], np.int32))
    out = torch.empty((2, H, cap), dtype=torch.int32, device="cuda")
    ws = fc.kv8_evict_workspace(2, H, cap, "cuda")
    run = lambda: fc.fc_kv8_evict(got, table, lens, keep, 10, *tracks, out=out, workspace=ws)
    run()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        run()
    for i, (L, K) in enumerate((([500, 300], [199, 1]), ([0, 17], [0, 16]), ([480, 290], [0, 290]), ([33, 256], [32, 128]))):
        rng = np.random.default_rng(40 + i)
        cache = random_cache(rng, got.n_pages, H, page)
        w = np.exp(rng.standard_normal((got.n_pages, H, page))).astype(np.float32)
        born = rng.permutation(w.size).reshape(w.shape).astype(np.int32)
        w0, b0 = np.zeros_like(w), np.zeros_like(born)
        for d, h in zip((got.k_codes, got.v_codes, got.k_scale, got.v_scale, tracks[0].weight, tracks[0].born, tracks[1].weight, tracks[1].born, lens, keep),
                        cache + [w, born, w0, b0, np.array(L, np.int32), np.array(K, np.int32)]):
            d.copy_(torch.from_numpy(h))
        graph.replay()
        ref = o8.evict(cache, s["table"], np.array(L), K, 10, [w, born], [w0, b0], cap)
        assert np.array_equal(out.cpu().numpy(), ref)
        same_cache(got, cache)
        assert np.array_equal(tracks[1].weight.cpu().numpy(), w0) and np.array_equal(tracks[1].born.cpu().numpy(), b0)
    assert fc.fc_get_error() == "FC_OK"


def test_evict_long_request(fc):
    """More tokens than the keys' place in shared memory holds."""
    rng = np.random.default_rng(20)
    L, K, page = 60000, 41000, 256
    s = setup(rng, [L], 1, 1, 1, page, stale=False)
    n_pages = len(s["cache"][0])
    w = (rng.integers(0, 5000, (n_pages, 1, page)) / 64).astype(np.float32)  # ties
    born = np.zeros((n_pages, 1, page), np.int32)
    i = np.arange(L)
    born[s["table"][0][i // page], 0, i % page] = rng.permutation(L)
    w0, b0 = np.zeros_like(w), np.zeros_like(born)
    got = on_gpu(fc, s["cache"])
    t_out = fc.Kv8Track(dev(w0), dev(b0))
    frm = fc.fc_kv8_evict(got, dev(s["table"]), dev(s["kv"]), dev(np.array([K], np.int32)), 3000, fc.Kv8Track(dev(w), dev(born)), t_out, cap=K)
    ref = o8.evict(s["cache"], s["table"], s["kv"], [K], 3000, [w, born], [w0, b0], K)
    assert np.array_equal(frm.cpu().numpy(), ref)
    same_cache(got, s["cache"])
    assert np.array_equal(t_out.weight.cpu().numpy(), w0) and np.array_equal(t_out.born.cpu().numpy(), b0)


def test_evict_leaves_what_it_refuses(fc):
    rng = np.random.default_rng(21)
    kv = [60, 60, 60, 60]
    s = setup(rng, kv, 1, 2, 2, 16, stale=False)
    n_pages = len(s["cache"][0])
    w, born = rng.random((n_pages, 2, 16)).astype(np.float32), rng.permutation(n_pages * 32).reshape(n_pages, 2, 16).astype(np.int32)
    good = [s["table"][3].copy(), [c.copy() for c in s["cache"]]]
    s["kv"][0] = -1
    s["table"][1, 2] = n_pages  # a page outside the pool
    keep = np.array([10, 10, 50, 20], np.int32)  # request 2: more than cap
    got = on_gpu(fc, s["cache"])
    w0, b0 = np.zeros_like(w), np.zeros_like(born)
    t_out = fc.Kv8Track(dev(w0), dev(b0))
    frm = fc.fc_kv8_evict(got, dev(s["table"]), dev(s["kv"]), dev(keep), 4, fc.Kv8Track(dev(w), dev(born)), t_out, cap=30)
    assert fc.fc_get_error() == "FC_ERR_CAPACITY" and (frm[:3] == -1).all()
    ref = o8.evict(good[1], good[0][None], [60], [20], 4, [w, born], [w0, b0], 30)
    assert np.array_equal(frm[3:].cpu().numpy(), ref)
    same_cache(got, good[1])
    assert np.array_equal(t_out.weight.cpu().numpy(), w0)


def test_pages_past_four_gigabytes(fc):
    """The last pages of a pool of 5.2 GB of keys and as much of values do as those of a small one."""
    rng = np.random.default_rng(17)
    P, H, page = 40000, 8, 128
    s = setup(rng, [700, 129, 0], 40, 16, H, page, stale=False)
    few = on_gpu(fc, s["cache"])
    n = few.n_pages
    big = fc.Kv8Cache.empty(P, H, page)
    last = slice(P - n, P)
    for x in ("k_codes", "v_codes", "k_scale", "v_scale"):
        getattr(big, x)[last].copy_(getattr(few, x))
    tables = [dev(s["table"]), dev(np.where(s["table"] >= 0, s["table"] + P - n, s["table"]).astype(np.int32))]
    tracks = [[fc.Kv8Track.empty(c) for _ in range(2)] for c in (few, big)]
    born = rng.permutation(n * H * page).reshape(n, H, page).astype(np.int32)
    tracks[0][0].born.copy_(dev(born))
    tracks[1][0].born[last].copy_(dev(born))
    kv, q, k, v = dev(s["kv"]), s["q"].cuda(), s["k"].cuda(), s["v"].cuda()
    keep = dev(np.array([300, 128, 0], np.int32))
    slots = torch.from_numpy(s["table"][[0, 0, 1]][:, 0] * page + np.array([1, 30, 3])).int().cuda()
    got = []
    for c, table, (now, then), off in zip((few, big), tables, tracks, (0, (P - n) * page)):
        ws = fc.kv8_attn_workspace(3, 40, 16, H, "cuda")
        out = [fc.fc_kv8_attn(q, c, table, kv, k, v, workspace=ws)]
        ws = fc.kv8_attn_workspace(3, 1, 16, H, "cuda", table.shape[1] * page)
        out.append(fc.fc_kv8_attn(q[:, :1].contiguous(), c, table, kv, workspace=ws, weight=now.weight))
        out += [now.weight[c.n_pages - n:].clone(), fc.fc_kv8_evict(c, table, kv, keep, 20, now, then, cap=300)]
        fc.fc_kv8_write(c, k[:, :, 0], v[:, :, 0], slots + off, track=then, pos=slots)
        out += [*fc.fc_kv8_read(c, slots + off), then.weight[c.n_pages - n:], then.born[c.n_pages - n:]]
        got.append(out + [getattr(c, x)[c.n_pages - n:] for x in ("k_codes", "v_codes", "k_scale", "v_scale")])
    assert fc.fc_get_error() == "FC_OK"
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert got[1][2].any() and (got[1][3] >= 0).any() and got[1][4].any()


def test_arguments_that_do_not_fit_are_refused(fc):
    """Before anything runs: ranks, a missing partner, numbers past 32 bits."""
    bf = torch.bfloat16
    new = lambda *s: torch.zeros(s, dtype=bf, device="cuda")
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q, k, w, pos = new(1, 2, 4, 128), new(1, 2, 2, 128), new(128), ints(1, 2)
    for bad in ((q[0], k, None), (q, k[0], None), (q, k[0, 0, 0], None), (q, k, new(1, 2, 2, 64)), (q, k[..., :64], None)):
        with pytest.raises(ValueError):
            fc.fc_qk_norm_rope(*bad, w, w, pos)
    with pytest.raises(TypeError):
        fc.fc_qk_norm_rope(q, k, [1], w, w, pos)
    cache = fc.Kv8Cache.empty(2, 2, 16)
    table, kv_len = ints(1, 2), ints(1)
    kn = new(1, 2, 2, 128)
    for pair in ((kn, None), (None, kn)):
        with pytest.raises(ValueError):
            fc.fc_kv8_attn(q, cache, table, kv_len, *pair)
    now, then = fc.Kv8Track.empty(cache), fc.Kv8Track.empty(cache)
    for recent in (-1, -(1 << 32), (1 << 22) + 1, 1 << 32):
        with pytest.raises(fc.FastCoderError):
            fc.fc_kv8_evict(cache, table, kv_len, kv_len, recent, now, then, cap=4)
    with pytest.raises(fc.FastCoderError):  # the same arrays in and out
        fc.fc_kv8_evict(cache, table, kv_len, kv_len, 0, now, now, cap=4)


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (3, 4, 1), (16, 1, 1)])
@pytest.mark.parametrize("kv", [[200, 70], [9000, 40]])
def test_weights_do_not_depend_on_new_values(fc, kv, n, H, Hkv):
    """New tokens whose values are not finite: the rows that see them are NaN, the weights of the cached tokens what
    they are without, bit for bit."""
    rng = np.random.default_rng(21)
    s = setup(rng, kv, n, H, Hkv, 32)
    masks = trees(rng, [n] * 2, n)
    ws = fc.kv8_attn_workspace(2, n, H, Hkv, "cuda", s["table"].shape[1] * 32)
    before = dev(rng.random(s["cache"][0].shape[:3]).astype(np.float32))
    clean, weight = before.clone(), before.clone()
    ok = call(fc, s, masks, workspace=ws, weight=clean, decay=0.5)
    s["v"][0, Hkv - 1, 0, 5] = float("nan")  # the root, which every row sees
    s["v"][1, 0, n - 1, 3] = float("inf")
    got = call(fc, s, masks, workspace=ws, weight=weight, decay=0.5)
    assert torch.equal(weight, clean)
    want = torch.zeros(2, n, H, dtype=torch.bool)
    want[0, :, -(H // Hkv):] = True
    want[1, :, :H // Hkv] = torch.from_numpy((masks[1, :, 0] >> (n - 1)) & 1 == 1)[:, None]
    assert torch.equal(got.isnan().all(-1).cpu(), want) and torch.equal(got[~want.cuda()], ok[~want.cuda()])
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (3, 4, 1), (16, 1, 1)])
@pytest.mark.parametrize("kv", [[200, 70], [9000, 40]])
def test_weights_beside_cached_values_that_stand_for_nan(fc, kv, n, H, Hkv):
    """Blocks whose value scale is NaN: the rows of their request and head are NaN, the weights those of the scores,
    which spread far here (queries times 2)."""
    rng = np.random.default_rng(22)
    s = setup(rng, kv, n, H, Hkv, 32)
    s["q"] = s["q"] * 2
    ws = fc.kv8_attn_workspace(2, n, H, Hkv, "cuda", s["table"].shape[1] * 32)
    _, _, want, bound = reference(s, None, D ** -0.5, causal=True)
    for t in range(0, kv[0] // 32, 3):
        s["cache"][3][s["table"][0][t], 0, t % 2] = np.nan
    s["cache"][3][s["table"][1][0], Hkv - 1, 1] = np.nan
    weight = torch.zeros(s["cache"][0].shape[:3]).cuda()
    got = call(fc, s, workspace=ws, weight=weight, decay=0.0)
    assert np.all(np.abs(num(weight) - want) <= bound)
    G = H // Hkv
    nan = got.isnan().all(-1)
    assert nan[0, :, :G].all() and nan[1, :, -G:].all() and nan.sum() == 2 * n * G
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("apart", [1, 16, 30, 31, 32])
@pytest.mark.parametrize("lead", [0, 1, 15, 16, 31])
@pytest.mark.parametrize("many", [False, True])
def test_write_of_rows_of_a_block_that_stand_apart(fc, apart, lead, many):
    """Two rows of one block with rows between them that are left out or go to other blocks."""
    rng = np.random.default_rng(apart + lead)
    H, page = 4, 32
    slot = np.full(lead + apart + 40, -1, np.int32)
    slot[lead], slot[lead + apart] = 3 * page + 18, 3 * page + 21
    if apart > 2:
        slot[lead + 1], slot[lead + apart - 1] = 0, page + 16
    if many:  # enough rows for a warp to take several
        slot = np.concatenate([np.where(slot < 0, -1, slot + 4 * page * i) for i in range(60)]).astype(np.int32)
    cache = random_cache(rng, 4 * (60 if many else 1), H, page)
    got = on_gpu(fc, cache)
    track = fc.Kv8Track(torch.full(cache[0].shape[:3], 3.5).cuda(), torch.full(cache[0].shape[:3], -7, dtype=torch.int32).cuda())
    rt = [track.weight.cpu().numpy(), track.born.cpu().numpy()]
    x, pos = bf(rng, len(slot), H, D), rng.integers(0, 99, len(slot)).astype(np.int32)
    fc.fc_kv8_write(got, x.cuda(), x.cuda(), dev(slot), track=track, pos=dev(pos))
    o8.write(cache, num(x), num(x), slot, None, rt, pos)
    same_cache(got, cache)
    assert np.array_equal(track.weight.cpu().numpy(), rt[0]) and np.array_equal(track.born.cpu().numpy(), rt[1])
    assert fc.fc_get_error() == "FC_OK"


SIZES_APART = [(-60, 0), (-70, 68), (-112, 90), (-20, -60), (74, -70), (110, -60), (20, 88)]


def sized(rng, kv, n, H, Hkv, q_exp, k_exp):
    """Queries times 2^q_exp, keys, cached and new, times 2^k_exp, and the scale that takes both back."""
    s = setup(rng, kv, n, H, Hkv, 32, stale=False)
    s["q"] = (s["q"].float() * 2.0 ** q_exp).bfloat16()
    s["k"] = (s["k"].float() * 2.0 ** k_exp).bfloat16()
    s["cache"][2] *= np.float32(2.0 ** k_exp)
    return s, D ** -0.5 * 2.0 ** -(q_exp + k_exp)


@pytest.mark.parametrize("q_exp,k_exp", SIZES_APART)
@pytest.mark.parametrize("n,H,Hkv", [(20, 4, 4), (40, 4, 2)])
def test_trees_of_tiny_and_large_queries_and_keys(fc, n, H, Hkv, q_exp, k_exp):
    """Scores of some units, whatever makes them up."""
    s, scale = sized(np.random.default_rng(23), [300, 45], n, H, Hkv, q_exp, k_exp)
    ref, tol, _, _ = reference(s, None, scale, causal=True)
    got = call(fc, s, scale=scale, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    assert np.all(np.abs(num(got) - ref) <= tol)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("q_exp,k_exp", SIZES_APART)
@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (4, 16, 4)])
def test_few_rows_of_tiny_and_large_queries_and_keys(fc, n, H, Hkv, q_exp, k_exp):
    s, scale = sized(np.random.default_rng(24), [300, 45], n, H, Hkv, q_exp, k_exp)
    ref, tol, _, _ = reference(s, None, scale, causal=True)
    got = call(fc, s, scale=scale, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    assert np.all(np.abs(num(got) - ref) <= tol)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 2), (2, 16, 2), (40, 4, 2)])
def test_scores_of_zero_between_large_queries_and_keys(fc, n, H, Hkv):
    """Queries of 2^100 in one half of the dimensions, keys of 2^60 in the other: every score is 0, every weight the same."""
    s = setup(np.random.default_rng(25), [300, 45], n, H, Hkv, 32, stale=False)
    s["q"][..., 64:] = 0
    s["k"][..., :64] = 0
    s["cache"][0][..., :64] = 0
    zero = dict(s, q=torch.zeros_like(s["q"]))
    ref, tol, _, _ = reference(zero, None, D ** -0.5, causal=True)
    s["q"] = (s["q"].float() * 2.0 ** 100).bfloat16()
    s["k"] = (s["k"].float() * 2.0 ** 20).bfloat16()
    s["cache"][2] *= np.float32(2.0 ** 60)
    got = call(fc, s, workspace=fc.kv8_attn_workspace(2, n, H, Hkv, "cuda"))
    assert np.all(np.abs(num(got) - ref) <= tol)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("L", [30, 34, 500])
def test_evict_the_last_block_counts_up_to_the_old_length(fc, L):
    """20 tokens stay; place 17 takes one, and the scale of its block is the one for its 16 places below the old
    length, an evicted token's large numbers at place 25 among them."""
    rng = np.random.default_rng(L)
    H, page, K = 2, 16, 20
    s = setup(rng, [L], 1, H, H, page, stale=False)
    at = lambda i: (s["table"][0][i // page], slice(None), i % page)
    for i in range(2):
        s["cache"][i][at(25)] = o8.encode(448.0)
        s["cache"][2 + i][s["table"][0][1]] = 2.0 ** 10  # place 25's block
    w, born = np.zeros(s["cache"][0].shape[:3], np.float32), np.zeros(s["cache"][0].shape[:3], np.int32)
    for i in range(L):
        w[at(i)], born[at(i)] = (2.0 if i < K and i != 17 or i == L - 1 else 1 / (i + 2)), i
    w0, b0 = np.zeros_like(w), np.zeros_like(born)
    got = on_gpu(fc, s["cache"])
    t_out = fc.Kv8Track(dev(w0), dev(b0))
    frm = fc.fc_kv8_evict(got, dev(s["table"]), dev(s["kv"]), dev(np.array([K], np.int32)), 0, fc.Kv8Track(dev(w), dev(born)), t_out, cap=K)
    assert (frm[0, :, 17] == L - 1).all() and (frm >= 0).sum() == H
    o8.evict(s["cache"], s["table"], s["kv"], [K], 0, [w, born], [w0, b0], K)
    same_cache(got, s["cache"])
    assert (got.k_scale[int(s["table"][0][1])] == 2.0 ** 10).all() and fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("pages", [300, 3000])
def test_weights_and_evictions_under_a_wide_table(fc, pages):
    """Short requests under tables for 19200 and 192000 tokens, as wide as their longest allowed request."""
    rng = np.random.default_rng(26)
    kv, n, H, Hkv, page, K = [700, 0, 333], 2, 8, 2, 64, 200
    s = setup(rng, kv, n, H, Hkv, page)
    s["table"] = np.concatenate((s["table"], np.full((3, pages - s["table"].shape[1]), -9, np.int32)), 1)
    masks = trees(rng, [n] * 3, n)
    weight, born = dev(np.zeros(s["cache"][0].shape[:3], np.float32)), np.zeros(s["cache"][0].shape[:3], np.int32)
    for b, L in enumerate(kv):
        i = np.arange(L)
        born[s["table"][b][i // page], :, i % page] = i[:, None]
    got = call(fc, s, masks, workspace=fc.kv8_attn_workspace(3, n, H, Hkv, "cuda", pages * page), weight=weight, decay=1.0)
    ref, tol, want, bound = reference(s, masks.view(np.uint64), D ** -0.5)
    assert np.all(np.abs(num(got) - ref) <= tol) and np.all(np.abs(num(weight) - want) <= bound)
    w = weight.cpu().numpy()
    w0, b0 = np.zeros_like(w), np.zeros_like(born)
    cache, t_out = on_gpu(fc, s["cache"]), fc.Kv8Track(dev(w0), dev(b0))
    frm = fc.fc_kv8_evict(cache, dev(s["table"]), dev(s["kv"]), dev(np.full(3, K, np.int32)), 16, fc.Kv8Track(weight, dev(born)), t_out, cap=K)
    assert np.array_equal(frm.cpu().numpy(), o8.evict(s["cache"], s["table"], kv, [K] * 3, 16, [w, born], [w0, b0], K))
    same_cache(cache, s["cache"])
    assert np.array_equal(t_out.weight.cpu().numpy(), w0) and np.array_equal(t_out.born.cpu().numpy(), b0)
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("chunk", [4, 48, 128])
def test_prompts_in_chunks(fc, chunk):
    """Prompts taken in by chunks: attention over what is cached, causal among the new, then the chunk is written.  Each
    chunk against the oracle over the cache as it is."""
    rng = np.random.default_rng(27)
    H, Hkv, page, lens = 8, 4, 32, [300, 131, 17]
    B, most = len(lens), 10
    n_pages = B * most
    table = rng.permutation(n_pages).astype(np.int32).reshape(B, most)
    cache = [np.zeros((n_pages, Hkv, page, D), np.uint8) for _ in range(2)] + [np.ones((n_pages, Hkv, page // 16), np.float32) for _ in range(2)]
    held = on_gpu(fc, cache)
    ws = fc.kv8_attn_workspace(B, chunk, H, Hkv, "cuda")
    for at in range(0, max(lens), chunk):
        kv = np.minimum(at, lens).astype(np.int32)
        nodes = np.clip(np.array(lens) - at, 0, chunk).astype(np.int32)
        s = dict(kv=kv, nodes=nodes, table=table, cache=cache, q=bf(rng, B, chunk, H, D), k=bf(rng, B, Hkv, chunk, D), v=bf(rng, B, Hkv, chunk, D))
        k, v = s["k"].cuda(), s["v"].cuda()
        got = fc.fc_kv8_attn(s["q"].cuda(), held, dev(table), dev(kv), k, v, None, dev(nodes), workspace=ws)
        ref, tol, _, _ = reference(s, None, D ** -0.5, causal=True)
        assert np.all(np.abs(num(got) - ref) <= tol)
        p = at + np.arange(chunk)
        slot = np.where(np.arange(chunk) < nodes[:, None], table[:, np.minimum(p // page, most - 1)] * page + p % page, -1).astype(np.int32).reshape(-1)
        fc.fc_kv8_write(held, k.transpose(1, 2), v.transpose(1, 2), dev(slot))
        o8.write(cache, *(num(x).transpose(0, 2, 1, 3).reshape(-1, Hkv, D) for x in (s["k"], s["v"])), slot)
        same_cache(held, cache)
    assert fc.fc_get_error() == "FC_OK"


def test_tracks_change_places_after_an_eviction(fc):
    """Attention with weights, writes, an eviction whose output track is the next steps': three times over."""
    rng = np.random.default_rng(28)
    B, n, H, Hkv, page, K = 2, 1, 4, 2, 16, 40
    s = setup(rng, [70, 41], n, H, Hkv, page, stale=False)
    s["table"] = np.arange(2 * 6, dtype=np.int32).reshape(2, 6)
    s["cache"] = random_cache(rng, 12, Hkv, page)
    cache, table = on_gpu(fc, s["cache"]), dev(s["table"])
    now, then = fc.Kv8Track.empty(cache), fc.Kv8Track.empty(cache)
    t_now, t_then = ([x.weight.cpu().numpy().copy(), x.born.cpu().numpy().copy()] for x in (now, then))
    ws = fc.kv8_attn_workspace(B, n, H, Hkv, "cuda", 6 * page)
    born = 1000
    for _ in range(3):
        for _ in range(20):
            s["k"], s["v"], s["q"] = bf(rng, B, Hkv, n, D), bf(rng, B, Hkv, n, D), bf(rng, B, n, H, D)
            k, v = s["k"].cuda(), s["v"].cuda()
            got = fc.fc_kv8_attn(s["q"].cuda(), cache, table, dev(s["kv"]), k, v, workspace=ws, weight=now.weight, decay=0.9)
            ref, tol, want, bound = reference(s, None, D ** -0.5, causal=True)
            assert np.all(np.abs(num(got) - ref) <= tol)
            for b in range(B):  # the tokens' alone decay
                i = np.arange(s["kv"][b])
                p, o = s["table"][b][i // page], i % page
                new = num(now.weight)[p, :, o]
                assert np.all(np.abs(new - (0.9 * t_now[0][p, :, o] + want[p, :, o])) <= bound[p, :, o] + 2.0 ** -22 * new)
            t_now[0] = now.weight.cpu().numpy().copy()
            slot = np.array([s["table"][b][L // page] * page + L % page for b, L in enumerate(s["kv"])], np.int32)
            pos = np.full(B, born, np.int32)
            fc.fc_kv8_write(cache, k.transpose(1, 2), v.transpose(1, 2), dev(slot), track=now, pos=dev(pos))
            o8.write(s["cache"], num(s["k"])[:, :, 0], num(s["v"])[:, :, 0], slot, None, t_now, pos)
            s["kv"], born = s["kv"] + 1, born + 1
        fc.fc_kv8_evict(cache, table, dev(s["kv"]), dev(np.full(B, K, np.int32)), 8, now, then, cap=K)
        o8.evict(s["cache"], s["table"], s["kv"], [K] * B, 8, t_now, t_then, K)
        same_cache(cache, s["cache"])
        now, then, t_now, t_then = then, now, t_then, t_now
        s["kv"] = np.minimum(s["kv"], K).astype(np.int32)
        for x, y in zip((now.weight, now.born), t_now):
            for b in range(B):
                i = np.arange(K)
                assert np.array_equal(x.cpu().numpy()[s["table"][b][i // page], :, i % page], y[s["table"][b][i // page], :, i % page])
    assert fc.fc_get_error() == "FC_OK"


@pytest.mark.parametrize("dim", [16, 64, 128, 256, 512])
@pytest.mark.parametrize("exp,eps", [(70, 1e-6), (110, 1e-6), (125, 0.0), (-70, 0.0), (-110, 0.0), (-70, 1e-6), (-45, 1e-26), (0, 1e30)])
def test_norm_rope_of_large_and_small_rows(fc, dim, exp, eps):
    """Rows whose squares pass fp32's range, beside ordinary ones and rows of zeros."""
    rng = np.random.default_rng(dim)
    q, k = bf(rng, 2, 5, 3, dim), bf(rng, 2, 5, 2, dim)
    q[:, ::2], k[:, 1, 1] = (q[:, ::2].float().clamp(-2, 2) * 2.0 ** exp).bfloat16(), (k[:, 1, 1].float().clamp(-2, 2) * 2.0 ** exp).bfloat16()
    if eps:
        q[1, 1, 1] = 0
    w, pos = bf(rng, dim), rng.integers(0, 9, (2, 5)).astype(np.int32)
    got = fc.fc_qk_norm_rope(q.cuda(), k.cuda(), None, w.cuda(), w.cuda(), dev(pos), 1e4, eps)
    for x, y, turn in ((q, got[0], False), (k, got[1], True)):
        ref, mag = o8.norm_rope(num(x), num(w), pos.astype(np.float64), 1e4, eps)
        if turn:
            ref, mag = ref.transpose(0, 2, 1, 3), mag.transpose(0, 2, 1, 3)
        assert np.all(np.abs(num(y) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * mag + 2.0 ** -133)
    assert fc.fc_get_error() == "FC_OK"
