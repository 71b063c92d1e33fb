"""The operators of serving in four bits: their cases, their plain forms in torch and their definitions in 64 bits.

Four operators, two of them with a partner that undoes them:

* pages   - block tables and slot maps of a paged cache from request lengths (fc_kv_pages_plan);
* write   - keys and values quantised into the pages of a 4-bit cache, and read back (fc_kv4_write, fc_kv4_read);
* attn    - attention of one token, or of a draft tree's tokens, over that cache (fc_kv4_attn);
* matvec  - products of a few rows with weights in 4 bits under group scales (fc_w4_matvec).

Formulas.  A row x of D = 128 values (or a group of g weights of one column) is held as whole numbers c in -7..7 and one
scale: s = bf16(max|x| / 7), c = clamp(rint(x / s), -7, 7), ties to even, all zeros where s = 0; it stands for c * s.  In
memory a number is c + 8, two to a byte, the first in the low half.

``own`` false: elementary torch operations in 32 bits.  ``own`` true: the framework's calls.
"""
import math

import torch

own = False

D = 128
DEV = "cuda"


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one decoding step of 32 requests, one token each: the call sits before every step, so its latency counts
        dict(name="pages decode b32", op="pages", batch=32, new=1, kv=16384, page=64),
        # a step that admits many prompts of ragged lengths beside running requests
        dict(name="pages prompts b1000", op="pages", batch=1000, new=487, kv=4096, page=16),
        # the tokens of one decoding step: 32 rows, keys and values cut out of one fused projection
        dict(name="write decode 32x8", op="write", rows=32, heads=8, page=64, fused=True, skip=False),
        # prompts: 65,000 rows at once, some of them padding
        dict(name="write prompts 65000x8", op="write", rows=65000, heads=8, page=64, fused=False, skip=True),
        # one short request, one token: latency
        dict(name="attn token b1 kv500", op="attn", batch=1, nodes=1, heads=32, kv_heads=8, kv=500, page=64, ragged=False),
        # the step loop's shape (32 requests, 32 / 8 heads, 16384 keys), one token each: the cache read bounds it
        dict(name="attn token b32 kv16384", op="attn", batch=32, nodes=1, heads=32, kv_heads=8, kv=16384, page=64, ragged=False),
        # one request with a long context: the keys have to be split over the whole GPU
        dict(name="attn token b1 kv131071", op="attn", batch=1, nodes=1, heads=32, kv_heads=8, kv=131071, page=128, ragged=False),
        # 16 requests of ragged lengths, 32 heads without sharing, draft trees of 64 nodes
        dict(name="attn tree64 b16 mha", op="attn", batch=16, nodes=64, heads=32, kv_heads=32, kv=4096, page=64, ragged=True),
        # the step loop's whole shape: trees of 128 nodes over 16384 keys; the matrix products bound it
        dict(name="attn tree128 b32", op="attn", batch=32, nodes=128, heads=32, kv_heads=8, kv=16384, page=64, ragged=False),
        # an attention projection of a small decoder, one token: latency
        dict(name="matvec 1x2048x2048", op="matvec", rows=1, k=2048, n=2048, group=128),
        # the vocabulary projection of the same decoder, one token: the weights' read
        dict(name="matvec 1x2048x32256", op="matvec", rows=1, k=2048, n=32256, group=128),
        # a large projection for the 16 tokens of a small draft tree
        dict(name="matvec 16x8192x28672", op="matvec", rows=16, k=8192, n=28672, group=64),
    ]


def log_int(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "write", "attn", "attn", "matvec"])
    if op == "pages":
        batch = log_int(rng, 1, 2000)
        return dict(op=op, batch=batch, new=log_int(rng, 1, max(1, min(4000, 400000 // batch))), kv=log_int(rng, 1, 30000),
                    page=rng.choice([16, 32, 64, 128]))
    if op == "write":
        heads = rng.choice([1, 2, 4, 8, 16, 32])
        return dict(op=op, rows=log_int(rng, 1, 520000 // heads), heads=heads, page=rng.choice([16, 32, 64, 128]),
                    fused=rng.random() < 0.5, skip=rng.random() < 0.5)
    if op == "attn":
        kv_heads, group = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 2, 4, 8])
        batch = log_int(rng, 1, 64)
        kv = log_int(rng, 1, max(1, min(131072, 4_000_000 // (batch * kv_heads))))
        nodes = rng.choice([1, 1, log_int(rng, 2, 16), log_int(rng, 17, 128)])
        return dict(op=op, batch=batch, nodes=nodes, heads=kv_heads * group, kv_heads=kv_heads, kv=kv,
                    page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.5)
    k = 64 * log_int(rng, 2, 128)
    k += 64 if k == 3072 else 0
    return dict(op=op, rows=rng.choice([1, rng.randint(2, 16)]), k=k, n=log_int(rng, 16, 28672),
                group=rng.choice([g for g in (32, 64, 128) if k % g == 0]))


# ------------------------------------------------------------------ sizes that follow from a case alone
def spread(n, lo, hi):
    """n whole numbers between lo and hi, in no order."""
    return [lo + int((hi - lo) * ((0.6180339887 * (i + 1)) % 1.0) + 0.5) for i in range(n)]


def pages_lens(case):
    b, new = case["batch"], case["new"]
    kv = spread(b, 0, case["kv"])
    return kv, ([1] * b if new == 1 else spread(b, 1, new))


def attn_lens(case):
    b, kv = case["batch"], case["kv"]
    if not case["ragged"]:
        return [kv] * b, [case["nodes"]] * b
    lens = spread(b, max(0, kv // 4), kv)
    if b >= 8:
        lens[1] = 0  # a request without a cache
    return lens, spread(b, max(1, case["nodes"] // 2), case["nodes"])


def up(a, b):
    return -(-a // b)


def work(case):
    op = case["op"]
    if op == "pages":
        kv, new = pages_lens(case)
        taken = sum(up(k + n, case["page"]) - up(k, case["page"]) for k, n in zip(kv, new))
        # lengths in; offsets and new lengths out; pages from the free list into the table; four numbers a new token
        return dict(bytes=4 * (2 * len(kv) + 2 * len(kv) + 2 * taken + 4 * sum(new)), flops=len(kv) + 4 * sum(new))
    if op == "write":
        n = case["rows"] * case["heads"]
        # keys and values in, numbers and scales out, and the values that they stand for
        return dict(bytes=2 * n * (2 * D + D // 2 + 2 + 2 * D) + 4 * case["rows"], flops=2 * n * D * 3)
    if op == "attn":
        kv, nodes = attn_lens(case)
        B, n, H, G = case["batch"], case["nodes"], case["heads"], case["kv_heads"]
        byts = 2 * sum(kv) * G * (D // 2 + 2) + 2 * B * n * H * D * 2 + 2 * sum(nodes) * G * D * 2
        byts += 4 * sum(up(k, case["page"]) for k in kv)
        return dict(bytes=byts, flops=4 * D * H * sum(m * k for m, k in zip(nodes, kv)))
    M, K, N = case["rows"], case["k"], case["n"]
    return dict(bytes=K * N // 2 + 2 * (K // case["group"]) * N + 2 * M * (K + N), flops=2 * M * K * N)


# ------------------------------------------------------------------ inputs
def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def random_codes(shape, gen):
    """Numbers of a quantised normal distribution, two to a byte."""
    lo = (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float16) * 2.6).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
    hi = (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float16) * 2.6).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
    return lo | (hi << 4)


def tree_masks(nodes, n, seed):
    """Ancestor bits of random trees: node i sees its ancestors and itself."""
    import random
    r, words = random.Random(seed), up(n, 64)
    rows = []
    for m in nodes:
        bits = [1]
        for i in range(1, m):
            bits.append(bits[r.randrange(max(0, i - 8), i)] | (1 << i))
        for b in bits + [0] * (n - m):
            for w in range(words):
                v = (b >> (64 * w)) & (2 ** 64 - 1)
                rows.append(v - 2 ** 64 if v >= 2 ** 63 else v)
    return torch.tensor(rows, dtype=torch.int64).view(len(nodes), n, words).to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    if op == "pages":
        kv, new = pages_lens(case)
        P, B = case["page"], case["batch"]
        held = [up(k, P) for k in kv]
        most = max(up(k + n, P) for k, n in zip(kv, new)) + 2
        # a pool that serves almost every request: the last ones of a full step find it empty
        wanted = sum(up(k + n, P) for k, n in zip(kv, new)) - sum(held)
        n_free = wanted - wanted // 50
        n_pages = sum(held) + n_free
        order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
        table = torch.full((B, most), -1, dtype=torch.int32, device=DEV)
        where = torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]
        table[where] = order[n_free:]
        free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        free[:n_free] = order[:n_free]
        st = dict(op=op, page=P, kv=ints(kv), new=ints(new), table=table, free=free, n_free=ints([n_free]), rows=max(1, sum(new)))
        if own:
            import paper_2502_17139_gb300.fastcoder as fc
            st["fc"] = fc
            st["pages"] = fc.KvPages(P, table, free)
            st["out"] = fc.kv_pages_outputs(B, st["rows"], DEV)
        return st
    if op == "write":
        R, H, P = case["rows"], case["heads"], case["page"]
        if case["fused"]:  # [rows][queries | keys | values], as one projection leaves them
            qkv = torch.randn((R, 6 * H * D), generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)
            k, v = qkv[:, 4 * H * D:5 * H * D].view(R, H, D), qkv[:, 5 * H * D:].view(R, H, D)
        else:
            k = torch.randn((R, H, D), generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)
            v = torch.randn((R, H, D), generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)
        n_pages = up(R, P) + 3
        slot = torch.randperm(n_pages * P, generator=gen, device=DEV)[:R].to(torch.int32)
        if R >= P:  # whole pages in a random order, as a prompt is laid out
            page = torch.randperm(n_pages, generator=gen, device=DEV)
            at = torch.arange(R, device=DEV)
            slot = (page[at // P] * P + at % P).to(torch.int32)
        if case["skip"]:
            slot[::17] = -1
        st = dict(op=op, k=k, v=v, slot=slot, page=P, heads=H, n_pages=n_pages)
        st["cache"] = [torch.zeros((n_pages, H, P, D // 2), dtype=torch.uint8, device=DEV) for _ in range(2)]
        st["cache"] += [torch.zeros((n_pages, H, P), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        if own:
            import paper_2502_17139_gb300.fastcoder as fc
            st["fc"] = fc
            st["kv4"] = fc.Kv4Cache(*st["cache"])
            st["out"] = (torch.empty((R, H, D), dtype=torch.bfloat16, device=DEV), torch.empty((R, H, D), dtype=torch.bfloat16, device=DEV))
        return st
    if op == "attn":
        kv, nodes = attn_lens(case)
        B, n, H, G, P = case["batch"], case["nodes"], case["heads"], case["kv_heads"], case["page"]
        held = [up(k, P) for k in kv]
        n_pages, most = sum(held) + 2, max(held) + 1
        table = torch.zeros((B, most), dtype=torch.int32, device=DEV)
        table[torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]] = torch.randperm(n_pages, generator=gen, device=DEV)[:sum(held)].to(torch.int32)
        codes = [random_codes((n_pages, G, P, D // 2), gen) for _ in range(2)]
        scales = [(0.3 + 0.2 * torch.rand((n_pages, G, P), generator=gen, device=DEV)).to(torch.bfloat16) for _ in range(2)]
        if case["ragged"]:  # pages used before: what stands past a request's end is anything, NaN too
            at = torch.arange(most * P, device=DEV).view(1, most, P)
            stale = (at >= ints(kv).view(B, 1, 1)) & (at < P * ints(held).view(B, 1, 1))
            for s in scales:
                page = s[table.long()]
                page[stale[:, :, None, :].expand_as(page)] = float("nan")
                inside = torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]
                s[table[inside].long()] = page[inside]
        st = dict(op=op, page=P, kv=ints(kv), nodes=ints(nodes), table=table, codes=codes, scales=scales, mask=tree_masks(nodes, n, seed))
        st["q"] = torch.randn((B, n, H, D), generator=gen, device=DEV).to(torch.bfloat16)
        st["k_new"] = torch.randn((B, G, n, D), generator=gen, device=DEV).to(torch.bfloat16)
        st["v_new"] = torch.randn((B, G, n, D), generator=gen, device=DEV).to(torch.bfloat16)
        if own:
            import paper_2502_17139_gb300.fastcoder as fc
            st["fc"] = fc
            st["kv4"] = fc.Kv4Cache(codes[0], codes[1], scales[0], scales[1])
            st["ws"] = fc.kv4_attn_workspace(B, n, H, G, DEV)
            st["out"] = torch.empty_like(st["q"])
        return st
    M, K, N, g = case["rows"], case["k"], case["n"], case["group"]
    w = (torch.randn((K, N), generator=gen, device=DEV) * K ** -0.5).to(torch.bfloat16)
    st = dict(op=op, x=torch.randn((M, K), generator=gen, device=DEV).to(torch.bfloat16), group=g)
    if own:
        import paper_2502_17139_gb300.fastcoder as fc
        st["fc"] = fc
        st["w4"] = fc.fc_w4_pack(w, g)
        st["out"] = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
    else:
        c, s = quantised(w.float().view(K // g, g, N), 1)
        c = (c.view(K // 2, 2, N) + 8).to(torch.uint8)
        st["codes"], st["scale"] = c[:, 0] | (c[:, 1] << 4), s.view(K // g, N)
    return st


# ------------------------------------------------------------------ plain forms
def quantised(x, dim):
    """Whole numbers (as floats) and bf16 scales of x along dim."""
    s = (x.abs().amax(dim, keepdim=True) / 7).to(torch.bfloat16)
    sf = s.float()
    return torch.where(sf > 0, (x / sf).round().clamp(-7, 7), torch.zeros_like(x)), s


def halves(c):
    """The two numbers of each byte, in order along the last axis."""
    return torch.stack(((c & 15).float() - 8, (c >> 4).float() - 8), -1).flatten(-2)


def plain_pages(st):
    kv, new, P = st["kv"].long(), st["new"].long(), st["page"]
    B, most = st["table"].shape
    have, need = (kv + P - 1) // P, (kv + new + P - 1) // P
    fits = need <= most
    more = torch.where(fits, need - have, torch.zeros_like(need))
    end = more.cumsum(0)
    served = fits & ((more == 0) | (end <= st["n_free"]))
    j = torch.arange(most, device=kv.device)[None, :]
    at = st["n_free"] - 1 - (end - more)[:, None] - (j - have[:, None])
    fresh = served[:, None] & (j >= have[:, None]) & (j < need[:, None])
    table = torch.where(fresh, st["free"][at.clamp(0, st["free"].numel() - 1)], st["table"])
    cu = torch.cat((torch.zeros_like(kv[:1]), new.cumsum(0)))
    seq = torch.repeat_interleave(torch.arange(B, device=kv.device), new, output_size=st["rows"])
    inner = torch.arange(st["rows"], device=kv.device) - cu[seq]
    pos = kv[seq] + inner
    slot = torch.where(served[seq], table[seq, (pos // P).clamp(max=most - 1)].long() * P + pos % P, torch.full_like(pos, -1))
    out = dict(cu=cu, seq=seq, pos=pos, slot=slot, kv_len=torch.where(served, kv + new, kv),
               n_free=st["n_free"] - torch.where(served, more, torch.zeros_like(more)).sum())
    return dict({k: v.to(torch.int32) for k, v in out.items()}, table=table)


def plain_write(st):
    P = st["page"]
    live = st["slot"] >= 0
    slot = st["slot"][live].long()
    back = []
    for x, codes, scales in ((st["k"], st["cache"][0], st["cache"][2]), (st["v"], st["cache"][1], st["cache"][3])):
        c, s = quantised(x.float(), -1)
        c = (c + 8).to(torch.uint8).view(*c.shape[:-1], D // 2, 2)
        codes[slot // P, :, slot % P] = (c[..., 0] | (c[..., 1] << 4))[live]
        scales[slot // P, :, slot % P] = s[..., 0][live]
        at = st["slot"].clamp(min=0).long()
        val = halves(codes[at // P, :, at % P]) * scales[at // P, :, at % P].float()[..., None]
        back.append(torch.where(live[:, None, None], val, torch.zeros_like(val)).to(torch.bfloat16))
    return dict(k=back[0], v=back[1])


def plain_attn(st):
    B, n, H, _ = st["q"].shape
    P, G = st["page"], st["k_new"].shape[1]
    L = st["table"].shape[1] * P
    seen = torch.arange(L, device=DEV)[None, :] < st["kv"][:, None]
    table = st["table"].long()

    def cached(i):  # [B][G][L][D], zeros past a request's end
        s = st["scales"][i][table].transpose(1, 2).reshape(B, G, L).float()
        s = torch.where(seen[:, None, :], s, torch.zeros_like(s))
        return halves(st["codes"][i][table].transpose(1, 2).reshape(B, G, L, D // 2)) * s[..., None]

    q = st["q"].float().view(B, n, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, -1, D)
    bits = (st["mask"][..., None] >> torch.arange(64, device=DEV)) & 1
    bits = bits.flatten(-2)[..., :n].bool() & (torch.arange(n, device=DEV)[None, None, :] < st["nodes"][:, None, None])
    row = torch.arange(n, device=DEV)[None, :] < st["nodes"][:, None]
    sees = torch.cat((seen[:, None, :].expand(B, n, L), bits), -1) & row[:, :, None]
    sees = sees[:, None, None].expand(B, 1, H // G, n, L + n).reshape(B, 1, -1, L + n)
    score = torch.cat((q @ cached(0).transpose(-1, -2), q @ st["k_new"].float().transpose(-1, -2)), -1) * D ** -0.5
    score = score.masked_fill_(~sees, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p[..., :L] @ cached(1) + p[..., L:] @ st["v_new"].float()
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.view(B, G, H // G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H, D).to(torch.bfloat16)


def plain_matvec(st):
    c, s, g = st["codes"], st["scale"].float(), st["group"]
    w = torch.stack(((c & 15).float() - 8, (c >> 4).float() - 8), 1).flatten(0, 1)
    w = (w.view(s.shape[0], g, -1) * s[:, None]).flatten(0, 1)
    return (st["x"].float() @ w).to(torch.bfloat16)


def run(st):
    op = st["op"]
    if not own:
        return {"pages": plain_pages, "write": plain_write, "attn": plain_attn, "matvec": plain_matvec}[op](st)
    fc = st["fc"]
    if op == "pages":
        o = fc.fc_kv_pages_plan(st["pages"], st["kv"], st["new"], st["n_free"], out=st["out"])
        return dict(cu=o["cu"], seq=o["seq"], pos=o["pos"], slot=o["slot"], kv_len=o["kv_len"], n_free=o["n_free"], table=st["table"])
    if op == "write":
        fc.fc_kv4_write(st["kv4"], st["k"], st["v"], st["slot"])
        k, v = fc.fc_kv4_read(st["kv4"], st["slot"], out=st["out"])
        return dict(k=k, v=v)
    if op == "attn":
        return fc.fc_kv4_attn(st["q"], st["kv4"], st["table"], st["kv"], st["k_new"], st["v_new"], st["mask"], st["nodes"],
                              out=st["out"], workspace=st["ws"])
    return fc.fc_w4_matvec(st["x"], st["w4"], out=st["out"])


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "pages":
        return None  # whole numbers: nothing to round
    if op == "write":
        out = []
        for x in (st["k"], st["v"]):
            x = x.double()
            s = (x.abs().max(-1, keepdim=True).values / 7).bfloat16().double()
            c = torch.round(x / s).clamp(-7, 7)
            val = torch.nan_to_num(c * s, nan=0.0)
            val[st["slot"] < 0] = 0
            out.append(val)
        return dict(k=out[0], v=out[1])
    if op == "attn":
        B, n, H, _ = st["q"].shape
        P, G = st["page"], case["kv_heads"]
        kv, nodes = attn_lens(case)
        out = torch.zeros((B, n, H, D), dtype=torch.float64, device=DEV)
        weight = 2.0 ** torch.arange(4, device=DEV, dtype=torch.float64)  # the four bits of a number
        for b in range(B):
            L, m = kv[b], nodes[b]
            at = torch.arange(L, device=DEV)
            page, off = st["table"][b, at // P].long(), at % P
            vis = torch.ones((m, L + m), dtype=torch.bool, device=DEV)
            for j in range(m):
                vis[:, L + j] = (st["mask"][b, :m, j // 64] >> (j % 64)) & 1 == 1
            for g in range(G):
                def whole(i, new):
                    byte = st["codes"][i][page, g, off]
                    nib = ((byte[:, :, None] >> torch.arange(8, device=DEV, dtype=torch.uint8)) & 1).double().view(L, D, 4) @ weight
                    return torch.cat(((nib - 8) * st["scales"][i][page, g, off].double()[:, None], new[b, g, :m].double()))
                K, V = whole(0, st["k_new"]), whole(1, st["v_new"])
                for h in range(g * (H // G), (g + 1) * (H // G)):
                    z = (st["q"][b, :m, h].double() @ K.T) / math.sqrt(D)
                    out[b, :m, h] = torch.softmax(z.masked_fill(~vis, -math.inf), -1) @ V
        return out
    M, K, N, g = case["rows"], case["k"], case["n"], case["group"]
    c = torch.empty((K, N), dtype=torch.float64, device=DEV)
    c[0::2], c[1::2] = (st["codes"] % 16).double() - 8, torch.div(st["codes"], 16, rounding_mode="floor").double() - 8
    y = torch.zeros((M, N), dtype=torch.float64, device=DEV)
    for t in range(K // g):
        y += st["scale"][t].double() * (st["x"][:, t * g:(t + 1) * g].double() @ c[t * g:(t + 1) * g])
    return y
