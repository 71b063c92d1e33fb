"""The operators of serving from a cache in 8 bits that is kept to a budget: their cases, their plain forms in torch and
their definitions in 64 bits.

* norm    - queries and keys normed for each head and rotated by position, values laid beside them (fc_qk_norm_rope);
* write   - keys and values rounded into the pages of an 8-bit cache, and read back (fc_kv8_write, fc_kv8_read);
* attn    - attention of one token, or of a draft tree's tokens, over that cache, with the weight that each cached token
            received where it is asked for (fc_kv8_attn);
* evict   - the cache cut down to a number of tokens a request, by the weights that they received (fc_kv8_evict).

Formulas.  The cache holds e4m3 numbers, a power of two for each 16 tokens of a page and kv head (a block): s = 2^e with the
smallest e >= -120 such that max|x| <= 448 s; a number is e4m3(x / s).  Tokens added to a block that holds some already
make its scale the larger of the two, the numbers there rounded again.  Eviction keeps the tokens of the last ``recent``
positions, then those of the largest weights (ties: the lower index); kept tokens past the new length move, in order, into
the places that come free below it; a block that takes one gets the scale for what it then holds.

``own`` false: elementary torch operations in 32 bits.  ``own`` true: the framework's calls.
"""
import math

import torch

own = False

D = 128    # head dimension of the cache
BLOCK = 16  # tokens a scale
DEV = "cuda"


# ------------------------------------------------------------------ cases
def listed():
    return [
        # queries and keys of one decoding step of 32 requests: between two small products, latency
        dict(name="norm decode 32x32/8", op="norm", batch=32, n=1, heads=32, kv_heads=8, dim=128, far=131072),
        # prompts of 65,000 tokens at once, 16 heads without sharing (the 1.3B decoder's): the read and the write
        dict(name="norm prompts 65000x16/16", op="norm", batch=1, n=65000, heads=16, kv_heads=16, dim=128, far=65536),
        # one decoding step of 32 requests: a row each, into blocks that hold some tokens already
        dict(name="write decode b32", op="write", batch=32, new=1, kv=16384, heads=8, page=64),
        # prompts of ragged lengths behind cached prefixes
        dict(name="write prompts b40", op="write", batch=40, new=3001, kv=500, heads=8, page=64),
        # one short request, one token: latency
        dict(name="attn token b1 kv500", op="attn", batch=1, nodes=1, heads=32, kv_heads=8, kv=500, page=64, ragged=False, weights=False),
        # the step loop's shape (32 requests, 32 / 8 heads, 16384 keys), one token each: the cache read bounds it
        dict(name="attn token b32 kv16384", op="attn", batch=32, nodes=1, heads=32, kv_heads=8, kv=16384, page=64, ragged=False, weights=False),
        # one request with a long context: the keys have to be split over the whole GPU
        dict(name="attn token b1 kv131071", op="attn", batch=1, nodes=1, heads=32, kv_heads=8, kv=131071, page=128, ragged=False, weights=False),
        # the last four tokens of ragged prompts tell which cached tokens matter: weights from zero
        dict(name="attn weights b24 kv8192", op="attn", batch=24, nodes=4, heads=32, kv_heads=8, kv=8192, page=64, ragged=True, weights=True),
        # 16 requests of ragged lengths, 32 heads without sharing, draft trees of 64 nodes
        dict(name="attn tree64 b16 mha", op="attn", batch=16, nodes=64, heads=32, kv_heads=32, kv=4096, page=64, ragged=True, weights=False),
        # the step loop's whole shape: trees of 128 nodes over 16384 keys; the matrix products bound it
        dict(name="attn tree128 b32", op="attn", batch=32, nodes=128, heads=32, kv_heads=8, kv=16384, page=64, ragged=False, weights=False),
        # a running batch gives one page a request back, every 64 steps
        dict(name="evict a page b32", op="evict", batch=32, kv=4160, keep=4096, recent=128, heads=8, page=64, ragged=False),
        # prompts cut to half of their length after the first pass
        dict(name="evict half b16 kv16384", op="evict", batch=16, kv=16384, keep=8192, recent=256, heads=8, page=64, ragged=True),
    ]


def log_int(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "write", "attn", "attn", "evict"])
    if op == "norm":
        kv_heads, group, dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 256])
        batch = log_int(rng, 1, 200)
        most = 400_000_000 // (batch * kv_heads * (group + 2) * dim)
        return dict(op=op, batch=batch, n=rng.choice([1, log_int(rng, 1, max(1, min(30000, most)))]), heads=kv_heads * group, kv_heads=kv_heads,
                    dim=dim, far=log_int(rng, 1, 1000000))
    if op == "write":
        heads, batch = rng.choice([1, 2, 4, 8, 16, 32]), log_int(rng, 1, 256)
        return dict(op=op, batch=batch, new=log_int(rng, 1, max(1, min(8000, 480000 // (heads * batch)))),
                    kv=log_int(rng, 1, max(1, min(30000, 8000000 // (heads * batch)))), heads=heads, page=rng.choice([16, 32, 64, 128]))
    if op == "attn":
        kv_heads, group = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 2, 4, 8])
        batch = log_int(rng, 1, 64)
        kv = log_int(rng, 1, max(1, min(131072, 4_000_000 // (batch * kv_heads))))
        nodes = rng.choice([1, 1, log_int(rng, 2, 16), log_int(rng, 17, 128)])
        return dict(op=op, batch=batch, nodes=nodes, heads=kv_heads * group, kv_heads=kv_heads, kv=kv, page=rng.choice([16, 32, 64, 128]),
                    ragged=rng.random() < 0.5, weights=nodes * group <= 16 and rng.random() < 0.4)
    heads, batch = rng.choice([1, 2, 4, 8, 16, 32]), log_int(rng, 1, 64)
    kv = log_int(rng, 16, max(16, min(131072, 2_000_000 // (heads * batch))))
    keep = max(1, int(kv * rng.choice([0.98, 0.5, rng.uniform(0.05, 0.99)])))
    return dict(op=op, batch=batch, kv=kv, keep=keep, recent=rng.choice([0, log_int(rng, 1, keep)]), heads=heads, page=rng.choice([16, 32, 64, 128]),
                ragged=rng.random() < 0.5)


# ------------------------------------------------------------------ sizes that follow from a case alone
def up(a, b):
    return -(-a // b)


def spread(n, lo, hi):
    """n whole numbers between lo and hi, in no order."""
    return [lo + int((hi - lo) * ((0.6180339887 * (i + 1)) % 1.0) + 0.5) for i in range(n)]


def write_lens(case):
    b, new = case["batch"], case["new"]
    return spread(b, 0, case["kv"]), ([1] * b if new == 1 else spread(b, 1, new))


def attn_lens(case):
    b, kv = case["batch"], case["kv"]
    if not case["ragged"]:
        return [kv] * b, [case["nodes"]] * b
    lens = spread(b, max(0, kv // 4), kv)
    if b >= 8:
        lens[1] = 0  # a request without a cache
    return lens, spread(b, max(1, case["nodes"] // 2), case["nodes"])


def evict_lens(case):
    if not case["ragged"]:
        return [case["kv"]] * case["batch"]
    return spread(case["batch"], case["kv"] // 3, case["kv"])  # some are within the budget already


def work(case):
    op = case["op"]
    if op == "norm":
        rows, heads = case["batch"] * case["n"], case["heads"] + 2 * case["kv_heads"]
        return dict(bytes=4 * rows * heads * case["dim"] + 4 * rows + 4 * case["dim"], flops=10 * rows * (heads - case["kv_heads"]) * case["dim"])
    if op == "write":
        rows = sum(write_lens(case)[1])
        n = rows * case["heads"]
        # keys and values in, numbers and scales out, and the values that they stand for
        return dict(bytes=2 * n * (2 * D + D + 2 * D) + 8 * rows, flops=2 * n * D * 3)
    if op == "attn":
        kv, nodes = attn_lens(case)
        B, n, H, G = case["batch"], case["nodes"], case["heads"], case["kv_heads"]
        byts = 2 * sum(kv) * G * D + 2 * 4 * G * sum(up(k, BLOCK) for k in kv) + 2 * B * n * H * D * 2 + 2 * sum(nodes) * G * D * 2
        byts += 4 * sum(up(k, case["page"]) for k in kv) + (4 * sum(kv) * G if case["weights"] else 0)
        return dict(bytes=byts, flops=4 * D * H * sum(m * k for m, k in zip(nodes, kv)))
    lens = evict_lens(case)
    # the weights and positions of all, those of the kept; the rows that have to move: where a token's weight has nothing to
    # do with its place, a share (1 - keep / length) of the places below keep comes free
    byts, cut = 0, 0
    for n in lens:
        keep = min(n, case["keep"])
        moved = min(n - keep, int(keep * (1 - keep / max(1, n))) + min(case["recent"], n - keep) // 2)
        byts += case["heads"] * (8 * n + 12 * keep + 4 * D * moved)
        cut += n
    return dict(bytes=byts, flops=4 * cut * case["heads"])


# ------------------------------------------------------------------ inputs
def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def random_codes(shape, gen):
    """e4m3 numbers of a normal distribution."""
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float16) * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def random_cache(n_pages, heads, page, gen):
    """Numbers of keys and of values, and their blocks' scales: powers of two about 2^-7."""
    codes = [random_codes((n_pages, heads, page, D), gen) for _ in range(2)]
    scales = [torch.pow(2.0, torch.randint(-8, -5, (n_pages, heads, page // BLOCK), generator=gen, device=DEV).float()) for _ in range(2)]
    return codes + scales


def random_table(held, most, n_pages, gen):
    table = torch.zeros((len(held), most), dtype=torch.int32, device=DEV)
    table[torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]] = torch.randperm(n_pages, generator=gen, device=DEV)[:sum(held)].to(torch.int32)
    return table


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


def randn(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    st = dict(op=op)
    if own:
        import paper_2502_17139_gb300.fastcoder as fc
        st["fc"] = fc
    if op == "norm":
        B, n, H, G, dim = case["batch"], case["n"], case["heads"], case["kv_heads"], case["dim"]
        # two projections' rows, the second of keys and values side by side; norms' weights about 1
        q, kv = randn((B, n, H, dim), gen), randn((B, n, 2, G, dim), gen)
        st.update(q=q, k=kv[:, :, 0], v=kv[:, :, 1])
        st["wq"], st["wk"] = ((1 + 0.3 * torch.randn((dim,), generator=gen, device=DEV)).to(torch.bfloat16) for _ in range(2))
        first = torch.randint(0, max(1, case["far"]), (B, 1), generator=gen, device=DEV)
        st["pos"] = (first + torch.arange(n, device=DEV)[None, :]).to(torch.int32)
        st["base"], st["eps"] = 1e6, 1e-6
        if own:
            st["out"] = (torch.empty_like(q), *(torch.empty((B, G, n, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
        return st
    P = case["page"]
    st["page"] = P
    if op == "write":
        kv, new = write_lens(case)
        H, rows = case["heads"], sum(new)
        held = [up(k + n, P) for k, n in zip(kv, new)]
        n_pages, most = sum(held) + 2, max(held)
        table = random_table(held, most, n_pages, gen)
        seq = torch.repeat_interleave(torch.arange(len(new), device=DEV), ints(new).long(), output_size=rows)
        start = ints(new).long().cumsum(0) - ints(new)
        pos = ints(kv).long()[seq] + torch.arange(rows, device=DEV) - start[seq]
        st["slot"] = (table[seq, pos // P].long() * P + pos % P).to(torch.int32)
        if new[0] > 1:
            st["slot"][5::29] = -1  # padding rows
        qkv = randn((rows, 6 * H * D), gen) * torch.exp(torch.randn((rows, 1), generator=gen, device=DEV) * 0.7).to(torch.bfloat16)
        st["k"], st["v"] = qkv[:, 4 * H * D:5 * H * D].view(rows, H, D), qkv[:, 5 * H * D:].view(rows, H, D)
        st["cache"] = random_cache(n_pages, H, P, gen)
        if own:
            st["kv8"] = fc.Kv8Cache(*st["cache"])
            st["out"] = tuple(torch.empty((rows, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return st
    if op == "attn":
        kv, nodes = attn_lens(case)
        B, n, H, G = case["batch"], case["nodes"], case["heads"], case["kv_heads"]
        held = [up(k, P) for k in kv]
        n_pages, most = sum(held) + 2, max(held) + 1
        table = random_table(held, most, n_pages, gen)
        cache = random_cache(n_pages, G, P, gen)
        if case["ragged"]:  # pages used before: what stands past a request's end is anything, NaN too
            inside = torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]
            at = torch.arange(most * P, device=DEV).view(1, most, P)
            stale = (at >= ints(kv).view(B, 1, 1))[inside]  # [pages held][P]
            for i in range(2):
                page = cache[i][table[inside].long()]
                page[stale[:, None, :, None].expand_as(page)] = 0x7F
                cache[i][table[inside].long()] = page
                scale = cache[2 + i][table[inside].long()]
                scale[stale[:, None, ::BLOCK].expand_as(scale)] = float("nan")  # blocks that begin past the end
                cache[2 + i][table[inside].long()] = scale
        st.update(kv=ints(kv), nodes=ints(nodes), table=table, cache=cache, mask=tree_masks(nodes, n, seed), weights=case["weights"])
        st["q"], st["k_new"], st["v_new"] = randn((B, n, H, D), gen), randn((B, G, n, D), gen), randn((B, G, n, D), gen)
        st["weight"] = torch.zeros((n_pages, G, P), dtype=torch.float32, device=DEV) if case["weights"] else None
        if own:
            st["kv8"] = fc.Kv8Cache(*cache)
            st["ws"] = fc.kv8_attn_workspace(B, n, H, G, DEV, most * P if case["weights"] else 0)
            st["out"] = torch.empty_like(st["q"])
        return st
    kv, H, B = evict_lens(case), case["heads"], case["batch"]
    held = [up(k, P) for k in kv]
    n_pages, most = sum(held) + 2, max(held) + 1
    st.update(kv=ints(kv), keep=ints([case["keep"]] * B), cap=min(case["keep"], most * P), recent=case["recent"])
    st["table"] = random_table(held, most, n_pages, gen)
    st["cache"] = random_cache(n_pages, H, P, gen)
    # what attention leaves: many tokens with little weight, some of them none, few with much
    weight = torch.exp(2 * torch.randn((n_pages, H, P), generator=gen, device=DEV))
    st["weight"] = torch.where(torch.rand((n_pages, H, P), generator=gen, device=DEV) < 0.1, torch.zeros_like(weight), weight)
    # positions in an order that earlier evictions left, apart from the newest tokens
    born = torch.zeros((n_pages, H, P), dtype=torch.int32, device=DEV)
    at = torch.arange(most * P, device=DEV).view(1, 1, -1)
    old = torch.rand((B, H, most * P), generator=gen, device=DEV).masked_fill_(at >= ints(kv).view(B, 1, 1) * 7 // 8, 2.0).argsort(-1).argsort(-1)
    place = torch.where(at < ints(kv).view(B, 1, 1) * 7 // 8, old, at.expand_as(old)).to(torch.int32) + 1000
    inside = torch.arange(most, device=DEV)[None, :] < ints(held)[:, None]
    born[st["table"][inside].long()] = place.view(B, H, most, P).transpose(1, 2)[inside]
    st["born"] = born
    st["track_out"] = [torch.zeros_like(st["weight"]), torch.zeros_like(born)]
    st["from"] = torch.empty((B, H, st["cap"]), dtype=torch.int32, device=DEV)
    if own:
        st["kv8"] = fc.Kv8Cache(*st["cache"])
        st["track"], st["track2"] = fc.Kv8Track(st["weight"], born), fc.Kv8Track(*st["track_out"])
        st["ws"] = fc.kv8_evict_workspace(B, H, st["cap"], DEV)
    return st


# ------------------------------------------------------------------ plain forms
def plain_norm(st):
    q, k, v, dim = st["q"].float(), st["k"].float(), st["v"], st["q"].shape[-1]
    f = torch.pow(torch.tensor(st["base"], dtype=torch.float64, device=DEV), -2.0 * torch.arange(dim // 2, device=DEV).double() / dim)
    angle = st["pos"].double()[:, :, None, None] * f
    c, s = torch.cos(angle).float(), torch.sin(angle).float()

    def one(x, w):
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * w.float()
        a, b = x[..., :dim // 2], x[..., dim // 2:]
        return torch.cat((a * c - b * s, b * c + a * s), -1).to(torch.bfloat16)

    return dict(q=one(q, st["wq"]), k=one(k, st["wk"]).transpose(1, 2).contiguous(), v=v.transpose(1, 2).contiguous())


def scale_for(top):
    """The smallest power of two s >= 2^-120 with top <= 448 s."""
    m, e = torch.frexp(top / 448)
    e = torch.where(m > 0.5, e, e - 1).clamp(min=-120)
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), torch.full_like(top, 2.0 ** -120))


def value_of(codes):
    return codes.view(torch.float8_e4m3fn).float()


def plain_write(st):
    P = st["page"]
    live = st["slot"] >= 0
    slot = torch.where(live, st["slot"], torch.zeros_like(st["slot"])).long()
    block, off = slot // BLOCK, slot % BLOCK  # over the pool: page * (page / 16) + block in page
    n_blocks = st["cache"][0].shape[0] * (P // BLOCK)
    H = st["k"].shape[1]
    first = torch.full((n_blocks,), BLOCK, device=DEV).scatter_reduce_(0, block[live], off[live], "amin")
    hit = torch.nonzero(first < BLOCK)[:, 0]
    pg, pb = hit // (P // BLOCK), hit % (P // BLOCK)
    older = torch.arange(BLOCK, device=DEV)[None, :] < first[hit][:, None]  # tokens held already
    back = []
    for i, x in ((0, st["k"]), (1, st["v"])):
        codes = st["cache"][i].view(-1, H, P // BLOCK, BLOCK, D)
        scales = st["cache"][2 + i]
        x = x.float()
        top = torch.zeros((n_blocks, H), device=DEV).scatter_reduce_(0, block[live][:, None].expand(-1, H), x[live].abs().amax(-1), "amax")
        new = scale_for(top)
        new[hit] = torch.where((first[hit] > 0)[:, None], torch.maximum(new[hit], scales[pg, :, pb]), new[hit])
        was = codes[pg, :, pb]  # [blocks][H][16][D]
        again = (value_of(was) * (scales[pg, :, pb] / new[hit])[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        codes[pg, :, pb] = torch.where(older[:, None, :, None], again, was)
        scales[pg, :, pb] = new[hit]
        c = (x / new[block][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        st["cache"][i][slot[live] // P, :, slot[live] % P] = c[live]
        val = value_of(st["cache"][i][slot // P, :, slot % P]) * scales[slot // P, :, slot % P // BLOCK][..., None]
        back.append(torch.where(live[:, None, None], val, torch.zeros_like(val)).to(torch.bfloat16))
    # the rows written, and what the cache holds now
    return dict(k=back[0], v=back[1], codes=[st["cache"][i].view(torch.float8_e4m3fn) for i in range(2)], scales=st["cache"][2:])


def plain_attn(st):
    B, n, H, _ = st["q"].shape
    P, G = st["page"], st["k_new"].shape[1]
    L = st["table"].shape[1] * P
    seen = torch.arange(L, device=DEV)[None, :] < st["kv"][:, None]
    table = st["table"].long()

    def cached(i):  # [B][G][L][D], zeros past a request's end
        x = value_of(st["cache"][i][table]) * st["cache"][2 + i][table].repeat_interleave(BLOCK, -1)[..., None]
        return x.transpose(1, 2).reshape(B, G, L, D).masked_fill_(~seen[:, None, :, None], 0.0)

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
    o = o.view(B, G, H // G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H, D).to(torch.bfloat16)
    if not st["weights"]:
        return o
    w = torch.where(total > 0, p[..., :L] / total, torch.zeros_like(p[..., :L])).sum(2).view(B, G, -1, P).transpose(1, 2)  # [B][pages][G][P]
    inside = torch.arange(w.shape[1], device=DEV)[None, :] < ((st["kv"] + P - 1) // P)[:, None]
    st["weight"][table[inside]] = w[inside]
    return dict(o=o, weight=st["weight"])


def plain_evict(st):
    P, (B, H, cap) = st["page"], st["from"].shape
    table, kv = st["table"].long(), st["kv"].long()
    L = table.shape[1] * P
    keep = torch.minimum(st["keep"].long(), kv)
    w, born = (st[x][table].transpose(1, 2).reshape(B, H, L) for x in ("weight", "born"))
    born = born.long()
    at = torch.arange(L, device=DEV).view(1, 1, L)
    live = (at < kv.view(B, 1, 1)).expand(B, H, L)
    newest = born.masked_fill(~live, -1).amax(-1, keepdim=True)
    bits = (w + 0.0).view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))  # in the order of the weights
    key = torch.where(born > newest - st["recent"], born + 2 ** 40, key).masked_fill(~live, -2 ** 50)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, at.expand(B, H, L))
    kept = rank < keep.view(B, 1, 1)
    low = at < keep.view(B, 1, 1)
    hole, source = low & ~kept, ~low & kept
    # the i-th hole takes the i-th source
    nth = torch.where(source, source.cumsum(-1) - 1, torch.full_like(at, L))
    of = torch.zeros((B, H, L + 1), dtype=torch.int64, device=DEV).scatter_(-1, nth, at.expand(B, H, L))
    frm = torch.where(hole, of.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), torch.full_like(of[..., :L], -1))
    st["from"].copy_(frm[..., :cap])
    now = torch.where(hole, frm, at)[..., :L]  # the index that each place holds from here on
    put = low.expand(B, H, L)
    b, h, i = torch.nonzero(put, as_tuple=True)
    page, off = table[b, i // P], i % P
    st["track_out"][0][page, h, off] = w.gather(-1, now)[put]
    st["track_out"][1][page, h, off] = born.gather(-1, now)[put].to(torch.int32)
    # the rows, block by block of those that take any
    pad = hole.view(B, H, L // BLOCK, BLOCK)
    b, h, t = torch.nonzero(pad.any(-1), as_tuple=True)
    page, sub = table[b, t * BLOCK // P], t % (P // BLOCK)
    takes, held = pad[b, h, t], live.reshape(B, H, L // BLOCK, BLOCK)[b, h, t]
    src = frm.view(B, H, L // BLOCK, BLOCK)[b, h, t].clamp(min=0)
    sp, so = table[b[:, None], src // P], src % P
    for k in range(2):
        codes, scales = st["cache"][k], st["cache"][2 + k]
        block = codes.view(-1, H, P // BLOCK, BLOCK, D)
        was, came = block[page, h, sub], codes[sp, h[:, None], so]
        val = torch.where(takes[..., None], value_of(came) * scales[sp, h[:, None], so // BLOCK][..., None],
                          value_of(was) * scales[page, h, sub][:, None, None]).masked_fill_(~held[..., None], 0.0)
        new = scale_for(val.abs().amax((-1, -2)))
        val = (val / new[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        block[page, h, sub] = torch.where(held[..., None], val, was)
        scales[page, h, sub] = new
    return evicted(st)


def evicted(st):
    c = st["cache"]
    return dict(frm=st["from"], weight=st["track_out"][0], born=st["track_out"][1], k=c[0].view(torch.float8_e4m3fn),
                v=c[1].view(torch.float8_e4m3fn), k_scale=c[2], v_scale=c[3])


def run(st):
    op = st["op"]
    if not own:
        return {"norm": plain_norm, "write": plain_write, "attn": plain_attn, "evict": plain_evict}[op](st)
    fc = st["fc"]
    if op == "norm":
        q, k, v = fc.fc_qk_norm_rope(st["q"], st["k"], st["v"], st["wq"], st["wk"], st["pos"], st["base"], st["eps"], out=st["out"])
        return dict(q=q, k=k, v=v)
    if op == "write":
        fc.fc_kv8_write(st["kv8"], st["k"], st["v"], st["slot"])
        k, v = fc.fc_kv8_read(st["kv8"], st["slot"], out=st["out"])
        return dict(k=k, v=v, codes=[st["cache"][i].view(torch.float8_e4m3fn) for i in range(2)], scales=st["cache"][2:])
    if op == "attn":
        o = fc.fc_kv8_attn(st["q"], st["kv8"], st["table"], st["kv"], st["k_new"], st["v_new"], st["mask"], st["nodes"], out=st["out"],
                           workspace=st["ws"], weight=st["weight"], decay=0.0)
        return dict(o=o, weight=st["weight"]) if st["weights"] else o
    fc.fc_kv8_evict(st["kv8"], st["table"], st["kv"], st["keep"], st["recent"], st["track"], st["track2"], out=st["from"], workspace=st["ws"])
    return evicted(st)


# ------------------------------------------------------------------ the definitions in 64 bits
def e4m3(x):
    """x (64 bits, |x| <= 448) rounded to three bits after the first, ties to even, steps of 2^-9 near zero."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def decoded(codes):
    """What e4m3 bytes stand for, by their bits."""
    c = codes.to(torch.int16)
    e, m = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(e > 0, torch.ldexp(8 + m, (e - 10).int()), torch.ldexp(m, torch.full_like(e, -9).int()))
    return torch.where(c >= 128, -mag, mag)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "norm":
        half = case["dim"] // 2
        turn = torch.exp(-torch.arange(half, device=DEV).double() / half * math.log(st["base"]))
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), st["pos"].double()[..., None] * turn)[:, :, None]

        def one(x, w):
            x = x.double()
            x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + st["eps"])
            z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * turn
            return torch.cat((z.real, z.imag), -1)

        return dict(q=one(st["q"], st["wq"]), k=one(st["k"], st["wk"]).permute(0, 2, 1, 3), v=st["v"].double().permute(0, 2, 1, 3))
    P = case["page"]
    if op == "write":
        H, rows = case["heads"], st["slot"].numel()
        slot = st["slot"].long()
        run_of = torch.where(slot >= 0, slot // BLOCK, torch.full_like(slot, -1))
        blocks, where = torch.unique(run_of, return_inverse=True)
        n, real = blocks.numel(), blocks >= 0
        page, sub = blocks.clamp(min=0) // (P // BLOCK), blocks.clamp(min=0) % (P // BLOCK)
        start = torch.full((n,), BLOCK, dtype=torch.int64, device=DEV).scatter_reduce(0, where, slot.clamp(min=0) % BLOCK, "amin")
        out = dict(k=None, v=None, codes=[], scales=[])
        for i, (name, x) in enumerate((("k", st["k"]), ("v", st["v"]))):
            x = x.double()
            top = torch.zeros((n, H), dtype=torch.float64, device=DEV).scatter_reduce(0, where[:, None].expand(rows, H), x.abs().max(-1).values, "amax")
            e = torch.ceil(torch.log2(top / 448) - 1e-12).clamp(min=-120)
            e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
            s = torch.exp2(e)
            before = st["cache"][2 + i][page, :, sub].double()
            s = torch.where((start > 0)[:, None] & (before > s), before, s)
            scales = st["cache"][2 + i].double()
            codes = decoded(st["cache"][i])
            lie = torch.arange(BLOCK, device=DEV)
            spot = sub[:, None] * BLOCK + lie  # [n][16]
            held = codes[page[:, None], :, spot]  # [n][16][H][D]
            anew = torch.where((lie[None] < start[:, None])[..., None, None], e4m3(held * (before / s)[:, None, :, None]), held)
            codes[page[real][:, None], :, spot[real]] = anew[real]
            scales[page[real], :, sub[real]] = s[real]
            live = slot >= 0
            c = e4m3(x / s[where][..., None])
            codes[slot[live] // P, :, slot[live] % P] = c[live]
            val = c * s[where][..., None]
            val[~live] = 0
            out[name] = val
            out["codes"].append(codes)
            out["scales"].append(scales)
        return out
    if op == "attn":
        B, n, H, _ = st["q"].shape
        G = case["kv_heads"]
        kv, nodes = attn_lens(case)
        out = torch.zeros((B, n, H, D), dtype=torch.float64, device=DEV)
        weight = torch.zeros(st["weight"].shape, dtype=torch.float64, device=DEV) if case["weights"] else None
        for b in range(B):
            L, m = kv[b], nodes[b]
            at = torch.arange(L, device=DEV)
            page, off = st["table"][b, at // P].long(), at % P
            vis = torch.ones((m, L + m), dtype=torch.bool, device=DEV)
            for j in range(m):
                vis[:, L + j] = (st["mask"][b, :m, j // 64] >> (j % 64)) & 1 == 1
            for g in range(G):
                def whole(i, new):
                    x = decoded(st["cache"][i][page, g, off]) * st["cache"][2 + i][page, g, off // BLOCK].double()[:, None]
                    return torch.cat((x, new[b, g, :m].double()))
                K, V = whole(0, st["k_new"]), whole(1, st["v_new"])
                for h in range(g * (H // G), (g + 1) * (H // G)):
                    z = (st["q"][b, :m, h].double() @ K.T) / math.sqrt(D)
                    p = torch.softmax(z.masked_fill(~vis, -math.inf), -1)
                    out[b, :m, h] = p @ V
                    if weight is not None:
                        weight[page, g, off] += p[:, :L].sum(0)
        return out if weight is None else dict(o=out, weight=weight)
    B, H, cap = case["batch"], case["heads"], st["cap"]
    lens = evict_lens(case)
    if B * H > 600:
        return None
    k, v = decoded(st["cache"][0]), decoded(st["cache"][1])
    ks, vs = st["cache"][2].double(), st["cache"][3].double()
    weight = torch.zeros(st["weight"].shape, dtype=torch.float64, device=DEV)
    for b in range(B):
        L, keep = lens[b], min(lens[b], case["keep"])
        at = torch.arange(L, device=DEV)
        page, off = st["table"][b, at // P].long(), at % P
        for h in range(H):
            w, born = st["weight"][page, h, off].double(), st["born"][page, h, off]
            fresh = born > born.max() - case["recent"]
            w_first = torch.where(fresh, born.double() + 1e30, w)
            stay = torch.zeros(L, dtype=torch.bool, device=DEV)
            stay[torch.sort(-w_first, stable=True).indices[:keep]] = True
            holes, movers = torch.nonzero(~stay[:keep])[:, 0], torch.nonzero(stay[keep:])[:, 0] + keep
            held = at[:keep].clone()
            held[holes] = movers
            weight[page[:keep], h, off[:keep]] = w[held]
            if not holes.numel():
                continue
            for codes, scales in ((k, ks), (v, vs)):
                val = codes[page, h, off] * scales[page, h, off // BLOCK][:, None]
                now = torch.cat((held, at[keep:]))[:min(L, up(keep, BLOCK) * BLOCK)]  # to the end of the last block that keeps a token
                top = val[now].abs().max(-1).values
                n = up(now.numel(), BLOCK)
                top = torch.cat((top, torch.zeros(n * BLOCK - now.numel(), dtype=torch.float64, device=DEV))).view(n, BLOCK).max(-1).values
                takes = torch.zeros(n, dtype=torch.bool, device=DEV)
                takes[holes // BLOCK] = True
                e = torch.ceil(torch.log2(top / 448) - 1e-12).clamp(min=-120)
                s = torch.where(takes, torch.exp2(torch.where(448 * torch.exp2(e) < top, e + 1, e)), scales[page, h, off // BLOCK][::BLOCK][:n])
                anew = takes[at[:now.numel()] // BLOCK]
                put = e4m3(val[now] / s[at[:now.numel()] // BLOCK][:, None])
                p, o = page[:now.numel()], off[:now.numel()]
                codes[p[anew], h, o[anew]] = put[anew]
                scales[p[::BLOCK], h, o[::BLOCK] // BLOCK] = s
    return dict(frm=None, weight=weight, born=None, k=k, v=v, k_scale=ks, v_scale=vs)
