"""The 4-bit decoder (weights and paged cache) against the same arithmetic in
64 bits, step by step, and its cache against the quantiser."""
import numpy as np
import pytest
import torch

from oracle import kv4 as o4

pytestmark = pytest.mark.gpu

HID, LAYERS, H, HKV, INTER, VOCAB, D = 256, 2, 4, 2, 256, 500, 128


def num(t):
    return t.double().cpu().numpy()


def rope(x, pos, base):
    """x [rows, heads, D], rotate-half pairs (i, i + D/2) turned by pos base^(-2i/D)."""
    a = pos[:, None] * base ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    lo, hi = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


class Plain:
    """One sequence's decoder in 64 bits: weights and cached rows as held in 4
    bits, everything else unrounded."""

    def __init__(self, W, group, base, eps):
        held = lambda w: (lambda c, s: (c * s[:, None]).reshape(w.shape))(*o4.quantise(num(w).reshape(w.shape[0] // group, group, -1), 1))
        self.W = {k: (num(v) if k in ("embed", "final_norm") else held(v)) for k, v in W.items() if k != "layers"}
        self.L = [{k: (num(v) if "norm" in k else held(v)) for k, v in w.items()} for w in W["layers"]]
        self.K, self.V, self.base, self.eps = [[] for _ in self.L], [[] for _ in self.L], base, eps

    def norm(self, x, w):
        return x / np.sqrt((x * x).mean() + self.eps) * w

    def step(self, tok):
        x = self.W["embed"][tok]
        for l, w in enumerate(self.L):
            h = self.norm(x, w["attn_norm"])
            pos = np.array([len(self.K[l])])
            q = rope((h @ w["wq"]).reshape(1, H, D), pos, self.base)[0]
            kv = (h @ w["wkv"]).reshape(2, HKV, D)
            k = rope(kv[0][None], pos, self.base)[0]
            out = np.zeros((H, D))
            for i in range(H):
                g = i // (H // HKV)
                ks = np.array([r[g] for r in self.K[l]] + [k[g]])
                vs = np.array([r[g] for r in self.V[l]] + [kv[1][g]])
                z = ks @ q[i] * D ** -0.5
                p = np.exp(z - z.max())
                out[i] = p @ vs / p.sum()
            x = x + out.reshape(-1) @ w["wo"]
            h = self.norm(x, w["mlp_norm"])
            gu = h @ w["wgu"]
            x = x + (gu[:INTER] / (1 + np.exp(-gu[:INTER])) * gu[INTER:]) @ w["wd"]
        return self.norm(x, self.W["final_norm"]) @ self.W["lm_head"]

    def keep(self, l, k, v):
        for rows, r in ((self.K[l], k), (self.V[l], v)):
            c, s = o4.quantise(r)
            rows.append(c * s[:, None])


@pytest.fixture(scope="module")
def weights():
    from paper_2502_17139_gb300 import synth
    from paper_2502_17139_gb300.decoder import DecoderShape
    shape = DecoderShape(hidden=HID, layers=LAYERS, H=H, Hkv=HKV, inter=INTER, vocab=VOCAB)
    return shape, synth.decoder_weights(HID, LAYERS, H, HKV, D, INTER, VOCAB, 3, device="cuda")


def test_steps_follow_the_plain_decoder(weights):
    """Logits of 40 single-token steps of three sequences over pages of 16.
    The GPU rounds to bf16 (2^-8 at most, about a third of that in the mean)
    some ten times a layer and three times outside; independent errors of 23
    roundings add up to about 5 * 2^-8 / 3 of the logits' norm.  Bound: 4 times
    that.  The plain decoder keeps the GPU's own new keys and values, in 4 bits
    by its own quantiser: quantising rows that differ by a rounding puts
    numbers on other sides of ties, a step of the scale each, and two plain
    decoders that differ in roundings alone then drift apart by 2 to 4%."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    dec = Q4Decoder(shape, W, 3, 12, 4, page_size=16, group=64)
    plain = [Plain(W, 64, shape.rope_base, shape.eps) for _ in range(3)]
    rng = np.random.default_rng(4)
    for t in range(40):
        tok = rng.integers(0, VOCAB, 3).astype(np.int32)
        got = num(dec.forward(torch.from_numpy(tok).cuda().view(3, 1)))[:, 0]
        want = np.stack([p.step(int(x)) for p, x in zip(plain, tok)])
        err = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
        assert err.max() < 4 * 5 * 2.0 ** -8 / 3, (t, err)
        k_new, v_new = [num(k) for k in dec.k_new], [num(v) for v in dec.v_new]
        for l in range(LAYERS):
            for b, p in enumerate(plain):
                p.keep(l, k_new[l][b, :, 0], v_new[l][b, :, 0])
        dec.append()
        # the rows just written stand for the step's own keys, quantised
        slot = dec.plan["slot"].clone()
        for l in range(LAYERS):
            k, _ = fc.fc_kv4_read(dec.caches[l], slot)
            c, s = o4.quantise(k_new[l][:, :, 0])
            assert np.array_equal(num(k), o4.bf16_round(c * s[..., None]))
    assert fc.fc_get_error() == "FC_OK"
    assert dec.kv_len[dec.cur].tolist() == [40] * 3 and dec.n_free[dec.cur].item() == 12 - 9
    dec.release(torch.tensor([0, 17, 40], dtype=torch.int32, device="cuda"))
    assert dec.kv_len[dec.cur].tolist() == [0, 17, 40] and dec.n_free[dec.cur].item() == 12 - 5


def test_a_chunk_equals_its_tokens_one_by_one(weights):
    """Four tokens in one step (causal) against four steps: the same caches'
    lengths, and logits that differ by the cache's quantisation and roundings
    alone; the first token's, which no cached token precedes, by roundings of
    the same sums (none: the kernels treat a row alike)."""
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    tok = torch.randint(0, VOCAB, (2, 4), dtype=torch.int32, device="cuda")
    a = Q4Decoder(shape, W, 2, 8, 4, nodes=4, page_size=16)
    whole = a.forward(tok).clone()
    a.append()
    b = Q4Decoder(shape, W, 2, 8, 4, page_size=16)
    for t in range(4):
        one = b.forward(tok[:, t:t + 1].contiguous()).clone()
        b.append()
        err = (one[:, 0].double() - whole[:, t].double()).norm(dim=1) / one[:, 0].double().norm(dim=1)
        assert err.max() < (2.0 ** -6 if t == 0 else 0.5)
    assert a.kv_len[a.cur].tolist() == b.kv_len[b.cur].tolist() == [4, 4]


def test_an_accepted_path_is_kept_and_rows_are_limited(weights):
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    dec = Q4Decoder(shape, W, 2, 8, 4, nodes=6, page_size=16)
    mask = torch.tensor([1, 3, 5, 11, 21, 37], dtype=torch.int64, device="cuda").view(1, 6, 1).repeat(2, 1, 1).contiguous()
    pos = torch.tensor([[0, 1, 1, 2, 2, 2]] * 2, dtype=torch.int32, device="cuda")
    dec.forward(torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6), pos=pos, mask=mask)
    path = torch.tensor([[0, 2, 5, -1], [0, -1, -1, -1]], dtype=torch.int32, device="cuda")
    dec.append(torch.tensor([3, 1], dtype=torch.int32, device="cuda"), path=path)
    assert dec.kv_len[dec.cur].tolist() == [3, 1]
    k, v = fc.fc_kv4_read(dec.caches[1], dec.plan["slot"][:4].contiguous())
    want = dec.v_new[1].transpose(1, 2)[[0, 0, 0, 1], [0, 2, 5, 0]]
    c, s = o4.quantise(num(want))
    assert np.array_equal(num(v), o4.bf16_round(c * s[..., None]))
    assert dec.plan["slot"][4:].tolist() == [-1] * 8
    with pytest.raises(ValueError):
        Q4Decoder(shape, W, 17, 17, 1)


def test_greedy_decoding_takes_the_largest_logit(weights):
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    tok = torch.tensor([5, 7], dtype=torch.int32, device="cuda")
    a, b = (Q4Decoder(shape, W, 2, 8, 4, page_size=16) for _ in range(2))
    got = a.generate(tok, 20)
    for t in range(20):
        tok = b.forward(tok.view(2, 1)).view(2, -1).float().argmax(1).to(torch.int32)
        b.append()
        assert torch.equal(got[:, t], tok)
    assert a.kv_len[a.cur].tolist() == [20, 20]


def test_a_captured_step_is_good_for_every_step(weights):
    """forward() and append() captured once and replayed follow the same calls
    made one by one, over page boundaries and a release."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    a, b = (Q4Decoder(shape, W, 2, 8, 4, page_size=16) for _ in range(2))
    tok = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(9)
    g = None
    for t in range(40):
        if t == 25:
            for d in (a, b):
                d.release(torch.tensor([3, 19], dtype=torch.int32, device="cuda"))
        tok.copy_(torch.randint(0, VOCAB, (2, 1), generator=gen, dtype=torch.int32, device="cuda"))
        want = b.forward(tok).clone()
        b.append()
        if t < 2:  # the steps before the capture
            got = a.forward(tok)
            a.append()
        else:
            if g is None:
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    got = a.forward(tok)
                    a.append()
            g.replay()
        assert torch.equal(got, want), t
    assert a.kv_len[a.cur].tolist() == b.kv_len[b.cur].tolist() == [18, 34]
    assert fc.fc_get_error() == "FC_OK"


def test_generate_says_when_the_pool_is_empty(weights):
    """A sequence that finds no page cannot go on: no tokens, but an error."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    tok = torch.tensor([5, 7], dtype=torch.int32, device="cuda")
    dec = Q4Decoder(shape, W, 2, 3, 4, page_size=16)  # pages for 32 and 16 tokens
    with pytest.raises(fc.FastCoderError) as e:
        dec.generate(tok, 20)
    assert e.value.status == "FC_ERR_CAPACITY"
    assert sorted(dec.kv_len[dec.cur].tolist()) == [16, 20]
    assert fc.fc_get_error() == "FC_OK"
    dec.release(torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert dec.generate(tok, 16).shape == (2, 16)


@pytest.mark.parametrize("nodes", [2, 4])
def test_chunks_follow_the_plain_decoder(weights, nodes):
    """Chunks of several tokens (causal among themselves) over a growing cache
    against the plain decoder, which sees a chunk's own rows as they are and the
    cached ones in 4 bits; the bound is the one of single-token steps."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    dec = Q4Decoder(shape, W, 2, 8, 4, nodes=nodes, page_size=16, group=64)
    plain = [Plain(W, 64, shape.rope_base, shape.eps) for _ in range(2)]
    rng = np.random.default_rng(6)
    for t in range(0, 24, nodes):
        tok = rng.integers(0, VOCAB, (2, nodes)).astype(np.int32)
        got = num(dec.forward(torch.from_numpy(tok).cuda()))
        k_new, v_new = [num(k) for k in dec.k_new], [num(v) for v in dec.v_new]
        for b, p in enumerate(plain):
            for i in range(nodes):
                want = p.step(int(tok[b, i]))
                err = np.linalg.norm(got[b, i] - want) / np.linalg.norm(want)
                assert err < 4 * 5 * 2.0 ** -8 / 3, (t, b, i, err)
                for l in range(LAYERS):  # the chunk's own rows, unquantised
                    p.K[l].append(k_new[l][b, :, i])
                    p.V[l].append(v_new[l][b, :, i])
            for l in range(LAYERS):
                del p.K[l][-nodes:], p.V[l][-nodes:]
                for i in range(nodes):
                    p.keep(l, k_new[l][b, :, i], v_new[l][b, :, i])
        dec.append()
    assert dec.kv_len[dec.cur].tolist() == [24, 24] and fc.fc_get_error() == "FC_OK"
