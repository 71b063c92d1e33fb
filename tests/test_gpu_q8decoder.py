"""The decoder over a cache in 8 bits, with normed queries and keys and a token
budget, against the same arithmetic in 64 bits over the cache as it is, step by
step; its cache, weights and evictions against the oracle."""
import numpy as np
import pytest
import torch

from oracle import kv4 as o4
from oracle import kv8 as o8

pytestmark = pytest.mark.gpu

HID, LAYERS, H, HKV, INTER, VOCAB, D, PAGE = 256, 2, 4, 2, 256, 500, 128, 16


def num(t):
    return t.double().cpu().numpy()


@pytest.fixture(scope="module")
def weights():
    from paper_2502_17139_gb300 import synth
    from paper_2502_17139_gb300.decoder import DecoderShape
    shape = DecoderShape(hidden=HID, layers=LAYERS, H=H, Hkv=HKV, inter=INTER, vocab=VOCAB)
    W = synth.decoder_weights(HID, LAYERS, H, HKV, D, INTER, VOCAB, 5, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    for w in W["layers"]:
        w["q_norm"], w["k_norm"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16() for _ in range(2))
    return shape, W


class Plain:
    """The decoder in 64 bits: weights as held in 4 bits, cached rows as the GPU
    holds them."""

    def __init__(self, shape, W, group):
        held = lambda w: (lambda c, s: (c * s[:, None]).reshape(w.shape))(*o4.quantise(num(w).reshape(w.shape[0] // group, group, -1), 1))
        self.W = {k: (num(v) if k in ("embed", "final_norm") else held(v)) for k, v in W.items() if k != "layers"}
        self.L = [{k: (num(v) if "norm" in k else held(v)) for k, v in w.items()} for w in W["layers"]]
        self.s = shape

    def norm(self, x, w):
        return x / np.sqrt((x * x).mean() + self.s.eps) * w

    def step(self, tok, pos, cached):
        """cached(layer, head) -> (K, V) of the sequence.  Logits, and the weights
        that the cached tokens received by layer and head."""
        x, got = self.W["embed"][tok], []
        for l, w in enumerate(self.L):
            h = self.norm(x, w["attn_norm"])
            at = np.array([[float(pos)]])
            q = o8.norm_rope((h @ w["wq"]).reshape(1, 1, H, D), w["q_norm"], at, self.s.rope_base, self.s.eps)[0][0, 0]
            kv = (h @ w["wkv"]).reshape(2, HKV, D)
            k = o8.norm_rope(kv[0][None, None], w["k_norm"], at, self.s.rope_base, self.s.eps)[0][0, 0]
            out, received = np.zeros((H, D)), []
            for g in range(HKV):
                K, V = cached(l, g)
                ks, vs = np.concatenate((K, k[g][None])), np.concatenate((V, kv[1][g][None]))
                rows = slice(g * (H // HKV), (g + 1) * (H // HKV))
                out[rows], p, _, _ = o8.attend(q[rows], ks, vs, np.ones((H // HKV, len(ks)), bool), D ** -0.5)
                received.append(p[:, :-1].sum(0))
            got.append(received)
            x = x + out.reshape(-1) @ w["wo"]
            h = self.norm(x, w["mlp_norm"])
            gu = h @ w["wgu"]
            x = x + (gu[:INTER] / (1 + np.exp(-gu[:INTER])) * gu[INTER:]) @ w["wd"]
        return self.norm(x, self.W["final_norm"]) @ self.W["lm_head"], got


def arrays(cache):
    return [t.cpu().numpy().copy() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]


@pytest.mark.parametrize("captured", [False, True])
def test_steps_with_a_budget_follow_the_plain_decoder(weights, captured):
    """60 single-token steps of three sequences, cut to 24 tokens whenever they
    hold 32.  The GPU rounds to bf16 (2^-8 at most, about a third of that in the
    mean) some eleven times a layer and three times outside: 25 independent
    errors add up to about 5 * 2^-8 / 3 of the logits' norm.  Bound: 4 times
    that.  Weights: those of a step follow scores whose relative error is the
    rows' (some 2^-6 of scores of about 1); they are compared with 2^-4 of the
    largest."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    KEEP, RECENT, FULL = 24, 6, 32
    dec = Q4Decoder(shape, W, 3, 12, 4, page_size=PAGE, group=64, cache_bits=8, keep=KEEP, recent=RECENT)
    plain = Plain(shape, W, 64)
    rng = np.random.default_rng(4)
    tok = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    step = lambda: (dec.forward(tok), dec.append())
    if captured:
        warm = Q4Decoder(shape, W, 3, 12, 4, page_size=PAGE, group=64, cache_bits=8, keep=KEEP, recent=RECENT)
        warm.forward(tok)
        warm.append()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        step = graph.replay
    held = 0
    for t in range(60):
        t_np = rng.integers(0, VOCAB, 3).astype(np.int32)
        tok.copy_(torch.from_numpy(t_np).view(3, 1))
        table, before = dec.pages.table.cpu().numpy(), [arrays(c) for c in dec.caches]
        was = [(num(x.weight), x.born.cpu().numpy()) for x, _ in dec.tracks]
        step()
        got = num(dec.logits)
        after = [arrays(c) for c in dec.caches]
        weight = [num(x.weight) for x, _ in dec.tracks]
        slot = dec.plan["slot"].cpu().numpy()
        i = np.arange(held)
        for b in range(3):
            cached = lambda l, g: tuple(o8.cached(before[l], w, table[b], held, g) for w in range(2))
            want, received = plain.step(int(t_np[b]), t, cached)
            assert np.linalg.norm(got[b] - want) < 4 * 5 * 2.0 ** -8 / 3 * np.linalg.norm(want), (t, b)
            if held:
                p, o = table[b][i // PAGE], i % PAGE
                for l in range(LAYERS):
                    for g in range(HKV):
                        added = weight[l][p, g, o] - was[l][0][p, g, o]
                        assert np.abs(added - received[l][g]).max() <= 2.0 ** -4 * received[l][g].max() + 2.0 ** -20 * was[l][0].max()
        k_new, v_new = ([num(x)[:, :, 0] for x in y] for y in (dec.k_new, dec.v_new))
        for l in range(LAYERS):  # the step's rows in the pages, their weights and positions
            o8.write(before[l], k_new[l], v_new[l], slot)
            for x, y in zip(before[l], after[l]):
                assert np.array_equal(x, y)
            born = dec.tracks[l][0].born.cpu().numpy()
            assert (born[slot // PAGE, :, slot % PAGE] == t).all() and (weight[l][slot // PAGE, :, slot % PAGE] == 0).all()
        held += 1
        assert dec.kv_len[0].tolist() == [held] * 3
        if held == FULL:
            table = dec.pages.table.cpu().numpy()
            tracks = [[x.weight.cpu().numpy().copy(), x.born.cpu().numpy().copy()] for x, _ in dec.tracks]
            dec.evict()
            for l in range(LAYERS):
                outs = [x.copy() for x in tracks[l]]
                o8.evict(after[l], table, [FULL] * 3, [KEEP] * 3, RECENT, tracks[l], outs, KEEP)
                for x, y in zip(after[l], arrays(dec.caches[l])):
                    assert np.array_equal(x, y)
                j = np.arange(KEEP)
                for b in range(3):
                    p, o = table[b][j // PAGE], j % PAGE
                    born = dec.tracks[l][0].born.cpu().numpy()[p, :, o]
                    assert np.array_equal(born, outs[1][p, :, o])
                    assert np.array_equal(dec.tracks[l][0].weight.cpu().numpy()[p, :, o], outs[0][p, :, o])
                    for g in range(HKV):  # the newest are there, no token twice
                        assert set(range(t - RECENT + 1, t + 1)) <= set(born[:, g]) and len(set(born[:, g])) == KEEP
            held = KEEP
            assert dec.kv_len[0].tolist() == [KEEP] * 3 and dec.ahead.tolist() == [t + 1 - KEEP] * 3
    assert fc.fc_get_error() == "FC_OK"


def test_four_and_eight_bits_without_norms(weights):
    """Without norms of queries and keys both caches serve the same decoder: their
    logits differ by the caches' rounding, and at the first step not at all."""
    from paper_2502_17139_gb300 import synth
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, _ = weights
    W = synth.decoder_weights(HID, LAYERS, H, HKV, D, INTER, VOCAB, 3, device="cuda")
    a, b = (Q4Decoder(shape, W, 2, 8, 4, page_size=PAGE, cache_bits=n) for n in (4, 8))
    for t in range(20):
        tok = torch.randint(0, VOCAB, (2, 1), dtype=torch.int32, device="cuda")
        x, y = a.forward(tok).double(), b.forward(tok).double()
        a.append()
        b.append()
        assert (x - y).norm() < (2.0 ** -6 if t == 0 else 0.6) * x.norm()


def test_refusals(weights):
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    for kw in (dict(cache_bits=5), dict(keep=8), dict(cache_bits=8, keep=-1), dict(cache_bits=8, recent=-1)):
        with pytest.raises(ValueError):
            Q4Decoder(shape, W, 1, 4, 4, page_size=PAGE, **kw)
    with pytest.raises(ValueError):
        Q4Decoder(shape, W, 1, 4, 4, page_size=PAGE, cache_bits=8).evict()
