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


def rope(x, pos, base):
    """x [heads, D] turned by pos."""
    a = pos * base ** (-2.0 * np.arange(D // 2) / D)
    lo, hi = x[:, :D // 2], x[:, D // 2:]
    return np.concatenate((lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)), 1)


class PlainTree(Plain):
    """The decoder in 64 bits over some nodes at once, with or without norms of queries and keys."""

    def heads(self, x, w, pos):
        if w is not None:
            x = x / np.sqrt((x * x).mean(1, keepdims=True) + self.s.eps) * w
        return rope(x, pos, self.s.rope_base)

    def step(self, tok, pos, sees, cached):
        """tok, pos [m], sees [m, m]: logits [m], and by layer and head the weights that the cached tokens received."""
        m, received = len(tok), []
        x = self.W["embed"][tok]
        for l, w in enumerate(self.L):
            h = np.stack([self.norm(r, w["attn_norm"]) for r in x])
            q = np.stack([self.heads(r.reshape(H, D), w.get("q_norm"), p) for r, p in zip(h @ w["wq"], pos)])
            kv = (h @ w["wkv"]).reshape(m, 2, HKV, D)
            k = np.stack([self.heads(r, w.get("k_norm"), p) for r, p in zip(kv[:, 0], pos)])
            out, got = np.zeros((m, H, D)), []
            for g in range(HKV):
                K, V = cached(l, g)
                seen = np.concatenate((np.ones((m, len(K)), bool), sees), 1)
                total = np.zeros(len(K))
                for i in range(g * (H // HKV), (g + 1) * (H // HKV)):
                    out[:, i], p, _, _ = o8.attend(q[:, i], np.concatenate((K, k[:, g])), np.concatenate((V, kv[:, 1, g])), seen, D ** -0.5)
                    total += p[:, :len(K)].sum(0)
                got.append(total)
            received.append(got)
            x = x + out.reshape(m, -1) @ w["wo"]
            h = np.stack([self.norm(r, w["mlp_norm"]) for r in x])
            gu = h @ w["wgu"]
            x = x + (gu[:, :INTER] / (1 + np.exp(-gu[:, :INTER])) * gu[:, INTER:]) @ w["wd"]
        return np.stack([self.norm(r, self.W["final_norm"]) for r in x]) @ self.W["lm_head"], received


@pytest.mark.parametrize("normed,keep,steps", [(True, 24, 80), (False, 24, 80), (False, 0, 30)])
def test_trees_with_accepted_paths_and_evictions_follow_the_plain_decoder(weights, normed, keep, steps):
    """Draft trees of up to four nodes of three sequences: each step a path of none to all of them is kept (rows
    head-major by src, several a block, some left out), and whoever holds 32 tokens or more is cut to 24.  Logits,
    weights and bounds as in test_steps_with_a_budget_follow_the_plain_decoder; written rows, weights and positions
    equal to the oracle's."""
    from paper_2502_17139_gb300 import fastcoder as fc
    from paper_2502_17139_gb300.q4decoder import Q4Decoder
    shape, W = weights
    if not normed:
        W = dict(W, layers=[{k: v for k, v in w.items() if k not in ("q_norm", "k_norm")} for w in W["layers"]])
    B, N, RECENT, FULL = 3, 4, 6, 32
    dec = Q4Decoder(shape, W, B, 15, 5, nodes=N, page_size=PAGE, group=64, cache_bits=8, keep=keep, recent=RECENT if keep else 0)
    plain = PlainTree(shape, W, 64)
    rng = np.random.default_rng(8)
    held, ahead, evicted = np.zeros(B, int), np.zeros(B, int), 0
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    for t in range(steps):
        nodes = rng.integers(1, N + 1, B) if t % 3 else np.full(B, N)
        tok, depth, sees = rng.integers(0, VOCAB, (B, N)), np.zeros((B, N), int), np.zeros((B, N, N), bool)
        path, accepted = np.full((B, N), -1), np.zeros(B, int)
        for b in range(B):
            parent = [-1] + [int(rng.integers(0, i)) for i in range(1, N)]
            for i in range(N):
                if i:
                    sees[b, i], depth[b, i] = sees[b, parent[i]], depth[b, parent[i]] + 1
                sees[b, i, i] = True
            tip = int(rng.integers(0, nodes[b]))
            line = [j for j in range(N) if sees[b, tip, j]]
            accepted[b] = rng.integers(0, len(line) + 1)
            path[b, :len(line)] = line
        pos = held[:, None] + ahead[:, None] + depth
        bits = (sees * (1 << np.arange(N))).sum(-1)[..., None]
        table, before = dec.pages.table.cpu().numpy(), [arrays(c) for c in dec.caches]
        was = [(num(x.weight), x.born.cpu().numpy()) for x, _ in dec.tracks] if keep else None
        got = num(dec.forward(i32(tok), i32(pos), torch.from_numpy(bits.astype(np.int64)).cuda(), i32(nodes)))
        added = [num(x.weight) - y[0] for (x, _), y in zip(dec.tracks, was)] if keep else None
        for b in range(B):
            m, L = nodes[b], held[b]
            cached = lambda l, g: tuple(o8.cached(before[l], w, table[b], L, g) for w in range(2))
            want, received = plain.step(tok[b, :m], pos[b, :m], sees[b, :m, :m], cached)
            for i in range(m):
                assert np.linalg.norm(got[b, i] - want[i]) < 4 * 5 * 2.0 ** -8 / 3 * np.linalg.norm(want[i]), (t, b, i)
            if keep and L:
                j = np.arange(L)
                p, o = table[b][j // PAGE], j % PAGE
                for l in range(LAYERS):
                    for g in range(HKV):
                        assert np.abs(added[l][p, g, o] - received[l][g]).max() <= 2.0 ** -4 * received[l][g].max() + 2.0 ** -20 * was[l][0].max()
        tracks = [[x.weight.cpu().numpy().copy(), x.born.cpu().numpy().copy()] for x, _ in dec.tracks] if keep else None
        dec.append(i32(accepted), path=i32(path))
        slot, src, seq, place = (dec.plan[x].cpu().numpy() for x in ("slot", "src", "seq", "pos"))
        assert (slot >= 0).sum() == accepted.sum()
        for l in range(LAYERS):
            k, v = (num(x[l]).transpose(0, 2, 1, 3).reshape(B * N, HKV, D) for x in (dec.k_new, dec.v_new))
            o8.write(before[l], k, v, slot, src, tracks[l] if keep else None, place + ahead[np.maximum(seq, 0)])
            for x, y in zip(before[l], arrays(dec.caches[l])):
                assert np.array_equal(x, y)
            if keep:
                assert np.array_equal(tracks[l][0], dec.tracks[l][0].weight.cpu().numpy()) and np.array_equal(tracks[l][1], dec.tracks[l][0].born.cpu().numpy())
        held += accepted
        assert dec.kv_len[0].tolist() == held.tolist()
        if keep and held.max() >= FULL:
            table, evicted = dec.pages.table.cpu().numpy(), evicted + 1
            dec.evict()
            for l in range(LAYERS):
                after, outs = before[l], [x.copy() for x in tracks[l]]
                o8.evict(after, table, held, [keep] * B, RECENT, tracks[l], outs, keep)
                for x, y in zip(after, arrays(dec.caches[l])):
                    assert np.array_equal(x, y)
                for b in range(B):
                    j = np.arange(min(keep, held[b]))
                    p, o = table[b][j // PAGE], j % PAGE
                    for x, y in zip(outs, (dec.tracks[l][0].weight, dec.tracks[l][0].born)):
                        assert np.array_equal(x[p, :, o], y.cpu().numpy()[p, :, o])
            ahead += held - np.minimum(held, keep)
            held = np.minimum(held, keep)
            assert dec.kv_len[0].tolist() == held.tolist() and dec.ahead.tolist() == ahead.tolist()
    assert fc.fc_get_error() == "FC_OK" and (evicted > 1) == bool(keep)
