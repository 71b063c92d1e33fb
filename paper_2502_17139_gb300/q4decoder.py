"""Decoding in four bits: a LLaMA-family decoder whose weights are held in 4
bits (fc_w4_pack) and whose KV cache is paged and held in 4 bits (Kv4Cache) or
in 8 (Kv8Cache), for the few rows of a decoding step: single tokens of up to 16
sequences, or one small draft tree (batch * nodes <= 16).  Weights with
``q_norm`` and ``k_norm`` in a layer norm the queries and keys of each head.

A step: forward() runs the rows against the caches, with the new tokens' own
keys and values in bf16; append() plans where the kept ones go
(fc_kv_pages_plan, once) and quantises them into every layer's pages
(fc_kv4_write).  All on the current stream, no host round trip.  Both read and
write the same tensors at every step, so that a step captured in a CUDA graph
is good for all of them.  A cache in 8 bits can be kept to a budget (``keep``):
forward() adds up the weight that each cached token received, and evict() cuts
every sequence down to the tokens that received most (fc_kv8_evict).  Every
forward() counts, a tree's rejected nodes and a call that no append() follows
(a warm-up before a capture) among them.

    python -m paper_2502_17139_gb300.q4decoder [batch] [context] [cache bits]

times single-token steps of the 1.3B shape with random weights.
"""
from __future__ import annotations

import torch

from . import fastcoder as fc
from .decoder import DecoderShape

MAX_ROWS = 16


class Q4Decoder:
    """W: bf16 weights in synth.decoder_weights' layout, quantised here (one
    scale for ``group`` weights).  ``nodes`` new tokens a sequence and step.
    The pool has ``n_pages`` pages of ``page_size`` tokens; a sequence holds at
    most ``max_pages``.  ``cache_bits`` 4 or 8; with 8, ``keep`` > 0: evict()
    leaves a sequence that many tokens, the last ``recent`` positions' among them."""

    def __init__(self, shape: DecoderShape, W, batch, n_pages, max_pages, nodes=1, page_size=64, group=128,
                 device="cuda", cache_bits=4, keep=0, recent=0):
        if batch * nodes > MAX_ROWS:
            raise ValueError(f"a step has at most {MAX_ROWS} rows")
        if cache_bits not in (4, 8):
            raise ValueError("cache_bits must be 4 or 8")
        if keep < 0 or recent < 0 or (keep and cache_bits == 4):
            raise ValueError("keep and recent count tokens of a cache in 8 bits")
        if keep and nodes * (shape.H // shape.Hkv) > 16:
            raise ValueError("weights need at most 16 rows a kv head")
        s = shape
        self.s, self.B, self.n = s, batch, nodes
        pack = lambda w: fc.fc_w4_pack(w.contiguous(), group)
        self.embed, self.final_norm, self.lm_head = W["embed"], W["final_norm"], pack(W["lm_head"])
        self.layers = [dict(attn_norm=w["attn_norm"], mlp_norm=w["mlp_norm"], wq=pack(w["wq"]), wkv=pack(w["wkv"]),
                            wo=pack(w["wo"]), wgu=pack(w["wgu"]), wd=pack(w["wd"])) for w in W["layers"]]
        i32 = dict(dtype=torch.int32, device=device)
        self.pages = fc.KvPages(page_size, torch.zeros((batch, max_pages), **i32),
                                torch.arange(n_pages - 1, -1, -1, **i32))
        self.bits, self.keep, self.recent = cache_bits, keep, recent
        kind = fc.Kv4Cache if cache_bits == 4 else fc.Kv8Cache
        self.caches = [kind.empty(n_pages, s.Hkv, page_size, s.D, device) for _ in range(s.layers)]
        # lengths and the free count: the current ones, and a plan's results, which
        # are copied back (a plan's outputs are not its inputs)
        self.state = torch.zeros((2, batch + 1), **i32)
        self.state[0, batch] = n_pages
        self.kv_len = [self.state[0, :batch], self.state[1, :batch]]
        self.n_free = [self.state[0, batch:], self.state[1, batch:]]
        self.cur = 0  # the place of the current ones
        self.plan = fc.kv_pages_outputs(batch, batch * nodes, device, src=True)
        R = batch * nodes
        bf = lambda *shape_: torch.empty(shape_, dtype=torch.bfloat16, device=device)
        self.x, self.h, self.o = bf(R, s.hidden), bf(R, s.hidden), bf(R, s.hidden)
        self.q, self.attn, self.kv = bf(batch, nodes, s.H, s.D), bf(batch, nodes, s.H, s.D), bf(R, 2 * s.Hkv * s.D)
        self.gu, self.act, self.logits = bf(R, 2 * s.inter), bf(R, s.inter), bf(R, s.vocab)
        self.k_new = [bf(batch, s.Hkv, nodes, s.D) for _ in range(s.layers)]
        self.v_new = [bf(batch, s.Hkv, nodes, s.D) for _ in range(s.layers)]
        if cache_bits == 4:
            self.ws = fc.kv4_attn_workspace(batch, nodes, s.H, s.Hkv, device)
        else:
            self.ws = fc.kv8_attn_workspace(batch, nodes, s.H, s.Hkv, device, max_pages * page_size if keep else 0)
        if "q_norm" in W["layers"][0]:
            self.q_raw = bf(batch, nodes, s.H, s.D)
            for mine, w in zip(self.layers, W["layers"]):
                mine.update(q_norm=w["q_norm"], k_norm=w["k_norm"])
        # how far a sequence's positions are ahead of its cached tokens
        self.ahead = torch.zeros(batch, **i32)
        if keep:
            self.tracks = [[fc.Kv8Track.empty(c), fc.Kv8Track.empty(c)] for c in self.caches]
            self.keeps = torch.full((batch,), keep, **i32)
            self.from_ = torch.empty((batch, s.Hkv, keep), **i32)
            self.evict_ws = fc.kv8_evict_workspace(batch, s.Hkv, keep, device)
        self.steps = torch.arange(nodes, **i32)[None, :]
        self.ones = torch.full((batch,), nodes, **i32)

    def forward(self, tok, pos=None, mask=None, n_nodes=None):
        """tok [B, n] int32 -> logits [B, n, vocab].  pos [B, n] (None: the
        tokens follow the cache in order), mask [B, n, 1] int64 ancestor bits
        (None: each sees those before it), n_nodes [B].  With ``keep`` the cached
        tokens' weights grow by what this call gives them, each time it runs."""
        s, B, n, kv_len = self.s, self.B, self.n, self.kv_len[0]
        if pos is None:
            pos = (kv_len + self.ahead if self.keep else kv_len)[:, None] + self.steps
        fc.fc_embed(tok.reshape(-1), self.embed, self.x)
        r = None
        for l, w in enumerate(self.layers):
            fc.fc_add_rmsnorm(self.x, r, w["attn_norm"], self.h, s.eps)
            normed = "q_norm" in w
            fc.fc_w4_matvec(self.h, w["wq"], out=(self.q_raw if normed else self.q).view(B * n, -1))
            fc.fc_w4_matvec(self.h, w["wkv"], out=self.kv)
            if normed:
                kv = self.kv.view(B, n, 2, s.Hkv, s.D)
                fc.fc_qk_norm_rope(self.q_raw, kv[:, :, 0], kv[:, :, 1], w["q_norm"], w["k_norm"], pos, s.rope_base, s.eps,
                                   out=(self.q, self.k_new[l], self.v_new[l]))
            else:
                fc.fc_rope(self.q, pos, s.rope_base, out=self.q)
                stride = 2 * s.Hkv * s.D
                fc.fc_rope_heads(self.kv, 0, stride, self.k_new[l], B, n, s.Hkv, s.D, pos, s.rope_base)
                fc.fc_rope_heads(self.kv, s.Hkv * s.D, stride, self.v_new[l], B, n, s.Hkv, s.D, pos, 0.0)
            if self.bits == 4:
                fc.fc_kv4_attn(self.q, self.caches[l], self.pages.table, kv_len, self.k_new[l], self.v_new[l], mask, n_nodes,
                               out=self.attn, workspace=self.ws)
            else:
                fc.fc_kv8_attn(self.q, self.caches[l], self.pages.table, kv_len, self.k_new[l], self.v_new[l], mask, n_nodes,
                               out=self.attn, workspace=self.ws, weight=self.tracks[l][0].weight if self.keep else None)
            fc.fc_w4_matvec(self.attn.view(B * n, -1), w["wo"], out=self.o)
            fc.fc_add_rmsnorm(self.x, self.o, w["mlp_norm"], self.h, s.eps)
            fc.fc_w4_matvec(self.h, w["wgu"], out=self.gu)
            fc.fc_silu_mul(self.gu, self.act)
            fc.fc_w4_matvec(self.act, w["wd"], out=self.o)
            r = self.o
        fc.fc_add_rmsnorm(self.x, r, self.final_norm, self.h, s.eps)
        fc.fc_w4_matvec(self.h, self.lm_head, out=self.logits)
        return self.logits.view(B, n, s.vocab)

    def append(self, n_keep=None, path=None):
        """Keeps the step's first n_keep[b] tokens of each sequence (None: all),
        or those of an accepted path [B, path_cap], in the caches.  A sequence
        whose tokens find no free page keeps its length and none of them, and
        fc_get_error() says FC_ERR_CAPACITY."""
        out = dict(self.plan, kv_len=self.kv_len[1], n_free=self.n_free[1])
        fc.fc_kv_pages_plan(self.pages, self.kv_len[0], self.ones if n_keep is None else n_keep, self.n_free[0], path=path,
                            n_per_seq=self.n, out=out)
        self.state[0].copy_(self.state[1])
        born = None
        if self.keep:  # the rows' positions; out["pos"] are their places
            born = out["pos"] + self.ahead[out["seq"].clamp(min=0).long()]
        for l, (cache, k, v) in enumerate(zip(self.caches, self.k_new, self.v_new)):
            if self.bits == 4:
                fc.fc_kv4_write(cache, k.transpose(1, 2), v.transpose(1, 2), out["slot"], src=out["src"])
            else:
                fc.fc_kv8_write(cache, k.transpose(1, 2), v.transpose(1, 2), out["slot"], src=out["src"],
                                track=self.tracks[l][0] if self.keep else None, pos=born)

    def evict(self):
        """Cuts every sequence down to ``keep`` tokens, each layer and kv head
        choosing its own: those of the last ``recent`` positions, then those that
        received the largest attention weights.  Emptied pages are free again;
        positions go on.  For use between steps: a step captured in a CUDA graph
        stays good, as everything stays where it is."""
        if not self.keep:
            raise ValueError("a budget of tokens (keep) was not given")
        for l, cache in enumerate(self.caches):
            now, then = self.tracks[l]
            fc.fc_kv8_evict(cache, self.pages.table, self.kv_len[0], self.keeps, self.recent, now, then, out=self.from_,
                            workspace=self.evict_ws)
            now.weight.copy_(then.weight)
            now.born.copy_(then.born)
        had = self.kv_len[0].clone()
        self.release(self.keeps)
        self.ahead += had - self.kv_len[0]

    def release(self, keep):
        """Sequence b keeps its first keep[b] tokens (0: it is finished; one that
        takes its place starts at position 0); its other pages are free again.
        After evict() its tokens are in no order."""
        fc.fc_kv_pages_release(self.pages, self.kv_len[0], keep, self.n_free[0], out=(self.kv_len[1], self.n_free[1]))
        self.state[0].copy_(self.state[1])
        if self.keep:
            self.ahead.mul_(self.kv_len[0] > 0)

    def generate(self, tok, steps):
        """Greedy decoding of ``steps`` tokens from tok [B] (nodes = 1): [B, steps].
        Waits for them, and raises FastCoderError if an error was recorded: a
        sequence that found no free page (FC_ERR_CAPACITY) kept its length
        there, so that its later tokens are not to be used."""
        out, root = [], torch.full((self.B, 1), -1, dtype=torch.int32, device=tok.device)
        for _ in range(steps):
            tok = tok.view(self.B, 1)
            tok = fc.fc_argmax_accept(self.forward(tok), tok, root, self.ones, 2)["bonus"]
            self.append()
            out.append(tok)
        status = fc.LIB.fc_get_error(fc._stream())
        if status:
            raise fc.FastCoderError("Q4Decoder.generate", status)
        return torch.stack(out, 1)


def main(batch=1, context=4096, cache_bits=4, steps=20):
    from . import synth
    from .decoder import DEEPSEEK_CODER_1_3B as shape
    s = shape
    W = synth.decoder_weights(s.hidden, s.layers, s.H, s.Hkv, s.D, s.inter, s.vocab, 7, device="cuda")
    held, most = -(-context // 64), -(-(context + 2 * steps + 4) // 64)
    dec = Q4Decoder(s, W, batch, batch * most, most, cache_bits=cache_bits)
    # a context of random numbers, as if it had been decoded: the pages at the pool's end
    order = torch.arange(batch * most - 1, -1, -1, dtype=torch.int32, device="cuda")
    dec.pages.table[:, :held] = order[:batch * held].view(batch, held)
    dec.kv_len[dec.cur].fill_(context)
    dec.n_free[dec.cur].fill_(batch * (most - held))
    dec.pages.free.copy_(torch.arange(batch * most, dtype=torch.int32))
    for c in dec.caches:
        c.k_codes.random_(0x11, 0xFF if cache_bits == 4 else 0x7F)
        c.v_codes.random_(0x11, 0xFF if cache_bits == 4 else 0x7F)
        c.k_scale.fill_(0.1 if cache_bits == 4 else 2.0 ** -9)
        c.v_scale.fill_(0.1 if cache_bits == 4 else 2.0 ** -9)
    tok = torch.zeros((batch, 1), dtype=torch.int32, device="cuda")

    def step():
        dec.forward(tok)
        dec.append()

    for _ in range(3):
        step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    for _ in range(steps):
        g.replay()
    b.record()
    torch.cuda.synchronize()
    assert fc.fc_get_error() == "FC_OK"
    assert dec.kv_len[dec.cur].tolist() == [context + 3 + steps] * batch
    ms = a.elapsed_time(b) / steps
    print(f"batch {batch}, context {context}, cache in {cache_bits} bits: {ms:.3f} ms a step, {batch / ms * 1e3:.0f} tokens/s (forward and append, from a graph)")


if __name__ == "__main__":
    import sys
    main(*(int(v) for v in sys.argv[1:]))
