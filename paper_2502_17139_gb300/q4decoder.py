"""Decoding in four bits: a LLaMA-family decoder whose weights are held in 4
bits (fc_w4_pack) and whose KV cache is paged and held in 4 bits (Kv4Cache),
for the few rows of a decoding step: single tokens of up to 16 sequences, or
one small draft tree (batch * nodes <= 16).

A step: forward() runs the rows against the caches, with the new tokens' own
keys and values in bf16; append() plans where the kept ones go
(fc_kv_pages_plan, once) and quantises them into every layer's pages
(fc_kv4_write).  All on the current stream, no host round trip.  Both read and
write the same tensors at every step, so that a step captured in a CUDA graph
is good for all of them.

    python -m paper_2502_17139_gb300.q4decoder [batch] [context]

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
    most ``max_pages``."""

    def __init__(self, shape: DecoderShape, W, batch, n_pages, max_pages, nodes=1, page_size=64, group=128,
                 device="cuda"):
        if batch * nodes > MAX_ROWS:
            raise ValueError(f"a step has at most {MAX_ROWS} rows")
        s = shape
        self.s, self.B, self.n = s, batch, nodes
        pack = lambda w: fc.fc_w4_pack(w.contiguous(), group)
        self.embed, self.final_norm, self.lm_head = W["embed"], W["final_norm"], pack(W["lm_head"])
        self.layers = [dict(attn_norm=w["attn_norm"], mlp_norm=w["mlp_norm"], wq=pack(w["wq"]), wkv=pack(w["wkv"]),
                            wo=pack(w["wo"]), wgu=pack(w["wgu"]), wd=pack(w["wd"])) for w in W["layers"]]
        i32 = dict(dtype=torch.int32, device=device)
        self.pages = fc.KvPages(page_size, torch.zeros((batch, max_pages), **i32),
                                torch.arange(n_pages - 1, -1, -1, **i32))
        self.caches = [fc.Kv4Cache.empty(n_pages, s.Hkv, page_size, s.D, device) for _ in range(s.layers)]
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
        self.ws = fc.kv4_attn_workspace(batch, nodes, s.H, s.Hkv, device)
        self.steps = torch.arange(nodes, **i32)[None, :]
        self.ones = torch.full((batch,), nodes, **i32)

    def forward(self, tok, pos=None, mask=None, n_nodes=None):
        """tok [B, n] int32 -> logits [B, n, vocab].  pos [B, n] (None: the
        tokens follow the cache in order), mask [B, n, 1] int64 ancestor bits
        (None: each sees those before it), n_nodes [B]."""
        s, B, n, kv_len = self.s, self.B, self.n, self.kv_len[0]
        if pos is None:
            pos = kv_len[:, None] + self.steps
        fc.fc_embed(tok.reshape(-1), self.embed, self.x)
        r = None
        for l, w in enumerate(self.layers):
            fc.fc_add_rmsnorm(self.x, r, w["attn_norm"], self.h, s.eps)
            fc.fc_w4_matvec(self.h, w["wq"], out=self.q.view(B * n, -1))
            fc.fc_rope(self.q, pos, s.rope_base, out=self.q)
            fc.fc_w4_matvec(self.h, w["wkv"], out=self.kv)
            stride = 2 * s.Hkv * s.D
            fc.fc_rope_heads(self.kv, 0, stride, self.k_new[l], B, n, s.Hkv, s.D, pos, s.rope_base)
            fc.fc_rope_heads(self.kv, s.Hkv * s.D, stride, self.v_new[l], B, n, s.Hkv, s.D, pos, 0.0)
            fc.fc_kv4_attn(self.q, self.caches[l], self.pages.table, kv_len, self.k_new[l], self.v_new[l], mask, n_nodes,
                           out=self.attn, workspace=self.ws)
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
        for cache, k, v in zip(self.caches, self.k_new, self.v_new):
            fc.fc_kv4_write(cache, k.transpose(1, 2), v.transpose(1, 2), out["slot"], src=out["src"])

    def release(self, keep):
        """Sequence b keeps its first keep[b] tokens (0: it is finished); its
        other pages are free again."""
        fc.fc_kv_pages_release(self.pages, self.kv_len[0], keep, self.n_free[0], out=(self.kv_len[1], self.n_free[1]))
        self.state[0].copy_(self.state[1])

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


def main(batch=1, context=4096, steps=20):
    from . import synth
    from .decoder import DEEPSEEK_CODER_1_3B as shape
    s = shape
    W = synth.decoder_weights(s.hidden, s.layers, s.H, s.Hkv, s.D, s.inter, s.vocab, 7, device="cuda")
    held, most = -(-context // 64), -(-(context + 2 * steps + 4) // 64)
    dec = Q4Decoder(s, W, batch, batch * most, most)
    # a context of random numbers, as if it had been decoded: the pages at the pool's end
    order = torch.arange(batch * most - 1, -1, -1, dtype=torch.int32, device="cuda")
    dec.pages.table[:, :held] = order[:batch * held].view(batch, held)
    dec.kv_len[dec.cur].fill_(context)
    dec.n_free[dec.cur].fill_(batch * (most - held))
    dec.pages.free.copy_(torch.arange(batch * most, dtype=torch.int32))
    for c in dec.caches:
        c.k_codes.random_(0x11, 0xFF)
        c.v_codes.random_(0x11, 0xFF)
        c.k_scale.fill_(0.1)
        c.v_scale.fill_(0.1)
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
    print(f"batch {batch}, context {context}: {ms:.3f} ms a step, {batch / ms * 1e3:.0f} tokens/s (forward and append, from a graph)")


if __name__ == "__main__":
    import sys
    main(*(int(v) for v in sys.argv[1:]))
