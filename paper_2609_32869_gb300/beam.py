"""Beam search of the target decoder over a paged 4-bit key/value cache.

`BeamDecoder` owns the device buffers of a batch of requests and runs the
decoder's passes: projections by `wf_gemm_bf16`, keys and values into the cache
by `wf_kv4_store`, both attentions by `wf_kv4_attention`, blocks and slots by
`wf_page_plan`, the selection by `wf_beam_select` and the beams' tables after it
by `wf_beam_reorder`.  Embeddings, LayerNorm and GELU are elementwise torch.
The host reads nothing back until the search is over.

    python -m paper_2609_32869_gb300.beam [--beams 5] [--requests 4] [--tokens 32]

decodes seeded synthetic requests with the tiny shapes.
"""
from __future__ import annotations

import numpy as np

from . import binding as B
from .session import _bf16_tensor, upload_weights


class Hypothesis:
    """A transcript (without prompt and end token) and the sum of its log-probabilities."""

    def __init__(self, tokens, score, ended):
        self.tokens, self.score, self.ended = tokens, score, ended

    def __repr__(self):
        return f"Hypothesis({self.tokens}, {self.score:.4f}, ended={self.ended})"


class BeamDecoder:
    """n_req requests of `beams` beams each, transcripts of up to max_ctx positions (prompt included)."""

    def __init__(self, cfg, weights, n_req: int, beams: int, max_ctx: int | None = None, block_size: int = 16, device="cuda"):
        import torch
        if n_req < 1 or not 1 <= beams <= B.WF_MAX_BEAMS or 2 * beams > cfg.vocab:
            raise ValueError(f"requests must be positive and beams from 1 to {B.WF_MAX_BEAMS}, at most half the vocabulary")
        if not B.wf_kv4_block_bytes(block_size, cfg.n_heads, cfg.head_dim):
            raise ValueError("the 4-bit cache takes blocks of 16, 32 or 64 positions and heads of 64 or 128")
        self.torch, self.cfg, self.n, self.W = torch, cfg, n_req, beams
        self.w = weights if isinstance(weights, dict) else upload_weights(weights, device)
        self.max_ctx, self.bs, self.device = max_ctx or cfg.max_pos, block_size, device
        self.rows = n_req * beams
        hd = cfg.head_dim
        self.cols = -(-self.max_ctx // block_size)
        # every beam may come to own its whole transcript
        self.n_blocks = self.rows * self.cols
        self.self_pool = self._pool(cfg.n_layers, self.n_blocks, block_size, hd)
        self.x_cols = -(-cfg.enc_frames // 64)
        self.cross_pool = self._pool(cfg.n_layers, n_req * self.x_cols, 64, hd)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.err = i32(1)
        self.free = i32(self.n_blocks)
        self.n_free = (i32(1), i32(1))
        self.tables = (i32(self.rows, self.cols), i32(self.rows, self.cols))
        self.lens = (i32(self.rows), i32(self.rows))
        self.want, self.offsets = i32(self.rows), i32(self.rows + 1)
        self.x_table, self.x_len = i32(n_req, self.x_cols), i32(n_req)
        self.scratch = torch.empty(max(
            256, B.wf_beam_select_scratch_bytes(n_req, beams, cfg.vocab), B.wf_beam_reorder_scratch_bytes(n_req, beams, self.cols)),
            dtype=torch.uint8, device=device)

    def _pool(self, layers, blocks, bs, hd):
        H = self.cfg.n_heads
        buf = self.torch.empty(layers * blocks * B.wf_kv4_block_bytes(bs, H, hd), dtype=self.torch.uint8, device=self.device)
        return B.kv4_pool(buf, layers, blocks, bs, H, hd)

    # ------------------------------------------------------------- pieces --
    def _linear(self, x, w, b):
        y = self.torch.empty(x.shape[0], w.shape[0], dtype=self.torch.float32, device=self.device)
        B.wf_gemm_bf16(x, w, b, y, x.shape[0], w.shape[0], x.shape[1], None, 0)
        return y

    def _norm(self, x, g, b):
        return self.torch.nn.functional.layer_norm(x, x.shape[-1:], g.float(), b.float(), self.cfg.ln_eps).bfloat16()

    def _attend(self, pool, layer, q, stride, table, cols, lens, n_seq, rps, causal, max_len):
        d, H = self.cfg.d_model, self.cfg.n_heads
        out = self.torch.empty(n_seq * rps, d, dtype=self.torch.bfloat16, device=self.device)
        size = B.wf_kv4_attention_scratch_bytes(n_seq, rps, H, H, self.cfg.head_dim, max_len)
        scratch = self.torch.empty(max(size, 16), dtype=self.torch.uint8, device=self.device)
        B.wf_kv4_attention(pool, layer, q, stride, table, cols, lens, n_seq, rps, H, causal, self.cfg.head_dim ** -0.5, max_len, out, d,
                           scratch, size, self.err)
        return out

    def _plan(self, old, new, n, bs, free, n_blocks, n_free, table, cols, cap, lens, left):
        slots = self.torch.empty(cap, dtype=self.torch.int32, device=self.device)
        B.wf_page_plan(old, new, n, bs, free, n_blocks, n_free, table, cols, self.offsets, slots, cap, lens, left, self.err)
        return slots

    # -------------------------------------------------------------- passes --
    def _encode(self, enc):
        """The acoustic keys and values of every layer, 4 bits, once per request."""
        torch, cfg, n = self.torch, self.cfg, self.n
        T, d, total = cfg.enc_frames, cfg.d_model, n * cfg.enc_frames
        ids = torch.arange(n * self.x_cols, dtype=torch.int32, device=self.device)
        count = torch.full((1,), n * self.x_cols, dtype=torch.int32, device=self.device)
        slots = self._plan(torch.zeros_like(self.x_len), torch.full_like(self.x_len, T), n, 64, ids, n * self.x_cols, count, self.x_table,
                           self.x_cols, total, self.x_len, torch.empty_like(count))
        for i, lw in enumerate(self.w["target_layers"]):
            kv = self._linear(enc.reshape(total, d), lw["xkv_w"], lw["xkv_b"]).bfloat16()
            B.wf_kv4_store(self.cross_pool, i, kv, 2 * d, kv[:, d:], 2 * d, slots, total, self.err)

    def _forward(self, tokens):
        """tokens int32 [rows, R], the next R positions of every beam; fp32 logits of the last."""
        torch, cfg, d = self.torch, self.cfg, self.cfg.d_model
        R, t = tokens.shape[1], self.w["target"]
        a, b = self.lens
        torch.add(a, R, out=self.want)
        slots = self._plan(a, self.want, self.rows, self.bs, self.free, self.n_blocks, self.n_free[0], self.tables[0], self.cols,
                           self.rows * R, b, self.n_free[1])
        self.lens, self.n_free = (b, a), self.n_free[::-1]
        pos = (a[:, None] + torch.arange(R, device=self.device)).clamp(max=cfg.max_pos - 1)
        x = (t["tok_emb"][tokens.clamp(min=0).long()].float() + t["pos_emb"][pos.long()].float()).reshape(-1, d)
        for i, lw in enumerate(self.w["target_layers"]):
            qkv = self._linear(self._norm(x, lw["ln1_g"], lw["ln1_b"]), lw["qkv_w"], lw["qkv_b"]).bfloat16()
            B.wf_kv4_store(self.self_pool, i, qkv[:, d:], 3 * d, qkv[:, 2 * d:], 3 * d, slots, self.rows * R, self.err)
            att = self._attend(self.self_pool, i, qkv, 3 * d, self.tables[0], self.cols, b, self.rows, R, True, self.max_ctx)
            x = x + self._linear(att, lw["out_w"], lw["out_b"])
            q = self._linear(self._norm(x, lw["ln2_g"], lw["ln2_b"]), lw["xq_w"], lw["xq_b"]).bfloat16()
            # a request's beams read the same frames: their rows go together
            att = self._attend(self.cross_pool, i, q, d, self.x_table, self.x_cols, self.x_len, self.n, self.W * R, False, cfg.enc_frames)
            x = x + self._linear(att, lw["xout_w"], lw["xout_b"])
            h = self._linear(self._norm(x, lw["ln3_g"], lw["ln3_b"]), lw["fc1_w"], lw["fc1_b"])
            x = x + self._linear(torch.nn.functional.gelu(h).bfloat16(), lw["fc2_w"], lw["fc2_b"])
        last = x.view(self.rows, R, d)[:, -1]
        return self._linear(self._norm(last, t["lnf_g"], t["lnf_b"]), t["tok_emb"], None)

    def _reorder(self, parent):
        B.wf_beam_reorder(self.self_pool, self.tables[0], self.tables[1], self.cols, self.lens[0], parent, self.n, self.W, self.free,
                          self.n_free[0], self.n_free[1], self.scratch, self.scratch.numel(), self.err)
        self.tables, self.n_free = self.tables[::-1], self.n_free[::-1]

    # -------------------------------------------------------------- search --
    def _inputs(self, enc, prompt, max_new, suppress):
        """The arguments of decode, checked on the host: the kernels read them by address and index with them."""
        torch, cfg, n = self.torch, self.cfg, self.n
        device = self.err.device
        prompt = np.asarray(prompt)
        if prompt.ndim != 2 or prompt.shape[0] != n or prompt.shape[1] < 1 or prompt.dtype.kind not in "iu":
            raise ValueError(f"prompt must hold {n} rows of at least one token id")
        if prompt.min() < 0 or prompt.max() >= cfg.vocab:
            raise ValueError("a prompt's token id is outside the vocabulary")
        if max_new < 0 or prompt.shape[1] + max_new > min(self.max_ctx, cfg.max_pos):
            raise ValueError("prompt and new tokens exceed the positions of the cache")
        shape = (n, cfg.enc_frames, cfg.d_model)
        if isinstance(enc, np.ndarray):
            if enc.shape != shape or enc.dtype.kind not in "iu" or enc.dtype.itemsize != 2:
                raise ValueError(f"enc must be the bits of bf16 values of shape {shape}")
            enc = _bf16_tensor(enc, self.device)
        elif tuple(enc.shape) != shape or enc.dtype != torch.bfloat16 or enc.device != device:
            raise ValueError(f"enc must be a bf16 tensor of shape {shape} on {device}")
        if suppress is not None:
            if tuple(suppress.shape) != (cfg.vocab,) or suppress.dtype not in (torch.uint8, torch.bool) or suppress.device != device:
                raise ValueError(f"suppress must be a uint8 or bool tensor of {cfg.vocab} entries on {device}")
            suppress = suppress.contiguous()
        return enc, prompt.astype(np.int32), suppress

    def decode(self, enc, prompt, max_new: int, suppress=None, length_penalty: float = 1.0):
        """enc [n, frames, d] (bf16 tensor, or its bits in numpy), prompt int [n, P], suppress (optional)
        uint8 or bool [vocab], nonzero for ids that are never proposed.  Up to max_new tokens a beam; per
        request its hypotheses, best score / length ** length_penalty first."""
        torch, cfg, n, W = self.torch, self.cfg, self.n, self.W
        enc, prompt, suppress = self._inputs(enc, prompt, max_new, suppress)
        if max_new == 0:
            return [[Hypothesis([], 0.0, False)] for _ in range(n)]
        self.err.zero_()
        self.free.copy_(torch.arange(self.n_blocks, device=self.device))
        self.n_free[0].fill_(self.n_blocks)
        self.tables[0].fill_(-1)
        self.lens[0].zero_()
        self._encode(enc)
        # every beam runs the prompt; the first selection has one live beam, and its children share the blocks
        tokens = torch.as_tensor(prompt, device=self.device).repeat_interleave(W, 0).contiguous()
        score = torch.full((n, W), -float("inf"), device=self.device)
        score[:, 0] = 0
        steps = []
        for _ in range(max_new):
            logits = self._forward(tokens)
            token, parent, fin_parent = (torch.empty(n, W, dtype=torch.int32, device=self.device) for _ in range(3))
            new_score, fin_score = torch.empty_like(score), torch.empty_like(score)
            B.wf_beam_select(logits, B.WF_F32, cfg.vocab, score, suppress, n, W, cfg.vocab, cfg.eos_id, token, parent, new_score,
                             fin_parent, fin_score, self.scratch, self.scratch.numel())
            self._reorder(parent)
            steps.append((token, parent, new_score, fin_parent, fin_score))
            tokens, score = token.view(-1, 1), new_score
        # release the requests' blocks
        self._reorder(torch.full((n, W), -1, dtype=torch.int32, device=self.device))
        if self.err.item():
            raise RuntimeError(f"device error word {self.err.item():#x}")
        return self._hypotheses([[v.cpu().numpy() for v in s] for s in steps], length_penalty)

    def _hypotheses(self, steps, length_penalty):
        def path(i, t, w):
            out = []
            while t >= 0:
                out.append(int(steps[t][0][i, w]))
                w, t = int(steps[t][1][i, w]), t - 1
            return out[::-1]

        found = []
        for i in range(self.n):
            hyps = []
            for t, (_, _, _, fin_parent, fin_score) in enumerate(steps):
                hyps += [Hypothesis(path(i, t - 1, int(b)), float(s), True) for b, s in zip(fin_parent[i], fin_score[i]) if b >= 0]
            last = len(steps) - 1
            hyps += [Hypothesis(path(i, last, w), float(steps[last][2][i, w]), False) for w in range(self.W) if np.isfinite(steps[last][2][i, w])]
            found.append(sorted(hyps, key=lambda h: -h.score / max(1, len(h.tokens) + h.ended) ** length_penalty))
        return found


def main(argv=None):
    import argparse

    from . import synthetic as syn
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--beams", type=int, default=5)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=32)
    a = ap.parse_args(argv)
    cfg = syn.TINY
    dec = BeamDecoder(cfg, syn.make_weights(cfg, seed=0, std=0.05), a.requests, a.beams)
    for i, hyps in enumerate(dec.decode(syn.encoder_output(cfg, a.requests), syn.prompts(cfg, a.requests), a.tokens)):
        print(f"request {i}: {hyps[0]}")


if __name__ == "__main__":
    main()
