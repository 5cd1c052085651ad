"""A draft model held in 8 bits, proposing to the bf16 target: the operators of include/spec_q8.h as a decoder runs them.

    python -m paper_2411_00853_amd.draft8 [--model draft|target] [--batch B] [--context N] [--lookahead K] ...

Draft8 is the decoder (weights, caches, one `feed` for windows of any length); `Draft8.propose` is the draft loop of a round, whose
filtered rows are the draft logits of spec_verify_step.  The command runs rounds on the 7B-shape target with random weights and prints
the time of the parts.  With --model target the target drafts for itself in 8 bits: how many proposals are then accepted says how
near the 8-bit decoder's distribution is to the bf16 one's (less what the filters cut off).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as sv
from .prompt import Prompt, pack_weights

_F8 = torch.float8_e4m3fn


def quantise_weight(w: torch.Tensor):
    """[n_out][n_in] -> (e4m3 in the product's order, fp32 scale of each 128 x 128 block)."""
    n, k = w.shape
    p = torch.nn.functional.pad(w.float(), (0, -k % 128, 0, -n % 128))
    b = p.view(p.shape[0] // 128, 128, p.shape[1] // 128, 128)
    s = (b.abs().amax((1, 3)) / 448).clamp_min(2.0 ** -126)
    q = (b / s[:, None, :, None]).to(_F8).view(p.shape)[:n, :k].contiguous()
    return sv.spec_q8_pack_weight(q), s.contiguous()


def rope_table(max_pos: int, head_dim: int, theta: float, device="cuda") -> torch.Tensor:
    """fp32 [max_pos][head_dim/2][2]: cosine and sine of pos * theta^(-2i/head_dim)."""
    f = theta ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device=device) / head_dim)
    a = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


class Draft8:
    """A decoder of workload.ModelShape `shape` in 8 bits.  weights: as workload.make_weights gives them, on the device (kept in bf16:
    the embedding only).  Device memory is allocated in __init__ alone, so `feed` and `propose` can be captured into a HIP graph by any
    means.  max_window: the longest window of a `feed`; `propose` needs 2."""

    def __init__(self, shape, weights: dict, batch: int, max_kv_len: int, max_window: int, temperature: float = 1.0,
                 top_k: Optional[int] = None, top_p: Optional[float] = None, min_p: Optional[float] = None):
        self.shape, self.batch, self.max_kv_len, self.max_window = shape, batch, max_kv_len, max_window
        d, F, V, hd = shape.d_model, shape.d_ffn, shape.vocab, shape.head_dim
        self.embed, self.final_norm = weights["tok_embed"], weights["final_norm"]
        self.head = quantise_weight(weights["lm_head"])
        self.layers = [(lw["attn_norm"], quantise_weight(lw["w_qkv"]), quantise_weight(lw["w_o"]), lw["ffn_norm"],
                        quantise_weight(lw["w_gate_up"]), quantise_weight(lw["w_down"])) for lw in weights["layers"]]
        dev = self.embed.device
        pages = (max_kv_len + sv.KV8_PAGE - 1) // sv.KV8_PAGE
        table = torch.arange(batch * pages, dtype=torch.int32, device=dev).view(batch, pages)
        self.caches = [sv.Kv8Cache(torch.zeros((batch * pages, shape.n_kv_heads, 2, sv.KV8_PAGE * hd), dtype=_F8, device=dev),
                                   torch.ones((batch * pages, shape.n_kv_heads, 2), device=dev), table, hd)
                       for _ in range(shape.n_layers)]
        self.cos_sin = rope_table(max_kv_len, hd, shape.rope_theta, dev)
        R = batch * max_window
        new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device=dev)
        self.embedded, self.first, self.at = new(R, d, dtype=self.embed.dtype), new(batch, 2, dtype=torch.int32), new(batch, dtype=torch.int32)
        self.x, self.delta, self.qkv = new(R, d, dtype=torch.float32), new(R, d), new(R, shape.d_q + 2 * shape.d_kv)
        self.q, self.attn, self.gate_up = new(R, shape.d_q), new(R, shape.d_q), new(R, 2 * F)
        self.logits = new(R, V, dtype=torch.float32)
        # the operand of each width: the model's, the attention's, the FFN's
        self.rows8 = {n: (torch.empty(R * self._up(n), dtype=_F8, device=dev), torch.empty(R * self._up(n) // 128, device=dev))
                      for n in {d, shape.d_q, F}}
        self.work = torch.empty(max(16, sv.spec_kv8_workspace_bytes(R, shape.n_q_heads, hd)), dtype=torch.uint8, device=dev)
        self.draw_work = torch.empty(max(16, sv.spec_filter_workspace_bytes(batch, V)), dtype=torch.uint8, device=dev)
        self.drawn, self.filtered = torch.empty(batch, dtype=torch.int32, device=dev), torch.empty((batch, V), device=dev)
        per_row = lambda v, dtype: None if v is None else torch.full((batch,), v, dtype=dtype, device=dev)
        self.temperature = per_row(temperature, torch.float32)
        self.filters = dict(top_k=per_row(top_k, torch.int32), top_p=per_row(top_p, torch.float32), min_p=per_row(min_p, torch.float32))
        self.row0 = {w: torch.arange(batch + 1, dtype=torch.int32, device=dev) * w for w in range(1, max_window + 1)}

    @staticmethod
    def _up(n: int) -> int:
        return (n + 127) // 128 * 128

    def _operand(self, rows: int, cols: int):
        q, s = self.rows8[cols]
        kp = self._up(cols)
        return q[:rows * kp].view(rows, kp), s[:rows * kp // 128].view(kp // 128, rows)

    def feed(self, tokens: torch.Tensor, kv_len: torch.Tensor, max_len: int = 0, logits: bool = True):
        """tokens int32 [batch][w] (copied if not contiguous), the next w tokens of every sequence, at positions kv_len[b] + 0 .. w-1 -> fp32 logits
        [batch * w][vocab] of this object (None with logits=False).  kv_len is not changed."""
        s, w = self.shape, tokens.shape[1]
        if not 1 <= w <= self.max_window:
            raise ValueError(f"a window of {w} tokens, at most {self.max_window}")
        R = self.batch * w
        d, F, row0 = s.d_model, s.d_ffn, self.row0[w]
        x, delta = self.x[:R], None
        x.copy_(torch.index_select(self.embed, 0, tokens.reshape(-1), out=self.embedded[:R]))
        for cache, (attn_norm, w_qkv, w_o, ffn_norm, w_gate_up, w_down) in zip(self.caches, self.layers):
            a = sv.spec_q8_add_rmsnorm(x, delta, attn_norm, s.rms_eps, x, *self._operand(R, d))
            qkv = sv.spec_q8_gemm(*a, *w_qkv, self.qkv[:R])
            sv.spec_kv8_append(cache, qkv, row0, kv_len, s.n_q_heads, w, self.cos_sin, self.q[:R])
            o = sv.spec_kv8_attention(cache, self.q[:R], row0, kv_len, s.n_q_heads, w, max_len, s.head_dim ** -0.5, self.attn[:R],
                                      self.work)
            delta = sv.spec_q8_gemm(*sv.spec_q8_quantize(o, *self._operand(R, s.d_q)), *w_o, self.delta[:R])
            a = sv.spec_q8_add_rmsnorm(x, delta, ffn_norm, s.rms_eps, x, *self._operand(R, d))
            gate_up = sv.spec_q8_gemm(*a, *w_gate_up, self.gate_up[:R])
            delta = sv.spec_q8_gemm(*sv.spec_q8_swiglu(gate_up, *self._operand(R, F)), *w_down, self.delta[:R])
        if not logits:
            return None
        a = sv.spec_q8_add_rmsnorm(x, delta, self.final_norm, s.rms_eps, None, *self._operand(R, d))
        return sv.spec_q8_gemm(*a, *self.head, self.logits[:R])

    def propose(self, prev: torch.Tensor, last: torch.Tensor, kv_len: torch.Tensor, uniforms: torch.Tensor, tokens: torch.Tensor,
                logits: torch.Tensor, max_len: int = 0):
        """K = tokens.shape[1] proposals after `last`, the token at position kv_len[b] of each sequence: tokens int32 [batch][K] and the
        filtered rows they were drawn from, logits fp32 [batch][K][vocab].  prev: the token before last, whose keys the cache may
        not hold yet (the target's round may have ended on a proposal that was never fed).  uniforms: [K][batch]."""
        if self.max_window < 2:
            raise ValueError("proposals begin with a window of 2 tokens, max_window is 1")
        step = torch.stack((prev, last), 1, out=self.first)
        for i in range(tokens.shape[1]):
            rows = self.feed(step, torch.add(kv_len, i if i else -1, out=self.at), max_len)
            if i == 0:
                rows = rows.view(self.batch, 2, -1)[:, 1]
            sv.spec_filter_sample(rows, uniforms[i], self.temperature, self.drawn, logits_out=self.filtered, workspace=self.draw_work,
                                  **self.filters)
            logits[:, i].copy_(self.filtered)
            tokens[:, i].copy_(self.drawn)
            step = self.drawn[:, None]


class Rounds:
    """A bf16 target and the Draft8 that proposes to it: `feed` a context, then `round` after round.  Sequence b is slot b of both."""

    def __init__(self, target_shape, weights: dict, draft: Draft8, lookahead: int, prompt_rows: int = 0):
        """weights: as workload.make_weights gives them, on the device.  `feed` takes contexts of up to prompt_rows tokens in all through the
        target as whole prompts (prompt.py, whose cache differs from the windows' by its roundings), longer ones window by window."""
        B, V, K, dev = draft.batch, target_shape.vocab, lookahead, draft.embed.device
        self.draft, self.K, self.B = draft, K, B
        cfg = sv.make_cfg(target_shape, B, draft.max_kv_len, K)
        packed = pack_weights(weights)
        cache = torch.zeros(sv.spec_kv_cache_bytes(cfg), dtype=torch.uint8, device=dev)
        self.kv_len = torch.zeros(B, dtype=torch.int32, device=dev)   # of the target; the position of `last` on both sides
        self.handle = sv.spec_verify_init(cfg, packed, cache, self.kv_len)
        ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
        self.prev, self.last, self.slots = ints(B), ints(B), torch.arange(B, dtype=torch.int32, device=dev)
        self.tokens, self.n_accepted, self.out = ints(B, K), ints(B), ints(B, K + 1)
        self.logits = torch.zeros((B, K, V), device=dev)
        self.prompt = Prompt(self.handle, packed, prompt_rows) if prompt_rows else None

    def feed(self, context: torch.Tensor):
        """context int32 [batch][n], n >= 2: into both caches, in windows; its last token is the first one to be decoded."""
        d, n = self.draft, context.shape[1]
        at = torch.zeros_like(self.kv_len)
        for t in range(0, n - 1, d.max_window):
            window = context[:, t:min(t + d.max_window, n - 1)].contiguous()
            d.feed(window, at + t, logits=False)
        self.prev.copy_(context[:, n - 2])
        self.last.copy_(context[:, n - 1])
        if self.prompt is not None and self.B * (n - 1) <= self.prompt.max_rows:
            row0 = torch.arange(self.B + 1, dtype=torch.int32, device=context.device) * (n - 1)
            self.prompt.run(context[:, :n - 1].reshape(-1), row0, self.slots, n - 1, logits=False)
            self.kv_len.fill_(n - 1)
            return
        # the target scores a window as it does proposals, and keeps all of it
        half = torch.full((self.B, self.K + 1), 0.5, device=context.device)
        for t in range(0, n - 1, self.K + 1):
            window = context[:, t:min(t + self.K + 1, n - 1)].contiguous()
            self.tokens[:, :window.shape[1] - 1].copy_(window[:, 1:])
            sv.spec_verify_step(self.handle, [window.shape[1] - 1] * self.B, half, 1.0, self.n_accepted, self.out, seq_slot=self.slots,
                                last_token=window[:, 0].contiguous(), draft_tokens=self.tokens, draft_logits=self.logits,
                                auto_rollback=False)

    def propose(self, uniforms: torch.Tensor, max_len: int = 0):
        self.draft.propose(self.prev, self.last, self.kv_len, uniforms, self.tokens, self.logits, max_len)

    def verify(self, uniforms: torch.Tensor, temperature: float):
        """Scores the proposals; out [batch][K+1] then begins with n_accepted[b] + 1 new tokens of sequence b."""
        sv.spec_verify_step(self.handle, [self.K] * self.B, uniforms, temperature, self.n_accepted, self.out, seq_slot=self.slots,
                            last_token=self.last, draft_tokens=self.tokens, draft_logits=self.logits)
        a = self.n_accepted.long()[:, None]
        self.prev.copy_(torch.where(a > 0, self.out.gather(1, (a - 1).clamp_min(0)), self.last[:, None])[:, 0])
        self.last.copy_(self.out.gather(1, a)[:, 0])


def main():
    import argparse
    import time

    from . import workload as wl

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", choices=("draft", "target"), default="draft", help="what drafts: the configuration's draft shape or the target's own")
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--context", type=int, default=256)
    ap.add_argument("--lookahead", type=int, default=5)
    ap.add_argument("--rounds", type=int, default=20)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--top-k", type=int)
    ap.add_argument("--top-p", type=float)
    ap.add_argument("--min-p", type=float)
    ap.add_argument("--prompt", action="store_true", help="the context goes through the target as whole prompts, not window by window")
    a = ap.parse_args()
    B, K, T = a.batch, a.lookahead, a.temperature
    W = 3   # rounds before the clock starts
    max_kv = a.context + (a.rounds + W + 1) * (K + 1)
    weights = wl.make_weights(wl.SEVEN_B, wl.SEED_BASE + 2, "cuda")
    shape = wl.SEVEN_B if a.model == "target" else wl.SEVEN_B_DRAFT
    own = weights if a.model == "target" else wl.make_weights(shape, wl.SEED_BASE + 3, "cuda")
    draft = Draft8(shape, own, B, max_kv, 64, T, a.top_k, a.top_p, a.min_p)
    rounds = Rounds(wl.SEVEN_B, weights, draft, K, B * a.context if a.prompt else 0)
    del weights, own
    rng = wl.Rng(wl.SEED_BASE + 4, "cuda")
    rounds.feed(rng.randint(wl.S_TOKENS, (B, a.context), shape.vocab))
    draft_u = rng.uniform(wl.S_UNIFORMS, (a.rounds + W, K, B))
    verify_u = rng.uniform(wl.S_UNIFORMS + 1, (a.rounds + W, B, K + 1))
    # the draft loop is some hundred launches: recorded once, replayed every round
    u = draft_u[0].clone()
    rounds.propose(u, max_kv)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rounds.propose(u, max_kv)
    parts, kept = [0.0, 0.0], 0
    for r in range(W + a.rounds):
        u.copy_(draft_u[r])
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        graph.replay()
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        rounds.verify(verify_u[r], T)
        torch.cuda.synchronize()
        t2 = time.perf_counter()
        if r >= W:
            parts[0] += t1 - t0
            parts[1] += t2 - t1
            kept += int(rounds.n_accepted.sum())
    sv.spec_verify_poll(rounds.handle)
    n = a.rounds
    print(f"{B} sequences, {K} proposals a round, {n} rounds: draft loop {parts[0] / n * 1e3:.3f} ms "
          f"({parts[0] / n / K * 1e6:.0f} us a token), verification {parts[1] / n * 1e3:.3f} ms, "
          f"{kept / (n * B * K):.3f} of the proposals accepted, {(kept + n * B) / sum(parts):.0f} tokens/s", flush=True)


if __name__ == "__main__":
    main()
