"""Whole prompts through a bf16 target: the operators of include/spec_prompt.h as a decoder runs them.

    python -m paper_2411_00853_amd.prompt [--model draft|target] [--prompts B] [--tokens N] ...

Prompt.run takes packed prompts through all layers, leaves their keys and values in the cache of a handle of spec_verify_init and gives
the logits behind each prompt; the handle's steps, and decoding rounds on it, go on from there.  The command runs prompts of random
tokens through the 7B-shape target (or its draft) with random weights and prints the time.

The pass keeps less than spec_verify_step does.  That multiplies activations, queries and attention weights as bf16 numbers and what their rounding
leaves, and rotates fp32 projections; here normalised rows, queries, keys, values, attention weights, the attention's result and the activation are one bf16
number each, and the cache's keys have been rounded in front of the rotation as well as behind it.  Products, softmax, sums and the residual
stream are fp32 in both.  So the cache is not the one that steps over the same tokens would have left: with random weights of the 4-layer draft
of the 7B shape keys and values differ by 0.3 % of their root mean square in the first layer and by 1 % in the last.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as sv


def pack_weights(weights: dict) -> dict:
    """workload.make_weights' tensors, on the device -> the same with every projection in the order that the products read."""
    pack = sv.spec_pack_weight
    return {"tok_embed": weights["tok_embed"], "final_norm": weights["final_norm"], "lm_head": pack(weights["lm_head"]),
            "layers": [{"attn_norm": lw["attn_norm"], "ffn_norm": lw["ffn_norm"], "w_qkv": pack(lw["w_qkv"]), "w_o": pack(lw["w_o"]),
                        "w_gate_up": pack(lw["w_gate_up"], True), "w_down": pack(lw["w_down"])} for lw in weights["layers"]]}


class Prompt:
    """The pass of prompts of up to max_rows tokens in all, max_batch of them at most.  weights: those the handle was made with
    (pack_weights).  Device memory is allocated in __init__ alone, so `run` can be captured into a HIP graph; it is that of one run at a time.  The
    workspace (up to 130 MiB) is what any run that fits may ask for, so a short prompt takes the same time in large buffers as in its own."""

    def __init__(self, handle: sv.Handle, weights: dict, max_rows: int, max_batch: Optional[int] = None):
        c = handle.cfg
        self.handle, self.weights, self.max_rows, self.max_batch = handle, weights, max_rows, max_batch or c.max_batch
        d, hd, dev = c.d_model, c.head_dim, weights["tok_embed"].device
        self.d_q, self.d_kv = c.n_q_heads * hd, c.n_kv_heads * hd
        new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device=dev)
        R, B = max_rows, self.max_batch
        self.embedded, self.x, self.h = new(R, d), new(R, d, dtype=torch.float32), new(R, d)
        self.qkv, self.attn, self.act = new(R, self.d_q + 2 * self.d_kv), new(R, self.d_q), new(R, c.d_ffn)
        self.ends, self.last_x, self.last_h = new(B, dtype=torch.int32), new(B, d, dtype=torch.float32), new(B, d)
        self.logits = new(B, c.vocab, dtype=torch.float32)
        self.tokens, self.outside = new(R, dtype=torch.int32), new(R, dtype=torch.bool)
        shapes = ((R, self.d_q + 2 * self.d_kv, d, "none"), (R, d, self.d_q, "none"), (R, c.d_ffn, d, "swiglu"), (R, d, c.d_ffn, "none"),
                  (B, c.vocab, d, "none"))
        # of any run that fits: short prompts share out what long ones do not
        need = max([sv.spec_prompt_gemm_workspace_bytes_up_to(*s) for s in shapes] +
                   [sv.spec_prompt_attention_workspace_bytes_up_to(R, B, c.n_q_heads, c.n_kv_heads, hd)])
        self.work = torch.empty(max(16, need), dtype=torch.uint8, device=dev)

    def run(self, tokens: torch.Tensor, row0: torch.Tensor, seq_slot: torch.Tensor, max_len: int = 0, logits: bool = True):
        """tokens int32 [rows]: prompt b is tokens[row0[b]:row0[b+1]], from position 0 of slot seq_slot[b] on (device int32 [batch + 1] and
        [batch]; no slot twice).  Returns fp32 logits [batch][vocab] of this object, behind each prompt's last token (an empty prompt's row means nothing);
        None with logits=False.  The handle's kv_len is not changed.  max_len: the longest prompt, if known.  A token outside the vocabulary
        makes everything behind it in its prompt NaN, the logits too."""
        c, rows, batch = self.handle.cfg, tokens.numel(), seq_slot.numel()
        if not 1 <= rows <= self.max_rows or not 1 <= batch <= self.max_batch:
            raise ValueError(f"{rows} rows of {batch} prompts, at most {self.max_rows} and {self.max_batch}")
        x, h, qkv, attn, act = (t[:rows] for t in (self.x, self.h, self.qkv, self.attn, self.act))
        q, k, v = qkv[:, :self.d_q], qkv[:, self.d_q:self.d_q + self.d_kv], qkv[:, self.d_q + self.d_kv:]
        rotated, scale = qkv[:, :self.d_q + self.d_kv], c.head_dim ** -0.5
        if tokens.dtype != torch.int32 or tokens.dim() != 1:
            raise ValueError(f"tokens: expected int32 [rows], got {tokens.dtype} {tuple(tokens.shape)}")
        inside = torch.clamp(tokens, 0, c.vocab - 1, out=self.tokens[:rows])
        embedded = torch.index_select(self.weights["tok_embed"], 0, inside, out=self.embedded[:rows])
        x.copy_(embedded.masked_fill_(torch.ne(tokens, inside, out=self.outside[:rows])[:, None], float("nan")))
        for layer, w in enumerate(self.weights["layers"]):
            sv.spec_prompt_rmsnorm(x, w["attn_norm"], c.rms_eps, h)
            sv.spec_prompt_gemm(h, w["w_qkv"], qkv, workspace=self.work)
            sv.spec_prompt_append(self.handle, layer, qkv, rotated, row0, seq_slot)
            sv.spec_prompt_attention(q, k, v, c.n_q_heads, c.n_kv_heads, row0, attn, scale, max_q_len=max_len, max_k_len=max_len,
                                     workspace=self.work)
            sv.spec_prompt_gemm(attn, w["w_o"], x, residual=x, workspace=self.work)
            sv.spec_prompt_rmsnorm(x, w["ffn_norm"], c.rms_eps, h)
            sv.spec_prompt_gemm(h, w["w_gate_up"], act, activation="swiglu", workspace=self.work)
            sv.spec_prompt_gemm(act, w["w_down"], x, residual=x, workspace=self.work)
        if not logits:
            return None
        ends = torch.sub(row0[1:], 1, out=self.ends[:batch]).clamp_(0, rows - 1)
        last = torch.index_select(x, 0, ends, out=self.last_x[:batch])
        sv.spec_prompt_rmsnorm(last, self.weights["final_norm"], c.rms_eps, self.last_h[:batch])
        return sv.spec_prompt_gemm(self.last_h[:batch], self.weights["lm_head"], self.logits[:batch], workspace=self.work)


def main():
    import argparse
    import time

    from . import workload as wl

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", choices=("draft", "target"), default="target")
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=1024, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    shape = wl.SEVEN_B if a.model == "target" else wl.SEVEN_B_DRAFT
    weights = pack_weights(wl.make_weights(shape, wl.SEED_BASE + 2, "cuda"))
    cfg = sv.make_cfg(shape, a.prompts, a.tokens, 0)
    cache = torch.zeros(sv.spec_kv_cache_bytes(cfg), dtype=torch.uint8, device="cuda")
    kv_len = torch.zeros(a.prompts, dtype=torch.int32, device="cuda")
    handle = sv.spec_verify_init(cfg, weights, cache, kv_len)
    lens = [max(1, a.tokens * (2 * a.prompts - i) // (2 * a.prompts)) for i in range(a.prompts)]
    starts = [sum(lens[:i]) for i in range(a.prompts + 1)]
    tokens = wl.Rng(wl.SEED_BASE + 5, "cuda").randint(wl.S_TOKENS, (starts[-1],), shape.vocab)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    row0, slots = ints(starts), ints(list(range(a.prompts)))
    prompt = Prompt(handle, weights, starts[-1])
    for _ in range(2):
        prompt.run(tokens, row0, slots, max(lens))
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        prompt.run(tokens, row0, slots, max(lens))
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    sv.spec_verify_poll(handle)
    c = shape
    flops = 2 * starts[-1] * c.n_layers * (c.d_model * (2 * c.d_q + 2 * c.d_kv) + 3 * c.d_model * c.d_ffn) + \
        sum(2 * n * (n + 1) * c.d_q * c.n_layers for n in lens) + 2 * a.prompts * c.vocab * c.d_model
    print(f"{a.prompts} prompts, {starts[-1]} tokens: {t * 1e3:.2f} ms, {starts[-1] / t:.0f} tokens/s, {flops / t / 1e12:.0f} TFLOP/s", flush=True)


if __name__ == "__main__":
    main()
