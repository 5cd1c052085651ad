"""The operators that run whole prompts through a bf16 decoder and leave their keys and values in its cache.

A case is a dict of sizes.  Its "op" says which operator it takes:

  norm    spec_prompt_rmsnorm: the residual stream's rows, normalised, as the operand of a product
  gemm    spec_prompt_gemm: rows times a packed weight matrix; bias, activation and residual on the way out
  append  spec_prompt_append: rotary embedding of queries and keys, keys and values into a model's cache
  attn    spec_prompt_attention: causal attention over packed sequences, query heads that share kv heads

Rows of several sequences lie one after the other: sequence b has rows row0[b] .. row0[b+1]-1.

  weights  packed: [Kp/128][Np/16][4] tiles of [64][8], element (lane, e) of tile (kb / 4, j, kb % 4) is row 16j + lane % 16, column
           32kb + 8 (lane / 16) + e; of a gate and up matrix even j are gate rows and odd j the same up rows
  cache    of one layer [slot][position / 32][kv head][2][32 head_dim]: key (t, d) at [t/16][d/8][t%16][d%8], value (t, d) at
           [d/16][t%16/4][d%16][t/16][t%4]
"""
import math

import torch

own = False

BF16 = torch.bfloat16
EPS, THETA = 1e-5, 10000.0


# ---- cases -------------------------------------------------------------------------------------------

def _gemm(rows, n, k, y, act="none", bias=False, residual="none", **more):
    """n: columns of y (a gate and up matrix has twice as many rows)"""
    return dict({"op": "gemm", "rows": rows, "n": n, "k": k, "y": y, "act": act, "bias": bias, "residual": residual}, **more)


def _append(batch, lens, at, q_heads, kv_heads, head_dim, **more):
    return dict({"op": "append", "batch": batch, "q_min": lens[0], "q_max": lens[1], "at": at, "q_heads": q_heads, "kv_heads": kv_heads,
                 "head_dim": head_dim}, **more)


def _attn(batch, lens, before, q_heads, kv_heads, head_dim, **more):
    return dict({"op": "attn", "batch": batch, "q_min": lens[0], "q_max": lens[1], "before": before, "q_heads": q_heads,
                 "kv_heads": kv_heads, "head_dim": head_dim}, **more)


def listed():
    return [
        # one sequence's last row in front of the LM head, 1B shape: nothing but latency
        {"name": "norm_one_row", "op": "norm", "rows": 1, "cols": 2048, "x": "fp32"},
        # a prompt of the 7B shape
        {"name": "norm_prompt", "op": "norm", "rows": 4096, "cols": 4096, "x": "fp32"},
        # the last rows of eight prompts through the LM head of the 7B shape: the weights' stream
        _gemm(8, 32000, 4096, "fp32", name="gemm_last_rows"),
        # a short question, output projection of the 7B shape onto the residual stream
        _gemm(37, 4096, 4096, "fp32", residual="fp32", name="gemm_short_prompt"),
        # prompts packed to 2048 rows, gate and up projection of the 7B shape: the matrix cores
        _gemm(2048, 11008, 4096, "bf16", act="swiglu", name="gemm_gate_up"),
        # a ragged prompt through a feed-forward layer with biases, widths that are multiples of nothing much
        _gemm(1333, 4104, 2080, "bf16", act="gelu", bias=True, residual="bf16", name="gemm_ragged"),
        # one short question, 1B shape
        _append(1, (37, 37), 0, 32, 8, 64, name="append_short"),
        # ragged prompts, 7B shape, some 4700 rows
        _append(6, (60, 1500), 0, 32, 32, 128, name="append_packed"),
        # one short question, 1B shape: latency
        _attn(1, (64, 64), 0, 32, 8, 64, name="attn_short"),
        # a batch of prompts of all lengths, 1B shape
        _attn(16, (50, 2100), 0, 32, 8, 64, name="attn_packed"),
        # one long document, 7B shape: the matrix cores
        _attn(1, (8192, 8192), 0, 32, 32, 128, name="attn_long"),
        # single tokens behind long sequences, shared heads: the stream of keys and values
        _attn(8, (1, 1), 6000, 32, 8, 128, name="attn_tokens"),
    ]


def _log_int(rng, lo, hi, to=1):
    """A size between lo and hi, spread over its logarithm, rounded up to a multiple of `to`."""
    return -(-min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))) // to) * to


def _heads(rng):
    head_dim, kv_heads = rng.choice((64, 128)), rng.choice((1, 2, 4, 8, 8, 12, 32))
    return kv_heads * (rng.choice((1, 2, 3, 4, 8)) if kv_heads < 12 else 1), kv_heads, head_dim


def draw(rng):
    op = rng.choice(("norm", "gemm", "gemm", "gemm", "append", "attn", "attn", "attn"))
    if op == "norm":
        return {"op": op, "rows": _log_int(rng, 1, 4096), "cols": _log_int(rng, 64, 8192, rng.choice((1, 64, 64))),
                "x": rng.choice(("fp32", "fp32", "bf16"))}
    if op == "gemm":
        act = rng.choice(("none", "none", "relu", "gelu", "silu", "swiglu"))
        to = 16 if act == "swiglu" else rng.choice((1, 64, 64))
        n, k = _log_int(rng, 256, 16000, to), _log_int(rng, 256, 12288, 32)
        most = int(2.0e11 / (2 * n * k))        # rows
        residual = "none" if act == "swiglu" else rng.choice(("none", "fp32", "bf16"))
        return _gemm(_log_int(rng, 1, max(1, min(most, 4096))), n, k, rng.choice(("bf16", "fp32")), act, rng.random() < 0.3, residual)
    heads = _heads(rng)
    if op == "append":
        n = _log_int(rng, 1, 4096)
        batch = _log_int(rng, 1, max(1, min(64, 6000 // n)))
        return _append(batch, (int(n * rng.choice((0.0, 0.2, 1.0))), n), _log_int(rng, 1, 2000) - 1, *heads)
    n = _log_int(rng, 1, 6000)
    before = 0 if rng.random() < 0.5 else _log_int(rng, 1, 16000)
    per = lambda: n * (n + 2 * before) * heads[0] * heads[2]  # noqa: E731
    while per() > 2.5e11:       # no more than the longest listed document
        n, before = n * 3 // 4, before * 3 // 4
    batch = _log_int(rng, 1, max(1, min(64, int(1e11 / per()), int(1e8 / ((n + before) * heads[1] * heads[2])))))
    return _attn(batch, (int(n * rng.choice((0.0, 0.1, 0.5, 1.0))) if batch > 1 else n, n), before, *heads)


# ---- inputs ------------------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(((int(seed) * 1000003 + stream) * 7919 + 54321) % (1 << 62))
    return g


def _normal(seed, stream, shape, std=1.0):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda").mul_(std)


def _dtype(name):
    return BF16 if name == "bf16" else torch.float32


def _up(n, to):
    return -(-n // to) * to


def _activations(seed, stream, rows, cols):
    """Rows as a decoder has them: a few channels are much larger than the rest."""
    gain = torch.exp(_normal(seed, stream + 1, (cols,), 0.4))
    gain[:: 97] *= 8.0
    return _normal(seed, stream, (rows, cols)) * gain


def _spread(lo, hi, n, step, start):
    return [lo + int((hi - lo) * ((b * step + start) % 1.0) + 0.5) for b in range(n)]


def _lens(c):
    """Rows of each sequence; with lengths that differ, the first one has the most."""
    return [c["q_max"]] + _spread(c["q_min"], c["q_max"], c["batch"] - 1, 0.618034, 0.35)


def _before(c):
    """Positions of each sequence in front of its first row"""
    n = c["at"] if c["op"] == "append" else c["before"]
    return [n] + _spread(n // 8, n, c["batch"] - 1, 0.414214, 0.2)


def _starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _packed(w, interleave):
    """Row-major [n][k], k a multiple of 32, in the order that the product reads."""
    n, k = w.shape
    if interleave:      # tiles of 16 gate rows and of the same up rows in turn
        w = w.reshape(2, n // 32, 16, k).transpose(0, 1).reshape(n, k)
    p = torch.nn.functional.pad(w, (0, _up(k, 128) - k, 0, _up(n, 16) - n))
    return p.reshape(p.shape[0] // 16, 16, p.shape[1] // 128, 4, 4, 8).permute(2, 0, 3, 4, 1, 5).contiguous().reshape(-1)


def _prepare_rows(c, seed):
    rows, empty = c["rows"], lambda *shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    if c["op"] == "norm":
        return {"x": (4.0 * _activations(seed, 1, rows, c["cols"])).to(_dtype(c["x"])), "gain": 1.0 + _normal(seed, 7, (c["cols"],), 0.2),
                "y": empty(rows, c["cols"], dtype=BF16)}
    n, k = c["n"] * (2 if c["act"] == "swiglu" else 1), c["k"]
    x = _activations(seed, 1, rows, k)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True))
    w = _normal(seed, 4, (n, k), k ** -0.5).to(BF16)
    st = {"x": x.to(BF16), "w": w, "packed": _packed(w, c["act"] == "swiglu"), "y": empty(rows, c["n"], dtype=_dtype(c["y"])),
          "bias": _normal(seed, 5, (n,), 0.3) if c["bias"] else None, "residual": None, "work": empty(1 << 24, dtype=torch.float32)}
    if c["residual"] != "none":
        st["residual"] = (2.0 * _activations(seed, 8, rows, c["n"])).to(_dtype(c["residual"]))
    return st


def _prepare_append(c, seed):
    hq, hk, hd, batch = c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"]
    lens, at = _lens(c), _before(c)
    most = max(n + a for n, a in zip(lens, at))
    rows = sum(lens)
    slots = torch.randperm(batch, generator=_gen(seed, 1), device="cuda").to(torch.int32)
    st = {"qkv": _normal(seed, 2, (rows, (hq + 2 * hk) * hd)).to(BF16), "row0": _ints(_starts(lens)), "slot": slots, "pos0": _ints(at),
          "rotated": torch.empty((rows, (hq + hk) * hd), dtype=BF16, device="cuda"),
          "cache": torch.zeros((batch, _up(most, 32) // 32, hk, 2, 32 * hd), dtype=BF16, device="cuda")}
    if own:     # a model of one layer whose projections do not matter here
        from paper_2411_00853_amd import binding as sv
        cfg = sv.spec_model_cfg(1, 64, hq, hk, hd, 64, 64, batch, most, 0, sv.SPEC_DTYPE_BF16, EPS, THETA)
        flat = lambda n, k: torch.zeros(sv.spec_packed_weight_bytes(n, k) // 2, dtype=BF16, device="cuda")  # noqa: E731
        ones = torch.ones(64, device="cuda")
        w = {"tok_embed": flat(64, 64), "final_norm": ones, "lm_head": flat(64, 64),
             "layers": [{"attn_norm": ones, "ffn_norm": ones, "w_qkv": flat((hq + 2 * hk) * hd, 64), "w_o": flat(64, hq * hd),
                         "w_gate_up": flat(128, 64), "w_down": flat(64, 64)}]}
        st["kv_len"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
        st["handle"] = sv.spec_verify_init(cfg, w, st["cache"], st["kv_len"])
    return st


def _prepare_attn(c, seed):
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    lens, before = _lens(c), _before(c)
    rows, k_lens = sum(lens), [n + a for n, a in zip(lens, before)]
    st = {"q_row0": _ints(_starts(lens)), "out": torch.empty((rows, hq * hd), dtype=BF16, device="cuda"), "max_q": max(lens),
          "max_k": max(k_lens), "work": torch.empty(1 << 24, dtype=torch.float32, device="cuda")}
    spread = torch.exp(_normal(seed, 2, (hk, hd), 0.3))
    if c["before"]:     # new rows behind older keys and values
        kv = _normal(seed, 3, (sum(k_lens), 2, hk, hd)) * spread
        kv = kv.reshape(sum(k_lens), 2 * hk * hd).to(BF16)
        st.update(q=_normal(seed, 1, (rows, hq * hd)).to(BF16), k=kv[:, :hk * hd], v=kv[:, hk * hd:], k_row0=_ints(_starts(k_lens)))
    else:               # whole prompts, as a projection leaves them
        qkv = _normal(seed, 1, (rows, hq + 2 * hk, hd))
        qkv[:, hq:hq + hk] *= spread
        qkv[:, hq + hk:] *= spread
        qkv = qkv.reshape(rows, -1).to(BF16)
        st.update(q=qkv[:, :hq * hd], k=qkv[:, hq * hd:(hq + hk) * hd], v=qkv[:, (hq + hk) * hd:], k_row0=None)
    return st


def prepare(case, seed):
    c = dict(case)
    st = {"norm": _prepare_rows, "gemm": _prepare_rows, "append": _prepare_append, "attn": _prepare_attn}[c["op"]](c, seed)
    st["case"] = c
    return st


# ---- the plain forms ------------------------------------------------------------------------------------

def _plain_norm(st):
    x = st["x"].float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * st["gain"]).to(BF16)


def _plain_gemm(st):
    c = st["case"]
    v = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        v = v + st["bias"]
    if c["act"] == "relu":
        v = v.clamp_min(0.0)
    elif c["act"] == "gelu":
        v = 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    elif c["act"] == "silu":
        v = v / (1.0 + torch.exp(-v))
    elif c["act"] == "swiglu":
        g, u = v.chunk(2, -1)
        v = g / (1.0 + torch.exp(-g)) * u
    if st["residual"] is not None:
        v = v + st["residual"].float()
    return v.to(st["y"].dtype)


def _row_places(row0, rows):
    """The sequence of each row and its place in it."""
    r = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(row0[1:].long(), r, right=True)
    return seq, r - row0.long()[seq]


def _plain_append(st):
    c = st["case"]
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    rows = st["qkv"].shape[0]
    seq, j = _row_places(st["row0"], rows)
    slot, pos = st["slot"].long()[seq], st["pos0"].long()[seq] + j
    angle = pos.double()[:, None] * THETA ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = st["qkv"].float().reshape(rows, hq + 2 * hk, hd)
    a, b = x[:, :hq + hk, : hd // 2], x[:, :hq + hk, hd // 2:]
    turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(BF16)
    st["rotated"].copy_(turned.reshape(rows, -1))
    # [position][head][part of 2][32 head_dim]: where each number goes within its block
    t, d = (pos % 32)[:, None], torch.arange(hd, device="cuda")[None]
    key_at = ((t // 16 * (hd // 8) + d // 8) * 16 + t % 16) * 8 + d % 8
    value_at = 32 * hd + (((d // 16 * 4 + t % 16 // 4) * 16 + d % 16) * 2 + t // 16) * 4 + t % 4
    block = (slot * st["cache"].shape[1] + pos // 32)[:, None] * hk + torch.arange(hk, device="cuda")
    flat = st["cache"].view(-1)
    flat[(block[..., None] * (64 * hd) + key_at[:, None]).reshape(-1)] = turned[:, hq:].reshape(-1)
    flat[(block[..., None] * (64 * hd) + value_at[:, None]).reshape(-1)] = st["qkv"][:, (hq + hk) * hd:].reshape(-1)
    return {"rotated": st["rotated"], "cache": st["cache"]}


def _plain_attn(st):
    c = st["case"]
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    group = hq // hk
    q_row0 = st["q_row0"].tolist()
    k_row0 = q_row0 if st["k_row0"] is None else st["k_row0"].tolist()
    for b in range(c["batch"]):
        n, m = q_row0[b + 1] - q_row0[b], k_row0[b + 1] - k_row0[b]
        if not n:
            continue
        q = st["q"][q_row0[b]:q_row0[b + 1]].float().reshape(n, hk, group, hd)
        k = st["k"][k_row0[b]:k_row0[b + 1]].float().reshape(m, hk, hd)
        v = st["v"][k_row0[b]:k_row0[b + 1]].float().reshape(m, hk, hd)
        place = torch.arange(m, device="cuda")
        for i in range(0, n, 2048):     # a stretch of rows at a time
            w = min(2048, n - i)
            hidden = place > (m - n + i + torch.arange(w, device="cuda"))[:, None]
            for h in range(hk):
                score = q[i:i + w, h].reshape(w * group, hd) @ k[:, h].t().contiguous() * hd ** -0.5
                score = score.reshape(w, group, m).masked_fill_(hidden[:, None], float("-inf"))
                p = torch.exp(score - score.amax(-1, keepdim=True))
                o = p.reshape(w * group, m) @ v[:, h].contiguous() / p.sum(-1).reshape(w * group, 1)
                st["out"][q_row0[b] + i:q_row0[b] + i + w, h * group * hd:(h + 1) * group * hd] = o.reshape(w, group * hd).to(BF16)
    return st["out"]


_PLAIN = {"norm": _plain_norm, "gemm": _plain_gemm, "append": _plain_append, "attn": _plain_attn}


# ---- the framework's kernels ----------------------------------------------------------------------------

def _own(st):
    from paper_2411_00853_amd import binding as sv
    c = st["case"]
    if c["op"] == "norm":
        return sv.spec_prompt_rmsnorm(st["x"], st["gain"], EPS, st["y"])
    if c["op"] == "gemm":
        return sv.spec_prompt_gemm(st["x"], st["packed"], st["y"], bias=st["bias"], activation=c["act"], residual=st["residual"],
                                   workspace=st["work"])
    if c["op"] == "append":
        sv.spec_prompt_append(st["handle"], 0, st["qkv"], st["rotated"], st["row0"], st["slot"], st["pos0"])
        return {"rotated": st["rotated"], "cache": st["cache"]}
    return sv.spec_prompt_attention(st["q"], st["k"], st["v"], c["q_heads"], c["kv_heads"], st["q_row0"], st["out"], c["head_dim"] ** -0.5,
                                    k_row0=st["k_row0"], max_q_len=st["max_q"], max_k_len=st["max_k"], workspace=st["work"])


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------

_BYTES = {"bf16": 2, "fp32": 4, "none": 0}


def work(case):
    c = case
    if c["op"] == "norm":
        return {"bytes": c["rows"] * c["cols"] * (_BYTES[c["x"]] + 2) + 4 * c["cols"], "flops": 4 * c["rows"] * c["cols"]}
    if c["op"] == "gemm":
        m, n, k = c["rows"], c["n"], c["k"]
        of = 2 * n if c["act"] == "swiglu" else n
        return {"bytes": 2 * k * (m + of) + m * n * (_BYTES[c["y"]] + _BYTES[c["residual"]]) + (4 * of if c["bias"] else 0), "flops": 2 * m * of * k}
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    lens, before = _lens(c), _before(c)
    if c["op"] == "append":     # everything in and the rotated heads out, keys and values out once more
        most = max(n + a for n, a in zip(lens, before))
        return {"bytes": sum(lens) * hd * 2 * (2 * hq + 5 * hk) + most * hd * 4, "flops": 3 * sum(lens) * (hq + hk) * hd}
    seen = sum(n * a + n * (n + 1) // 2 for n, a in zip(lens, before))
    return {"bytes": 4 * sum(lens) * hq * hd + 4 * sum(n + a for n, a in zip(lens, before) if n) * hk * hd, "flops": 4 * seen * hq * hd}


# ---- the definition in 64 bits ------------------------------------------------------------------------------

def _exact_append(st):
    """Rotated heads; of the cache what the rotation decides (its values are copies) as the positions of a plain cache."""
    c, d64 = st["case"], torch.float64
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    row0, at = st["row0"].tolist(), st["pos0"].tolist()
    freq = torch.tensor([THETA ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=d64, device="cuda")
    out = []
    for b in range(c["batch"]):
        x = st["qkv"][row0[b]:row0[b + 1], :(hq + hk) * hd].to(d64).reshape(-1, hq + hk, 2, hd // 2)
        phase = torch.outer(torch.arange(at[b], at[b] + x.shape[0], device="cuda").to(d64), freq)
        z = torch.complex(x[:, :, 0], x[:, :, 1]) * torch.polar(torch.ones_like(phase), phase)[:, None]
        out.append(torch.cat((z.real, z.imag), -1).reshape(x.shape[0], -1))
    return {"rotated": torch.cat(out), "cache": None}


def _exact_attn(st):
    c, d64 = st["case"], torch.float64
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    q_row0 = st["q_row0"].tolist()
    k_row0 = q_row0 if st["k_row0"] is None else st["k_row0"].tolist()
    out = torch.zeros((q_row0[-1], hq, hd), dtype=d64, device="cuda")
    for b in range(c["batch"]):
        n, m = q_row0[b + 1] - q_row0[b], k_row0[b + 1] - k_row0[b]
        for h in range(hq):
            kv = slice(h // (hq // hk) * hd, (h // (hq // hk) + 1) * hd)
            keys = st["k"][k_row0[b]:k_row0[b + 1], kv].to(d64).t().contiguous()
            values = st["v"][k_row0[b]:k_row0[b + 1], kv].to(d64)
            for i in range(0, n, 4096):
                w = min(4096, n - i)
                q = st["q"][q_row0[b] + i:q_row0[b] + i + w, h * hd:(h + 1) * hd].to(d64)
                score = (q @ keys) / math.sqrt(hd)
                score += torch.full_like(score, -math.inf).triu(m - n + i + 1)
                out[q_row0[b] + i:q_row0[b] + i + w, h] = torch.softmax(score, -1) @ values
    return out.reshape(-1, hq * hd)


def exact(case, seed):
    st = prepare(case, seed)
    c, d64 = st["case"], torch.float64
    if c["op"] == "norm":
        x = st["x"].to(d64)
        return x / torch.sqrt((x * x).sum(1, keepdim=True) / c["cols"] + EPS) * st["gain"].to(d64)
    if c["op"] == "append":
        return _exact_append(st)
    if c["op"] == "attn":
        return _exact_attn(st)
    v = torch.addmm(torch.zeros((), dtype=d64, device="cuda") if st["bias"] is None else st["bias"].to(d64), st["x"].to(d64),
                    st["w"].to(d64).t().contiguous())
    if c["act"] == "relu":
        v = torch.maximum(v, torch.zeros_like(v))
    elif c["act"] == "gelu":
        v = v * torch.special.ndtr(v)
    elif c["act"] == "silu":
        v = v * torch.sigmoid(v)
    elif c["act"] == "swiglu":
        v = v[:, :c["n"]] * torch.sigmoid(v[:, :c["n"]]) * v[:, c["n"]:]
    return v if st["residual"] is None else v + st["residual"].to(d64)
