"""The operators of a decode step held in 8 bits, and the draw from a filtered distribution.

A case is a dict of sizes.  Its "op" says which operator it takes:

  norm    spec_q8_add_rmsnorm: the residual stream takes a projection's output, and its normalised rows leave in 8 bits
  swiglu  spec_q8_swiglu: silu(gate) * up, in 8 bits
  gemm    spec_q8_gemm: rows in 8 bits times a weight matrix in 8 bits, a scale for each block of 128 on both sides
  attn    spec_kv8_append and spec_kv8_attention: a window's keys and values go into an 8-bit paged cache, its queries read it
  sample  spec_filter_sample: temperature, top-k, top-p, min-p and one draw per row from a given random number

8-bit values are e4m3.  What they stand for is the value times its block's scale:

  rows     q [M][Kp], scales [Kp/128][M]: a scale per row and 128 columns, Kp = columns rounded up to 128, the rest zero
  weights  tiles [Kp/128][Np/16] of [2][4][16][16]: element (h, g, n, e) of tile (kb, j) is row 16j + n, column
           128kb + 64h + 16g + e; scales [ceil(N/128)][Kp/128]; Np = N rounded up to 16
  cache    pages [page][kv head][2][32 * head_dim], scales [page][kv head][2] (powers of two), 32 positions a page;
           key (t, d) at [t/16][d/16][t%16][d%16], value (t, d) at [d/32][(t%16)/4][d%16][(d%32)/16][t/16][t%4]
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
TINY = 2.0 ** -126      # the smallest amax / 448 a scale is made from
MASS_ONE = float(1 << 44)   # a token's mass is floor(MASS_ONE * exp(.)): whole numbers, so that sums are exact
EPS, THETA = 1e-5, 10000.0


# ---- cases -------------------------------------------------------------------------------------------

def _attn(batch, kv, window, q_heads, kv_heads, head_dim, **more):
    return dict({"op": "attn", "batch": batch, "kv_min": kv[0], "kv_max": kv[1], "w_min": window[0], "w_max": window[1],
                 "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim}, **more)


def listed():
    return [
        # one user's token between two layers of the 1B shape: nothing but latency
        {"name": "norm_one_row", "op": "norm", "rows": 1, "cols": 2048, "x": "fp32", "delta": "bf16"},
        # a prompt of the 7B shape
        {"name": "norm_prompt", "op": "norm", "rows": 4096, "cols": 4096, "x": "bf16", "delta": "bf16"},
        # eight users' windows of six, feed-forward of the 7B shape
        {"name": "swiglu_rows48", "op": "swiglu", "rows": 48, "cols": 11008, "x": "bf16"},
        # a ragged prompt, a width that ends inside a block of 128
        {"name": "swiglu_ragged", "op": "swiglu", "rows": 1333, "cols": 5504 + 36, "x": "fp32"},
        # one user's token, output projection of the 7B shape
        {"name": "gemm_one_row", "op": "gemm", "rows": 1, "n": 4096, "k": 4096, "y": "bf16"},
        # eight windows of six, gate and up projection of the 7B shape: the weights' stream
        {"name": "gemm_rows48", "op": "gemm", "rows": 48, "n": 22016, "k": 4096, "y": "bf16"},
        # a prompt, the same projection: the matrix cores
        {"name": "gemm_prompt", "op": "gemm", "rows": 2048, "n": 22016, "k": 4096, "y": "bf16"},
        # one user of the 1B shape, one token
        _attn(1, (1023, 1023), (1, 1), 32, 8, 64, name="attn_one_user"),
        # eight users of the 7B shape, windows of six: the verify step's attention
        _attn(8, (2048, 2048), (6, 6), 32, 32, 128, name="attn_windows"),
        # a full server with shared heads, lengths and windows of all sizes
        _attn(32, (512, 16384), (1, 8), 32, 8, 128, name="attn_ragged"),
        # one user's draw
        {"name": "sample_one_row", "op": "sample", "rows": 1, "vocab": 32000, "x": "fp32", "filters": "kpm", "std": 3.0, "out": True},
        # the draws of a large batch over a large vocabulary: the logits' stream
        {"name": "sample_batch64", "op": "sample", "rows": 64, "vocab": 128256, "x": "fp32", "filters": "kpm", "std": 3.0, "out": False},
    ]


def _log_int(rng, lo, hi, to=1):
    """A size between lo and hi, spread over its logarithm, rounded up to a multiple of `to`."""
    v = -(-min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))) // to) * to
    return v + to if v == 3072 else v       # which is the 1B shape's own projection


def _type(rng):
    return rng.choice(("bf16", "fp32"))


def draw(rng):
    op = rng.choice(("norm", "swiglu", "gemm", "gemm", "attn", "attn", "sample"))
    if op == "norm":
        return {"op": op, "rows": _log_int(rng, 1, 4096), "cols": _log_int(rng, 64, 8192, rng.choice((1, 64, 64))), "x": _type(rng),
                "delta": rng.choice(("bf16", "fp32", "none"))}
    if op == "swiglu":
        return {"op": op, "rows": _log_int(rng, 1, 2048), "cols": _log_int(rng, 64, 14336, rng.choice((1, 64, 64))), "x": _type(rng)}
    if op == "gemm":
        to = rng.choice((1, 128, 128))
        n, k = _log_int(rng, 256, 32003, to), _log_int(rng, 256, 12288, to)
        rows = _log_int(rng, 1, 2048) if n * k < 1 << 26 else _log_int(rng, 1, 768)
        return {"op": op, "rows": rows, "n": n, "k": k, "y": rng.choice(("bf16", "bf16", "fp32"))}
    if op == "attn":
        head_dim, kv_heads = rng.choice((64, 128)), rng.choice((1, 2, 4, 8, 8, 12, 32))
        group = rng.choice((1, 2, 3, 4, 8)) if kv_heads < 12 else 1
        n = _log_int(rng, 1, 32768)
        most = max(1, min(48, (1 << 28) // (n * kv_heads * head_dim * 2)))
        w = _log_int(rng, 1, 16) if rng.random() < 0.85 else _log_int(rng, 16, 256)
        batch = _log_int(rng, 1, min(most, 6) if w > 16 else most)
        return _attn(batch, (int(n * rng.choice((0.0, 0.1, 0.5, 1.0))), n), (rng.randint(0 if batch > 1 else 1, w), w),
                     group * kv_heads, kv_heads, head_dim)
    return {"op": op, "rows": _log_int(rng, 1, 128), "vocab": _log_int(rng, 1000, 131072), "x": _type(rng),
            "filters": rng.choice(("", "k", "p", "m", "kp", "pm", "kpm")), "std": rng.choice((1.0, 2.0, 3.0, 4.0)),
            "out": rng.random() < 0.3}


# ---- inputs ------------------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(((int(seed) * 1000003 + stream) * 7919 + 12345) % (1 << 62))
    return g


def _normal(seed, stream, shape, std=1.0):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda").mul_(std)


def _uniform(seed, stream, shape, lo=0.0, hi=1.0):
    return torch.rand(shape, generator=_gen(seed, stream), device="cuda").mul_(hi - lo).add_(lo)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _up(n, to):
    return -(-n // to) * to


def _activations(seed, stream, rows, cols):
    """Rows as a decoder has them: a few channels are much larger than the rest."""
    gain = torch.exp(_normal(seed, stream + 1, (cols,), 0.4))
    gain[:: 97] *= 12.0
    return _normal(seed, stream, (rows, cols)) * gain


def _blocks_of_rows(y):
    """y [M][K] fp32 -> its blocks [M][Kp/128][128], the last one filled with zeros."""
    m, k = y.shape
    return torch.nn.functional.pad(y, (0, _up(k, 128) - k)).reshape(m, -1, 128)


def _quantise_rows(y):
    b = _blocks_of_rows(y)
    s = b.abs().amax(-1).div(448.0).clamp_min(TINY)
    q = (b / s[..., None]).to(F8)
    return q.reshape(y.shape[0], -1), s.t().contiguous()


def _quantise_weight(w):
    """w [N][K] fp32 -> its 8-bit values [Np][Kp] and the scales of its 128 x 128 blocks."""
    n, k = w.shape
    p = torch.nn.functional.pad(w, (0, _up(k, 128) - k, 0, _up(n, 128) - n))
    b = p.reshape(p.shape[0] // 128, 128, p.shape[1] // 128, 128)
    s = b.abs().amax((1, 3)).div(448.0).clamp_min(TINY)
    q = (b / s[:, None, :, None]).to(F8).reshape(p.shape)[: _up(n, 16)]
    return q.contiguous(), s


def _tiles(q):
    """[Np][Kp] in the order the product reads."""
    n, k = q.shape
    return (q.view(torch.uint8).reshape(n // 16, 16, k // 128, 2, 4, 16).permute(2, 0, 3, 4, 1, 5).contiguous()
            .reshape(-1).view(F8))


def _lens(c, lo, hi):
    return [lo + int((hi - lo) * ((b * 0.618034 + 0.35) % 1.0) + 0.5) for b in range(c["batch"])]


def _windows(c):
    return [c["w_min"] + int((c["w_max"] - c["w_min"] + 1) * ((b * 0.414214 + 0.2) % 1.0)) for b in range(c["batch"])]


def _pow2_scale(amax):
    """The smallest power of two s with amax / s <= 448, at least TINY."""
    mantissa, exponent = torch.frexp(amax)          # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).to(torch.int32)   # 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp_min(-126)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _key_order(x):
    """[..., 32, hd] -> the order of a page's keys."""
    *lead, t, d = x.shape
    n = len(lead)
    return x.reshape(*lead, 2, 16, d // 16, 16).transpose(n + 1, n + 2).reshape(*lead, t * d)


def _value_order(x):
    *lead, t, d = x.shape
    n = len(lead)
    y = x.reshape(*lead, 2, 4, 4, d // 32, 2, 16)            # t/16, g, t%4, d/32, (d%32)/16, d%16
    return y.permute(*range(n), n + 3, n + 1, n + 5, n + 4, n, n + 2).reshape(*lead, t * d)


def _key_rows(x, d):
    *lead, _ = x.shape
    n = len(lead)
    return x.reshape(*lead, 2, d // 16, 16, 16).transpose(n + 1, n + 2).reshape(*lead, 32, d)


def _value_rows(x, d):
    *lead, _ = x.shape
    n = len(lead)
    y = x.reshape(*lead, d // 32, 4, 16, 2, 2, 4)            # d/32, g, d%16, (d%32)/16, t/16, t%4
    return y.permute(*range(n), n + 4, n + 1, n + 5, n, n + 3, n + 2).reshape(*lead, 32, d)


def _prepare_attn(c, seed):
    hq, hk, hd, batch = c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"]
    lens, win = _lens(c, c["kv_min"], c["kv_max"]), _windows(c)
    most = max(n + w for n, w in zip(lens, win))
    blocks = -(-most // 32)
    taken = [-(-(n + w) // 32) for n, w in zip(lens, win)]
    pages = sum(taken) + 3
    order = torch.randperm(pages, generator=_gen(seed, 1), device="cuda").to(torch.int32)
    table, at = torch.full((batch, blocks), -1, dtype=torch.int32, device="cuda"), 0
    for b, n in enumerate(taken):
        table[b, :n] = order[at:at + n]
        at += n
    data = torch.empty((pages, hk, 2, 32 * hd), dtype=F8, device="cuda")
    scales = torch.empty((pages, hk, 2), device="cuda")
    spread = torch.exp(_normal(seed, 2, (2, hk, 1, hd), 0.3))
    step = max(1, (1 << 26) // (hk * 64 * hd))
    for p in range(0, pages, step):     # a stretch of pages at a time
        n = min(step, pages - p)
        for kv, put in ((0, _key_order), (1, _value_order)):
            x = _normal(seed, 1000 + 2 * p + kv, (n, hk, 32, hd)) * spread[kv]
            s = _pow2_scale(x.abs().amax((2, 3)))
            scales[p:p + n, :, kv] = s
            data[p:p + n, :, kv] = put(x / s[:, :, None, None]).to(F8)
    rows = sum(win)
    row0 = [0]
    for w in win:
        row0.append(row0[-1] + w)
    qkv = _normal(seed, 3, (rows, hq + 2 * hk, hd))
    qkv[:, hq:hq + hk] *= spread[0, :, 0]
    qkv[:, hq + hk:] *= spread[1, :, 0]
    angle = torch.arange(most, device="cuda", dtype=torch.float64)[:, None] * \
        THETA ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)
    bf = lambda shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    return {"case": c, "data": data, "scales": scales, "table": table, "max_window": max(win), "max_len": most,
            "qkv": qkv.reshape(rows, -1).to(torch.bfloat16),
            "row0": torch.tensor(row0, dtype=torch.int32, device="cuda"),
            "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "cos_sin": torch.stack((angle.cos(), angle.sin()), -1).float().contiguous(),
            "q": bf((rows, hq * hd)), "out": bf((rows, hq * hd)),
            "work": torch.empty(1 << 24, dtype=torch.float32, device="cuda")}     # results of the parts of a long cache


def _logits(c, seed):
    x = _normal(seed, 1, (c["rows"], c["vocab"]), c["std"])
    x[:, :: 501] += 1.5 * c["std"]      # what a trained model singles out
    return x.to(_dtype(c["x"]))


def prepare(case, seed):
    c = dict(case)
    rows = c.get("rows", 0)
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["op"] in ("norm", "swiglu"):
        cols = c["cols"]
        kp = _up(cols, 128)
        st = {"case": c, "q": empty((rows, kp), F8), "s": empty((kp // 128, rows), torch.float32)}
        if c["op"] == "swiglu":
            st["x"] = _activations(seed, 1, rows, 2 * cols).to(_dtype(c["x"]))
            return st
        st["x"] = (4.0 * _activations(seed, 1, rows, cols)).to(_dtype(c["x"]))
        st["delta"] = None if c["delta"] == "none" else _activations(seed, 5, rows, cols).to(_dtype(c["delta"]))
        st["gain"] = 1.0 + _normal(seed, 7, (cols,), 0.2)
        st["h"] = torch.empty_like(st["x"])
        return st
    if c["op"] == "gemm":
        q, s = _quantise_rows(_activations(seed, 1, rows, c["k"]))
        w, ws = _quantise_weight(_normal(seed, 4, (c["n"], c["k"]), c["k"] ** -0.5))
        return {"case": c, "q": q, "s": s, "w": w, "ws": ws, "tiles": _tiles(w), "y": empty((rows, c["n"]), _dtype(c["y"]))}
    if c["op"] == "attn":
        return _prepare_attn(c, seed)
    on = c["filters"]
    st = {"case": c, "x": _logits(c, seed), "u": _uniform(seed, 2, (rows,)).clamp_max(1.0 - 2.0 ** -24),
          "t": _uniform(seed, 3, (rows,), 0.6, 1.2), "top_k": None, "top_p": None, "min_p": None,
          "tokens": empty((rows,), torch.int32), "kept": empty((rows,), torch.int32), "logprob": empty((rows,), torch.float32),
          "filtered": empty((rows, c["vocab"]), torch.float32) if c["out"] else None,
          "work": empty((rows, 32768), torch.float32)}      # what the parts of a long row leave to each other
    if "k" in on:
        st["top_k"] = torch.randint(20, 200, (rows,), generator=_gen(seed, 4), device="cuda", dtype=torch.int32)
    if "p" in on:
        st["top_p"] = _uniform(seed, 5, (rows,), 0.8, 0.98)
    if "m" in on:
        st["min_p"] = _uniform(seed, 6, (rows,), 0.01, 0.05)
    return st


# ---- the plain forms ------------------------------------------------------------------------------------

def _plain_norm(st):
    h = st["x"].float()
    if st["delta"] is not None:
        h = h + st["delta"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * st["gain"]
    q, s = _quantise_rows(y)
    return {"h": h.to(st["x"].dtype), "q": q, "scales": s}


def _plain_swiglu(st):
    g, u = st["x"].float().chunk(2, -1)
    q, s = _quantise_rows(g / (1.0 + torch.exp(-g)) * u)
    return {"q": q, "scales": s}


def _plain_gemm(st):
    n, m = st["case"]["n"], st["q"].shape[0]
    x = (st["q"].float().reshape(m, -1, 128) * st["s"].t()[..., None]).reshape(m, -1)
    w = st["w"].float()
    w = (w.reshape(w.shape[0], -1, 128) * st["ws"].repeat_interleave(128, 0)[: w.shape[0], :, None]).reshape(w.shape)
    return (x @ w.t())[:, :n].to(st["y"].dtype)


def _plain_attn(st):
    c, f = st["case"], torch.float32
    hq, hk, hd, batch = c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"]
    rows, most_w = st["qkv"].shape[0], st["max_window"]
    row0, kv_len, table = st["row0"].long(), st["kv_len"].long(), st["table"].long()
    win = row0[1:] - row0[:-1]
    arange = lambda n: torch.arange(n, device="cuda")  # noqa: E731
    seq = torch.searchsorted(row0[1:], arange(rows), right=True)
    slot = arange(rows) - row0[seq]                                  # a row's place in its window
    cs = st["cos_sin"][kv_len[seq] + slot][:, None]                  # [rows][1][hd/2][2]
    x = st["qkv"].to(f).reshape(rows, hq + 2 * hk, hd)
    a, b = x[:, :hq + hk, : hd // 2], x[:, :hq + hk, hd // 2:]
    turned = torch.cat((a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]), -1)
    q, new = turned[:, :hq].to(torch.bfloat16), torch.stack((turned[:, hq:], x[:, hq + hk:]), 1)   # new [rows][2][hk][hd]
    # the pages the windows reach: i-th from the one that holds position kv_len
    nb = (most_w + 30) // 32 + 1
    blk = kv_len[:, None] // 32 + arange(nb)                         # [batch][nb]
    live = blk * 32 < (kv_len + win)[:, None]
    page = table.gather(1, blk.clamp_max(table.shape[1] - 1))
    page = torch.where(live, page, 0)
    pos = blk[..., None] * 32 + arange(32)                           # [batch][nb][32]
    j = pos - kv_len[:, None, None]
    fresh = (j >= 0) & (j < win[:, None, None])
    older = j < 0
    incoming = new[(row0[:-1, None, None] + j).clamp(0, rows - 1)]   # [batch][nb][32][2][hk][hd]
    incoming = (incoming * fresh[..., None, None, None]).permute(0, 1, 4, 3, 2, 5)    # [batch][nb][hk][2][32][hd]
    need = _pow2_scale(incoming.abs().amax((-1, -2)))                # [batch][nb][hk][2]
    raw = st["data"].view(torch.uint8)[page].view(F8).to(f)          # [batch][nb][hk][2][32 hd]
    old = torch.stack((_key_rows(raw[..., 0, :], hd), _value_rows(raw[..., 1, :], hd)), 3)
    was = st["scales"][page]
    s = torch.where(older.any(-1)[..., None, None], torch.maximum(was, need), need)
    at = lambda mask: mask[:, :, None, None, :, None]  # noqa: E731
    put = torch.where(at(fresh), incoming / s[..., None, None], torch.where(at(older), old * (was / s)[..., None, None], old)).to(F8)
    put = torch.stack((_key_order(put[:, :, :, 0].view(torch.uint8)), _value_order(put[:, :, :, 1].view(torch.uint8))), 3)
    st["data"].view(torch.uint8)[page[live]] = put[live]
    st["scales"][page[live]] = s[live]
    # attention, windows and lengths filled up to the largest
    pages = table.clamp_min(0)
    span = pages.shape[1] * 32
    held = st["data"].view(torch.uint8)[pages].view(F8).to(f) * st["scales"][pages][..., None]    # [batch][blocks][hk][2][32 hd]
    k = _key_rows(held[..., 0, :], hd).transpose(1, 2).reshape(batch * hk, span, hd)
    v = _value_rows(held[..., 1, :], hd).transpose(1, 2).reshape(batch * hk, span, hd)
    group = hq // hk
    qp = q[(row0[:-1, None] + arange(most_w)).clamp_max(rows - 1)].to(f)                # [batch][most_w][hq][hd]
    qp = qp.reshape(batch, most_w, hk, group, hd).permute(0, 2, 3, 1, 4).reshape(batch * hk, group * most_w, hd)
    score = (qp @ k.transpose(1, 2).contiguous()).mul_(hd ** -0.5).reshape(batch, hk, group, most_w, span)
    sees = arange(span) <= (kv_len[:, None] + arange(most_w))[..., None]                 # [batch][most_w][span]
    score = score.masked_fill(~sees[:, None, None], float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).reshape(batch * hk, group * most_w, span)
    o = (p @ v).reshape(batch, hk, group, most_w, hd).permute(0, 3, 1, 2, 4).reshape(batch, most_w, hq * hd)
    return {"out": o[seq, slot].to(torch.bfloat16), "data": st["data"], "scales": st["scales"]}


def _plain_sample(st):
    x, t = st["x"].float(), st["t"]
    v = x.shape[1]
    top = x.amax(-1, keepdim=True)
    w = (torch.exp((x - top) / t[:, None]) * MASS_ONE).to(torch.int64)      # whole numbers: a sum does not depend on its order
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices         # equal logits: the lowest id first
    ws = w.gather(1, order)
    keep = ws > 0
    if st["top_k"] is not None:
        keep &= torch.arange(v, device="cuda") < st["top_k"][:, None]
    ws = ws * keep
    if st["top_p"] is not None:     # a token stays if the mass before it has not reached the share yet
        before = ws.cumsum(-1) - ws
        keep &= before < (ws.sum(-1).double() * st["top_p"].double()).ceil().to(torch.int64)[:, None]
    if st["min_p"] is not None:
        keep &= ws >= (st["min_p"].double() * MASS_ONE).ceil().to(torch.int64)[:, None]
    keep = torch.zeros_like(keep).scatter_(1, order, keep)                  # by id again
    w = w * keep
    c = w.cumsum(-1)
    total = c[:, -1]
    target = torch.minimum((st["u"].double() * total.double()).floor().to(torch.int64), total - 1)
    token = (c <= target[:, None]).sum(-1)
    mass = w.gather(1, token[:, None])[:, 0]
    out = {"tokens": token.to(torch.int32), "kept": keep.sum(-1).to(torch.int32),
           "logprob": torch.log(mass.float() / total.float())}
    if st["filtered"] is not None:
        out["filtered"] = x.masked_fill(~keep, float("-inf"))
    return out


_PLAIN = {"norm": _plain_norm, "swiglu": _plain_swiglu, "gemm": _plain_gemm, "attn": _plain_attn, "sample": _plain_sample}


# ---- the framework's kernels ----------------------------------------------------------------------------

def _own(st):
    from paper_2411_00853_amd import binding as sv
    c = st["case"]
    if c["op"] == "norm":
        sv.spec_q8_add_rmsnorm(st["x"], st["delta"], st["gain"], EPS, st["h"], st["q"], st["s"])
        return {"h": st["h"], "q": st["q"], "scales": st["s"]}
    if c["op"] == "swiglu":
        sv.spec_q8_swiglu(st["x"], st["q"], st["s"])
        return {"q": st["q"], "scales": st["s"]}
    if c["op"] == "gemm":
        sv.spec_q8_gemm(st["q"], st["s"], st["tiles"], st["ws"], st["y"])
        return st["y"]
    if c["op"] == "attn":
        cache = sv.Kv8Cache(st["data"], st["scales"], st["table"], c["head_dim"])
        sv.spec_kv8_append(cache, st["qkv"], st["row0"], st["kv_len"], c["q_heads"], st["max_window"], st["cos_sin"], st["q"])
        sv.spec_kv8_attention(cache, st["q"], st["row0"], st["kv_len"], c["q_heads"], st["max_window"], st["max_len"],
                              c["head_dim"] ** -0.5, st["out"], st["work"])
        return {"out": st["out"], "data": st["data"], "scales": st["scales"]}
    sv.spec_filter_sample(st["x"], st["u"], st["t"], st["tokens"], st["top_k"], st["top_p"], st["min_p"], st["logprob"],
                          st["kept"], st["filtered"], st["work"])
    out = {"tokens": st["tokens"], "kept": st["kept"], "logprob": st["logprob"]}
    if st["filtered"] is not None:
        out["filtered"] = st["filtered"]
    return out


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------

_BYTES = {"bf16": 2, "fp32": 4, "none": 0}


def work(case):
    c = case
    if c["op"] == "norm":
        m, k = c["rows"], c["cols"]
        return {"bytes": m * k * (2 * _BYTES[c["x"]] + _BYTES[c["delta"]] + 1) + 4 * k + 4 * m * (_up(k, 128) // 128), "flops": 7 * m * k}
    if c["op"] == "swiglu":
        m, k = c["rows"], c["cols"]
        return {"bytes": m * k * (2 * _BYTES[c["x"]] + 1) + 4 * m * (_up(k, 128) // 128), "flops": 7 * m * k}
    if c["op"] == "gemm":
        m, n, k = c["rows"], c["n"], c["k"]
        return {"bytes": m * k + n * k + m * n * _BYTES[c["y"]] + 4 * (m + n / 128) * (k / 128), "flops": 2 * m * n * k}
    if c["op"] == "attn":
        lens, win = _lens(c, c["kv_min"], c["kv_max"]), _windows(c)
        hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
        seen = sum(w * n + w * (w + 1) // 2 for n, w in zip(lens, win))
        # the cache before the window once, the window's queries, keys and values in, its keys, values and outputs out
        read = sum(n * hk * (2 * hd + 8 / 32) for n, w in zip(lens, win) if w)
        return {"bytes": read + sum(win) * (hq * hd * 4 + hk * hd * 6), "flops": 4 * seen * hq * hd}
    m, v = c["rows"], c["vocab"]
    return {"bytes": m * v * (_BYTES[c["x"]] + (4 if c["out"] else 0)) + 24 * m, "flops": 6 * m * v}


# ---- the definition in 64 bits ------------------------------------------------------------------------------

def _exact_rows(y):
    """What the 8-bit numbers stand for before they are rounded, in units of the scale, and the scales."""
    m, k = y.shape
    kp = _up(k, 128)
    s, q = torch.zeros((kp // 128, m), dtype=torch.float64, device="cuda"), torch.zeros((m, kp), dtype=torch.float64, device="cuda")
    for b in range(kp // 128):
        part = y[:, 128 * b:min(k, 128 * b + 128)]
        s[b] = torch.clamp(part.abs().max(1).values / 448, min=TINY)
        q[:, 128 * b:128 * b + part.shape[1]] = part / s[b][:, None]
    return q, s


def _exact_attn(st):
    c = st["case"]
    hq, hk, hd = c["q_heads"], c["kv_heads"], c["head_dim"]
    d64 = torch.float64
    t, d = torch.meshgrid(torch.arange(32, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    key_at = ((t // 16 * (hd // 16) + d // 16) * 16 + t % 16) * 16 + d % 16
    value_at = ((((d // 32 * 4 + t % 16 // 4) * 16 + d % 16) * 2 + d % 32 // 16) * 2 + t // 16) * 4 + t % 4
    row0, lens, out = st["row0"].tolist(), st["kv_len"].tolist(), []
    for b in range(c["batch"]):
        n, w = lens[b], row0[b + 1] - row0[b]
        if not w:
            continue
        new = st["qkv"][row0[b]:row0[b + 1]].to(d64).reshape(w, hq + 2 * hk, hd)
        cos, sin = st["cos_sin"][n:n + w].to(d64).unbind(-1)
        even, odd = new[..., : hd // 2], new[..., hd // 2:]
        rot = torch.cat((even * cos[:, None] - odd * sin[:, None], odd * cos[:, None] + even * sin[:, None]), -1)
        q = rot[:, :hq].to(torch.bfloat16).to(d64)
        pages = st["table"][b, : -(-(n + w) // 32)].long()
        held = [[], []]
        for kv, where in ((0, key_at), (1, value_at)):
            vals = st["data"].view(torch.uint8)[pages][:, :, kv][:, :, where].view(F8).to(d64)        # [pages][hk][32][hd]
            scale = st["scales"][pages][:, :, kv].to(d64)
            fresh = (rot[:, hq:hq + hk] if kv == 0 else new[:, hq + hk:]).transpose(0, 1)              # [hk][w][hd]
            whole = (vals * scale[..., None, None]).transpose(0, 1).reshape(hk, -1, hd)[:, :n]
            for blk in range(n // 32, len(pages)):
                lo, hi = max(32 * blk, n), min(32 * blk + 32, n + w)
                part = fresh[:, lo - n:hi - n]
                s = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)) / 448).clamp_min(-126.0)))
                if 32 * blk < n:
                    s = torch.maximum(s, scale[blk])
                    older = whole[:, 32 * blk:n] / s[:, None, None]
                    whole = torch.cat((whole[:, : 32 * blk], older.float().to(F8).to(d64) * s[:, None, None]), 1)
                part = (part / s[:, None, None]).float().to(F8).to(d64) * s[:, None, None]
                whole = torch.cat((whole, part), 1)
            held[kv] = whole
        seen = torch.arange(n + w, device="cuda")
        o = torch.empty((w, hq, hd), dtype=d64, device="cuda")
        for h in range(hk):
            g = slice(h * (hq // hk), (h + 1) * (hq // hk))
            score = torch.tensordot(q[:, g], held[0][h], dims=([2], [1])) / math.sqrt(hd)            # [w][group][n + w]
            score = score.masked_fill(seen > (n + torch.arange(w, device="cuda"))[:, None, None], -math.inf)
            o[:, g] = torch.tensordot(torch.softmax(score, -1), held[1][h], dims=([2], [0]))
        out.append(o.reshape(w, -1))
    return {"out": torch.cat(out), "data": None, "scales": None}


def exact(case, seed):
    st = prepare(case, seed)
    c, d64 = st["case"], torch.float64
    if c["op"] == "norm":
        h = st["x"].to(d64) + (0 if st["delta"] is None else st["delta"].to(d64))
        rms = torch.sqrt((h * h).sum(1) / c["cols"] + EPS)
        q, s = _exact_rows(h / rms[:, None] * st["gain"].to(d64))
        return {"h": h, "q": q, "scales": s}
    if c["op"] == "swiglu":
        g, u = st["x"][:, : c["cols"]].to(d64), st["x"][:, c["cols"]:].to(d64)
        q, s = _exact_rows(g * torch.sigmoid(g) * u)
        return {"q": q, "scales": s}
    if c["op"] == "gemm":
        y = torch.zeros((c["rows"], c["n"]), dtype=d64, device="cuda")
        for kb in range(st["s"].shape[0]):
            k = slice(128 * kb, 128 * kb + 128)
            part = st["q"][:, k].to(d64) @ st["w"][: c["n"], k].to(d64).t().contiguous()
            y += part * st["s"][kb].to(d64)[:, None] * st["ws"][:, kb].to(d64).repeat_interleave(128)[: c["n"]]
        return y
    if c["op"] == "attn":
        return _exact_attn(st)
    # the tokens and the kept sets are whole numbers; the probability of the token that the definition picks
    x, logp = st["x"].to(d64), []
    for r in range(c["rows"]):
        p = torch.exp((x[r] - x[r].max()) / st["t"][r].to(d64))
        ids = torch.argsort(p, descending=True, stable=True)
        ps = p[ids]
        n = c["vocab"] if st["top_k"] is None else int(st["top_k"][r])
        ps = torch.cat((ps[:n], torch.zeros_like(ps[n:])))
        if st["top_p"] is not None:
            ps = torch.where(torch.cumsum(ps, 0) - ps < float(st["top_p"][r]) * ps.sum(), ps, torch.zeros_like(ps))
        if st["min_p"] is not None:
            ps = torch.where(ps >= float(st["min_p"][r]), ps, torch.zeros_like(ps))
        kept = torch.zeros_like(p).scatter_(0, ids, ps)
        cdf = torch.cumsum(kept, 0)
        token = int((cdf <= float(st["u"][r]) * cdf[-1]).sum())
        logp.append(torch.log(kept[min(token, c["vocab"] - 1)] / cdf[-1]))
    out = {"tokens": None, "kept": None, "logprob": torch.stack(logp)}
    if st["filtered"] is not None:
        out["filtered"] = None
    return out
