"""Plain forms in 64 bits of the operators on packed prompts, and small helpers of their tests."""
import torch

from paper_2411_00853_amd import binding as sv

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
HALF_BF16 = 2.0 ** -8       # a rounding to bf16, relative to the value
HALF_F32 = 2.0 ** -24


def gen(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def normal(seed, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def small_ints(seed, *shape, most=8):
    """Whole numbers whose products and sums fp32 holds exactly."""
    return torch.randint(-most, most + 1, shape, generator=gen(seed), device="cuda").to(BF16)


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def activate(v, act):
    if act == "relu":
        return torch.where(v < 0, torch.zeros_like(v), v)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5))
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "swiglu":
        g, u = v.chunk(2, -1)
        return g * torch.sigmoid(g) * u
    return v


def product(x, w, bias=None, act="none", residual=None):
    v = x.to(F64) @ w.to(F64).t().contiguous()
    if bias is not None:
        v = v + bias.to(F64)
    v = activate(v, act)
    return v if residual is None else v + residual.to(F64)


def rotate(x, pos, theta):
    """x [rows][heads][hd] in 64 bits."""
    hd = x.shape[-1]
    a = pos.to(F64)[:, None] * theta ** (-torch.arange(0, hd, 2, device=x.device, dtype=F64) / hd)
    c, s = a.cos()[:, None], a.sin()[:, None]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


def attend(q, k, v, n_kv_heads, scale, q_lens, k_lens):
    """fp64 (out, sum of the weighted magnitudes of values, largest possible error of a score in units of 2^-24) of packed rows; rows that see
    nothing are zero."""
    rows, cols = q.shape
    hd = k.shape[1] // n_kv_heads
    heads = cols // hd
    out, mags, err = (torch.zeros((rows, heads, hd), dtype=F64, device=q.device) for _ in range(3))
    qs, ks = starts(q_lens), starts(k_lens)
    for b, (n, m) in enumerate(zip(q_lens, k_lens)):
        see = torch.arange(m, device=q.device) <= (m - n + torch.arange(n, device=q.device))[:, None]
        for h in range(heads):
            g = h // (heads // n_kv_heads)
            qq = q[qs[b]:qs[b] + n, h * hd:(h + 1) * hd].to(F64)
            kk = k[ks[b]:ks[b] + m, g * hd:(g + 1) * hd].to(F64)
            vv = v[ks[b]:ks[b] + m, g * hd:(g + 1) * hd].to(F64)
            s = (qq @ kk.t().contiguous() * scale).masked_fill(~see, float("-inf"))
            p = torch.softmax(s, -1)
            p = torch.where(see.any(-1)[:, None], p, torch.zeros_like(p))
            out[qs[b]:qs[b] + n, h] = p @ vv
            mags[qs[b]:qs[b] + n, h] = p @ vv.abs()
            if m and n:
                big = (qq.abs() @ kk.abs().t().contiguous() * abs(scale)).masked_fill(~see, 0).amax(-1)
                err[qs[b]:qs[b] + n, h] = big[:, None].expand(n, hd)
    return out.reshape(rows, cols), mags.reshape(rows, cols), err.reshape(rows, cols)


def attention_tolerance(out, mags, big, hd):
    """Weights: each is rounded to bf16 once (2^-8); its exponent, a sum of hd products in fp32 (hd 2^-23 of the sum of their magnitudes, at most),
    times a factor and less the maximum (three roundings of numbers up to that sum), is off by d, and so the weight by e^d - 1, as is the sum of
    weights; exp2, sums of the weights and the division: some 2^-20 and, in sums of up to 2^12 numbers added one by one, 2^-12 at
    the very most.  The result is rounded once (2^-8)."""
    d = big * ((hd + 6) * 2.0 ** -23)
    return mags * (HALF_BF16 + 2 * torch.expm1(2 * d) + 2.0 ** -12 + 2.0 ** -20) * (1 + HALF_BF16) + out.abs() * HALF_BF16 + 1e-30


def pack(w, interleave=False):
    return sv.spec_pack_weight(w.contiguous(), interleave)


def handle(n_layers=1, hq=4, hk=2, hd=64, slots=3, max_kv=96, pages=0, theta=10000.0, d=64, seed=1):
    """A small bf16 model whose projections do not matter; pages > 0: a pool of so many."""
    cfg = sv.spec_model_cfg(n_layers, d, hq, hk, hd, 64, 64, slots, max_kv, 3, sv.SPEC_DTYPE_BF16, 1e-5, theta)
    w = lambda n, k: pack(normal(seed, n, k, std=0.05, dtype=BF16))  # noqa: E731
    ones = torch.ones(d, device="cuda")
    weights = {"tok_embed": normal(seed, 64, d, dtype=BF16), "final_norm": ones, "lm_head": w(64, d),
               "layers": [{"attn_norm": ones, "ffn_norm": ones, "w_qkv": w((hq + 2 * hk) * hd, d), "w_o": w(d, hq * hd),
                           "w_gate_up": pack(normal(seed, 128, d, dtype=BF16), True), "w_down": w(d, 64)} for _ in range(n_layers)]}
    nbytes = pages * sv.spec_kv_page_bytes(cfg) if pages else sv.spec_kv_cache_bytes(cfg)
    cache = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
    kv_len = torch.zeros(slots, dtype=I32, device="cuda")
    return sv.spec_verify_init(cfg, weights, cache, kv_len, paged=bool(pages)), cache, kv_len
