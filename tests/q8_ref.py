"""Plain 64-bit forms of the 8-bit operators and the filtered draw, for their tests.  Works on CPU and GPU tensors."""
import math

import torch

F8 = torch.float8_e4m3fn
U = 2.0 ** -24       # unit roundoff of fp32
TINY = 2.0 ** -126


def blocks_of(cols):
    return (cols + 127) // 128


def within_half_step(q, value, slack=1e-5):
    """Whether e4m3 numbers q (as fp64) are nearest to `value`: half a step is 2^-4 of a normal number at most, and 2^-10 below
    the normal numbers.  slack: relative error of `value` itself."""
    step = torch.maximum(torch.exp2(torch.floor(torch.log2(value.abs().clamp_min(2.0 ** -6))) - 3), torch.full_like(value, 2.0 ** -9))
    return (q - value).abs() <= step / 2 + slack * value.abs() + 1e-30


def check_rows(q, scales, y, slack):
    """q [M][Kp], scales [Kp/128][M] against the fp64 rows y; slack: relative error allowed to what is rounded."""
    m, k = y.shape
    nb = blocks_of(k)
    assert q.shape == (m, nb * 128) and scales.shape == (nb, m)
    pad = torch.nn.functional.pad(y, (0, nb * 128 - k)).reshape(m, nb, 128)
    want = (pad.abs().amax(-1) / 448).clamp_min(TINY)
    s = scales.double().t()
    assert torch.all((s - want).abs() <= slack * want)
    qd = q.float().double().reshape(m, nb, 128)
    assert torch.all(within_half_step(qd, pad / s[..., None], slack))
    assert torch.all(q.view(torch.uint8).reshape(m, -1)[:, k:] & 0x7f == 0)


def quantise_rows(y):
    m, k = y.shape
    b = torch.nn.functional.pad(y.float(), (0, blocks_of(k) * 128 - k)).reshape(m, -1, 128)
    s = (b.abs().amax(-1) / 448).clamp_min(TINY)
    return (b / s[..., None]).to(F8).reshape(m, -1), s.t().contiguous()


def quantise_weight(w):
    n, k = w.shape
    p = torch.nn.functional.pad(w.float(), (0, -k % 128, 0, -n % 128))
    b = p.reshape(p.shape[0] // 128, 128, p.shape[1] // 128, 128)
    s = (b.abs().amax((1, 3)) / 448).clamp_min(TINY)
    q = (b / s[:, None, :, None]).to(F8).reshape(p.shape)
    return q[:n, :k].contiguous(), s


def gemm(q, scales, w, w_scales):
    """(y, sum of the magnitudes of what is added up, the largest product a block can hold summed over blocks) in fp64; w [N][K]."""
    n, k = w.shape
    kp = q.shape[1]
    x = (q.float().double().reshape(q.shape[0], -1, 128) * scales.double().t()[..., None]).reshape(q.shape)
    wd = torch.nn.functional.pad(w.float().double(), (0, kp - k))
    wd = wd * w_scales.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :kp]
    top = x.abs().reshape(x.shape[0], -1, 128).amax(-1) @ wd.abs().reshape(n, -1, 128).amax(-1).t().contiguous()
    return x @ wd.t().contiguous(), x.abs() @ wd.abs().t().contiguous(), top


# ---- the cache -----------------------------------------------------------------------------------------

def key_byte(t, d, hd):
    return ((t // 16) * (hd // 16) + d // 16) * 256 + (t % 16) * 16 + d % 16


def value_byte(t, d, hd):
    return (d // 32) * 1024 + ((t % 16) // 4) * 256 + (d % 16) * 16 + (d % 32 // 16) * 8 + (t // 16) * 4 + t % 4


def order(hd, kv, device):
    t = torch.arange(32, device=device)[:, None]
    d = torch.arange(hd, device=device)[None]
    return (value_byte if kv else key_byte)(t, d, hd)


def page_rows(data, hd):
    """data [..., 2, 32 * hd] e4m3 -> [..., 2, 32, hd] e4m3."""
    u = data.view(torch.uint8)
    return torch.stack([u[..., kv, :][..., order(hd, kv, u.device)] for kv in (0, 1)], -3).view(F8)


def make_pages(rows, hd):
    """[..., 2, 32, hd] e4m3 -> [..., 2, 32 * hd]."""
    u = rows.view(torch.uint8)
    out = torch.empty((*u.shape[:-2], 32 * hd), dtype=torch.uint8, device=u.device)
    for kv in (0, 1):
        out[..., kv, :][..., order(hd, kv, u.device).reshape(-1)] = u[..., kv, :, :].reshape(*u.shape[:-3], -1)
    return out.view(F8)


def pow2_scale(amax):
    """Smallest power of two s with amax / s <= 448, fp64 in and out, at least 2^-126."""
    s = torch.exp2(torch.ceil(torch.log2(amax.clamp_min(1e-300) / 448)).clamp_min(-126))
    s = torch.where(amax / s > 448, s * 2, s)
    return torch.where((amax / (s / 2) <= 448) & (s > TINY), s / 2, s)


def rotate(x, cos_sin):
    """x [w][heads][hd] fp64, cos_sin [w][hd/2][2]."""
    a, b = x.chunk(2, -1)
    c, s = cos_sin.double()[:, None, :, 0], cos_sin.double()[:, None, :, 1]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def attend(q, keys, values, lims, scale):
    """q [w][hq][hd], keys/values [T][hk][hd] fp64, lims [w] (last visible position), visible [T] bool or None.
    Returns (out [w][hq][hd], sum of weights times |value|)."""
    w, hq, hd = q.shape
    hk = keys.shape[1]
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    pos = torch.arange(keys.shape[0], device=q.device)
    for h in range(hq):
        kv = h // (hq // hk)
        for j in range(w):
            on = pos <= lims[j]
            if not bool(on.any()):
                continue
            p = torch.softmax((keys[on, kv] @ q[j, h]) * scale, 0)
            out[j, h] = p @ values[on, kv]
            mag[j, h] = p @ values[on, kv].abs()
    return out, mag


# ---- the filtered draw -----------------------------------------------------------------------------------

def filtered(x, t, k, p, mp, slack=0.0):
    """The kept tokens of one row (bool [V]) and the masses, fp64.  slack: moves the thresholds of top-p and min-p by that share,
    a negative one keeps less."""
    x = x.double()
    v = x.numel()
    if t <= 0:
        w = torch.zeros_like(x)
        w[int(torch.argmax(x))] = 1.0
        return w > 0, w
    w = torch.exp((x - x.max()) / t)
    w = torch.where(w < 2.0 ** -44 * (1 - slack), torch.zeros_like(w), w)
    ids = torch.sort(x, dim=0, descending=True, stable=True).indices
    ws = w[ids]
    keep = ws > 0
    if k > 0:
        keep[min(k, v):] = False
    z = float(ws[keep].sum())
    if p < 1:
        before = torch.cumsum(ws, 0) - ws
        keep &= before < max(p * z * (1 + slack), 1e-300)
    if mp > 0:
        keep &= ws >= min(mp, 1.0) * (1 - slack)
    keep[0] = True
    out = torch.zeros(v, dtype=torch.bool, device=x.device)
    out[ids] = keep
    return out, w


def check_draw(x, u, t, k, p, mp, token, n_kept, logprob, row_out, margin=1e-5):
    """One row's results against the definition.  A mass has a relative error of at most margin / 2: the exponent (at most 31) is a
    rounded difference and a rounded quotient, 2 * 31 * 2^-24, the exponential another 2^-23, in all below 5e-6."""
    few, w = filtered(x, t, k, p, mp, -margin)
    many, _ = filtered(x, t, k, p, mp, margin)
    assert int(few.sum()) <= n_kept <= int(many.sum())
    if row_out is not None:
        kept = row_out > -math.inf
        assert int(kept.sum()) == n_kept
        assert bool((kept | ~few).all()) and bool((many | ~kept).all())
        assert torch.equal(row_out[kept], x.float()[kept])
    else:
        kept = filtered(x, t, k, p, mp)[0]
    assert bool(many[token])
    w = w * kept
    c = torch.cumsum(w, 0)
    total = float(c[-1])
    lo, hi = float(c[token] - w[token]), float(c[token])
    extra = 0.0 if row_out is not None else float((w * 0 + (many & ~few)).sum())   # what an unknown kept set may add
    assert lo - 2 * margin * total - extra <= u * total <= hi + 2 * margin * total + extra
    if not extra:
        assert abs(logprob - math.log(float(w[token]) / total)) <= 2 * margin
