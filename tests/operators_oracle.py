"""Plain implementations in 64 bits of the operators round the layer (8-bit products, the norms round a block, AdamW over many
tensors), on the CPU and from their formulas.  Test infrastructure only."""
import math

import torch

D = torch.float64


# ---- 8-bit floating point -----------------------------------------------------------------------------------------------------
def e4m3_values():
    """The non-negative values of e4m3 in ascending order, by code."""
    return torch.tensor([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)], dtype=D)


def to_codes(y):
    """|y| <= 448 to the nearest code (uint8), ties to the even one; NaN to 0x7f."""
    v = e4m3_values()
    a = y.abs().nan_to_num(0.0)
    hi = torch.searchsorted(v, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    down, up = a - v[lo], v[hi] - a
    c = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = torch.where(v[hi] == a, hi, c)
    c = c + 128 * ((y < 0) | ((y == 0) & torch.signbit(y))).long()
    return torch.where(torch.isnan(y), torch.full_like(c, 127), c).to(torch.uint8)


def from_codes(c):
    v = e4m3_values()[(c.long() & 127).clamp(max=126)]
    v = torch.where((c & 127) == 127, torch.full_like(v, math.nan), v)
    return torch.where(c >= 128, -v, v)


def exponent(largest):
    """Biased exponent of the least power of two 2^e with largest / 2^e <= 448."""
    if largest == 0:
        return 127
    e = math.frexp(largest / 448)  # f in [0.5, 1): largest / 448 <= 2^e unless f is 0.5
    return max(0, (e[1] - 1 if e[0] == 0.5 else e[1]) + 127)


def quant(x, block):
    """(codes [rows, cols padded] uint8, scales uint8) of x [rows, cols] in 64 bits."""
    rows, cols = x.shape
    cp, rp = -(-cols // 128) * 128, -(-rows // 128) * 128
    p = torch.zeros((rp, cp), dtype=D)
    p[:rows, :cols] = x
    p = torch.where(torch.isfinite(p), p, torch.full_like(p, math.nan))
    h = 128 if block else 1
    t = p.view(rp // h, h, cp // 128, 128)
    top = t.nan_to_num(0.0).abs().amax(dim=(1, 3))
    e = torch.tensor([[exponent(float(v)) for v in r] for r in top], dtype=torch.int64).view(top.shape)
    codes = to_codes(torch.ldexp(t, (127 - e)[:, None, :, None].to(D)).view(rp, cp))
    return codes[:rows], (e if block else e[:rows]).to(torch.uint8)


def value(codes, scales, cols, block):
    """The matrix [rows, cols] that codes and scales stand for."""
    e = scales.long()
    if block:
        e = e.repeat_interleave(128, 0)[:codes.shape[0]]
    return (from_codes(codes) * torch.pow(torch.tensor(2.0, dtype=D), e.to(D) - 127).repeat_interleave(128, 1))[:, :cols]


def gelu(y):
    return 0.5 * y * torch.special.erfc(-y * math.sqrt(0.5))


# ---- the norms round a block --------------------------------------------------------------------------------------------------
def statistics(v, rms, eps):
    mean = torch.zeros_like(v[:, :1]) if rms else v.mean(1, keepdim=True)
    return torch.cat([mean, 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)], 1)


def normed(v, stats, w, b):
    y = (v - stats[:, :1]) * stats[:, 1:]
    y = y if w is None else y * w
    return y if b is None else y + b


def rows_of(gate, T):
    return gate.repeat_interleave(T // gate.shape[0], 0)


def block_norm(x, f, post, pre, rms, eps, x_scale, gate, w_post, b_post, w_pre, b_pre, round_z=lambda z: z):
    """(Z, H, stats_post, stats_pre); all but x may be None."""
    sp = sq = h = None
    n = f
    if post:
        sp = statistics(f, rms, eps)
        n = normed(f, sp, w_post, b_post)
    if gate is not None:
        n = n * rows_of(gate, x.shape[0])
    z = x_scale * x if n is None else x_scale * x + n
    if pre:
        r = round_z(z)
        sq = statistics(r, rms, eps)
        h = normed(r, sq, w_pre, b_pre)
    return z, h, sp, sq


def norm_gradient(d, v, stats, w, rms):
    hat = (v - stats[:, :1]) * stats[:, 1:]
    g = d if w is None else d * w
    dv = g - hat * (g * hat).mean(1, keepdim=True) - (0 if rms else g.mean(1, keepdim=True))
    return dv * stats[:, 1:], (d * hat).sum(0), d.sum(0)


def block_norm_backward(dz, dh, z, f, post, pre, rms, x_scale, gate, w_post, b_post, w_pre, stats_post, stats_pre):
    out = {}
    d = torch.zeros_like(dh) if dz is None else dz
    if pre:
        g, out["dw_pre"], out["db_pre"] = norm_gradient(dh, z, stats_pre, w_pre, rms)
        d = d + g
    out["dx"] = x_scale * d
    n, df = f, d
    if post:
        n = normed(f, stats_post, w_post, b_post)
    if gate is not None:
        if n is not None:
            out["dgate"] = (d * n).view(gate.shape[0], -1, d.shape[1]).sum(1)
        df = d * rows_of(gate, d.shape[0])
    if post:
        df, out["dw_post"], out["db_post"] = norm_gradient(df, f, stats_post, w_post, rms)
    out["df"] = df
    return out


# ---- AdamW --------------------------------------------------------------------------------------------------------------------
def random_bits(n, t, seed, first=0):
    """(16 bits for m, 16 bits for r) of the elements first .. first + n - 1."""
    low = 0xFFFFFFFF
    x = (torch.arange(first, first + n) + ((seed * 0x9E3779B1 + t * 0x6A09E667) & low)) & low
    x = ((x ^ (x >> 16)) * 0xBB67AE85) & low
    x = ((x ^ (x >> 15)) * 0x3C6EF373) & low
    x = x ^ (x >> 16)
    return x & 0xFFFF, x >> 16


def stored(x, bits, up):
    """x (flat) as (values of its codes, scales, how far each was from the next rounding decision in steps)."""
    n = x.numel()
    blocks = torch.cat([x, torch.zeros(-n % 256, dtype=D)]).view(-1, 256)
    top = blocks.abs().amax(1)
    there = top >= 2.0 ** -100
    y = torch.where(there[:, None], blocks * 448 / torch.where(there, top, torch.ones_like(top))[:, None], torch.zeros_like(blocks)).view(-1)[:n]
    a = y.abs().clamp(max=448)
    unit = torch.pow(torch.tensor(2.0, dtype=D), (torch.frexp(a).exponent - 1).clamp(min=-6).to(D) - 3)
    place = a / unit + bits.to(D) / 65536
    q = torch.floor(place) * unit
    if up:
        q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
    return torch.where(y < 0, -q, q), torch.where(there, top / 448, torch.zeros_like(top)), (place - torch.round(place)).abs()


def adamw(w, g, m, v, lr, beta1, beta2, eps, decay, t, keep=None, alpha=None, lam=0.0, R=1, grad_scale=1.0):
    """(w, m, v) after the step, all [M, N] in 64 bits; v is the second moment."""
    g = g * grad_scale
    if alpha is not None:
        g = g + lam * alpha.repeat_interleave(R, 0) * w
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    w = w - lr * decay * w - lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
    if keep is not None:
        w = w * keep.repeat_interleave(R, 0)
    return w, m, v
