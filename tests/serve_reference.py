"""Plain forms in 64 bits (torch, CPU) of the serving-layer operators, and bounds on how far fp32 kernels may be from them."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4}
E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()


def e4m3_round(x):
    """Nearest E4M3 value of doubles with |x| <= 448, ties to the even code, computed from the format."""
    a = x.abs()
    _, e = torch.frexp(a)                                  # a = m * 2^e, m in [1/2, 1)
    step = torch.ldexp(torch.ones_like(a), torch.clamp(e - 1, min=-6) - 3)
    return torch.copysign(torch.round(a / step) * step, x)  # torch.round: ties to even


def quantize(x, block_rows):
    """(codes as doubles, fp32 scales [column block, row block]) by the stated fp32 operations."""
    rows, cols = x.shape
    x = x.float()
    codes = torch.zeros(rows, cols, dtype=torch.float64)
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    scales = torch.zeros(nc, nr, dtype=torch.float32)
    for j in range(nc):
        for i in range(nr):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(j * 128, (j + 1) * 128))
            b = x[at]
            a = torch.clamp_min(b.abs().max(), 2.0 ** -100)
            factor = torch.tensor(448.0) / a
            scales[j, i] = a / torch.tensor(448.0)
            codes[at] = e4m3_round((b * factor).double())
    return codes, scales


def dequantize(codes, scales, block_rows):
    rows, cols = codes.shape
    r = torch.arange(rows) // block_rows
    c = torch.arange(cols) // 128
    return codes.double() * scales.double()[c][:, r].t()


def gelu(y):
    return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))


def linear(x, w, bias, act):
    """(result, sum of the magnitudes of its terms, sum over sixteens of columns of 16 times the largest term)"""
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    peak = torch.zeros_like(y)
    for k in range(0, x.shape[1], 16):
        top = torch.zeros_like(y)
        for i in range(k, min(k + 16, x.shape[1])):
            top = torch.maximum(top, x[:, i:i + 1].abs() * w[:, i].abs())
        peak += 16 * top
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return (gelu(y) if act else y), size, peak


def linear_bound(y, size, peak, K, dtype):
    # K products and their sums, each off by at most 2^-23 of a partial sum (truncation allowed) that never exceeds `size`;
    # 16-bit results: a product loses less than 2^-13 of the largest of its sixteen; GELU's slope is below 1.13, its own
    # evaluation within 2^-21 of |y|
    dropped = 0.0 if dtype == torch.float32 else 2.0 ** -13
    return 1.13 * ((K + 8) * 2.0 ** -23 * size + dropped * peak) + 2.0 ** -21 * size + HALF[dtype] * y.abs() + tiny(dtype)


def tiny(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 0.0     # half a step of the smallest numbers


def norm_rotate(x, kind, gamma, beta, eps, cos, sin, interleaved):
    """x [tokens, heads, dim] in doubles -> (result, magnitude that rounding errors scale with)."""
    size = x.abs()
    if kind != "none":
        mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
        r = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
        size = (x.abs() + mean.abs()) * r * gamma.double().abs()
        x = (x - mean) * r * gamma.double()
        if beta is not None:
            x, size = x + beta.double(), size + beta.double().abs()
    if cos is not None:
        half = cos.shape[-1]
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos.double()[:, None], sin.double()[:, None]
        out, big = x.clone(), size.clone()
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        big[..., a] = big[..., b] = size[..., a] + size[..., b]
        x, size = out, big
    return x, size


def attention(q, keys, values, place, scale, causal, window, kv_len, visible=None):
    """One sequence: q [n, Hq, D], keys / values [kv, Hk, D] doubles, place [n] -> out, lse, sum p|v|, largest sum |q k|,
    sum |v| over what is seen."""
    n, Hq, D = q.shape
    Hk = keys.shape[1]
    j = torch.arange(keys.shape[0])
    seen = (j[None] < kv_len).expand(n, -1)
    if causal:
        seen = seen & (j[None] <= place[:, None])
    if window:
        seen = seen & (j[None] > place[:, None] - window)
    if visible is not None:
        seen = seen & visible[None]
    keys = torch.where(seen.any(0)[:, None, None], keys, torch.zeros_like(keys))
    values = torch.where(seen.any(0)[:, None, None], values, torch.zeros_like(values))
    out, lse = torch.zeros_like(q), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    mass, reach, total_v = torch.zeros_like(q), torch.zeros(n, Hq, dtype=torch.float64), torch.zeros_like(q)
    for h in range(Hq):
        k, v = keys[:, h * Hk // Hq], values[:, h * Hk // Hq]
        z = (q[:, h] @ k.t()) * scale
        z = torch.where(seen, z, torch.full_like(z, -math.inf))
        some = seen.any(1)
        if not bool(some.any()):
            continue
        p = torch.softmax(z[some], dim=1)
        fine = torch.isfinite(v)
        out[some, h] = p @ torch.where(fine, v, torch.zeros_like(v))
        for key in torch.nonzero(~fine.all(1)).flatten().tolist():        # what is not finite reaches the rows that see its key alone
            rows = torch.nonzero(some & seen[:, key]).flatten()
            out[rows, h] = out[rows, h] + torch.where(fine[key], torch.zeros_like(v[key]), v[key])
        v = torch.where(fine, v, torch.zeros_like(v))
        lse[some, h] = torch.logsumexp(z[some], dim=1)
        mass[some, h] = p @ v.abs()
        reach[some, h] = torch.where(seen, (q[:, h].abs() @ k.abs().t()) * abs(scale), torch.zeros_like(z))[some].max(1).values
        total_v[some, h] = seen[some].double() @ v.abs()
    return out, lse, mass, reach, total_v


def attention_bounds(out, lse, mass, reach, total_v, dtype, D, keys):
    """A score is off by at most d = (D + 4) 2^-23 reach (relative error e^d - 1 of a probability, twice with the sum's);
    a probability enters rounded to the output's type, and sums over the keys in fp32 lose 2^-23 each at most."""
    d = ((D + 4) * 2.0 ** -23 * reach).unsqueeze(-1)
    share = 2 * torch.expm1(d) + HALF[dtype] + (keys + 32) * 2.0 ** -23 + 2.0 ** -20
    bound = share * mass + HALF[dtype] * out.abs() + tiny(dtype) * (1 + total_v)
    return bound, d.squeeze(-1) + (keys + 32) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).abs()
