"""Plain 64-bit forms of the 8-bit decoder operators (torch on the CPU), written from their
definitions; the tests compare the kernels with them.

Half steps, as multiples of a value: bf16 2^-8, fp32 2^-24."""
from __future__ import annotations

import math

import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def normal(seed, *shape, dtype="bf16", std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std).to(TYPES[dtype])


def strided(t, pad, device="cuda"):
    """The same rows on the device with `pad` elements of NaN (of -99 in int8) behind each."""
    fill = -99 if t.dtype == torch.int8 else float("nan")
    whole = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=device)
    whole[:, :t.shape[1]] = t.to(device)
    return whole[:, :t.shape[1]]


def rmsnorm(x, gamma, eps, residual=None):
    """(h, y) in float64."""
    h = x.double() + (0.0 if residual is None else residual.double())
    return h, gamma.double() * h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)


def eight(y):
    """(q, scale) of float64 rows, and how far y / scale is from a border between two steps."""
    scale = y.abs().amax(1) / 127.0
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    z = torch.where(scale[:, None] > 0, y / scale[:, None], 0.0)
    return torch.round(z), scale, (z - torch.floor(z) - 0.5).abs()


def gelu(y, act):
    if act == 1:
        return 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    if act == 2:
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def rotary(x, pos, freq, amplitude, heads, head_dim, half, inverse=False):
    """Complex multiplication of each pair, float64; pos [T], freq [rot_dim / 2] float64."""
    T, P = x.shape[0], freq.numel()
    y = x.double().reshape(T, heads, head_dim).clone()
    a, b = (y[..., :P], y[..., P:2 * P]) if half else (y[..., 0:2 * P:2], y[..., 1:2 * P:2])
    angle = pos.double()[:, None] * freq
    z = torch.complex(a, b) * torch.polar(torch.full_like(angle, amplitude), -angle if inverse else angle)[:, None]
    if half:
        y[..., :P], y[..., P:2 * P] = z.real, z.imag
    else:
        y[..., 0:2 * P:2], y[..., 1:2 * P:2] = z.real, z.imag
    return y.reshape(T, heads * head_dim)


def window_attention(L, heads, kv_heads, q, k, v, first, kv_len, window, sinks, scale):
    """Dense masked attention per sequence and head in float64.  Returns (out, magnitude, bound): magnitude is
    sum_j p_j |v_j| of each output, bound the largest sum_c |q_c k_c| |scale| over a row's visible keys."""
    T, G = q.shape[0], heads // kv_heads
    q, k, v = q.double(), k.double(), v.double()
    out, mag = torch.zeros(T, heads * 64, dtype=torch.float64), torch.zeros(T, heads * 64, dtype=torch.float64)
    bound, count = torch.zeros(T, heads, dtype=torch.float64), torch.zeros(T, heads, dtype=torch.float64)
    t0 = 0
    for b, n in enumerate(L):
        m = kv_len[b]
        if n and m:
            p = torch.arange(m - n, m)[:, None]
            j = torch.arange(m)[None]
            seen = (j <= p) & ((j > p - window) | (j < sinks))
            for h in range(heads):
                qq = q[t0:t0 + n, 64 * h:64 * h + 64]
                g = 64 * (h // G)
                kk, vv = k[first[b]:first[b] + m, g:g + 64], v[first[b]:first[b] + m, g:g + 64]
                s = (qq @ kk.t() * scale).masked_fill(~seen, -math.inf)
                e = torch.exp(s - s.amax(1, keepdim=True).clamp_min(-1e300))
                e = e / e.sum(1, keepdim=True).clamp_min(1e-300)
                out[t0:t0 + n, 64 * h:64 * h + 64] = e @ vv
                mag[t0:t0 + n, 64 * h:64 * h + 64] = e @ vv.abs()
                a = (qq.abs() @ kk.abs().t() * abs(scale)).masked_fill(~seen, 0.0)
                bound[t0:t0 + n, h] = a.amax(1)
                count[t0:t0 + n, h] = seen.sum(1)
        t0 += n
    return out, mag, bound, count


def window_tolerance(dtype, ref, mag, bound, count):
    """Half steps: a score is a sum of 64 products (64 roundings of at most `bound`), scaled (3); an
    exponential then errs by that and 2; sums over the keys by one per key, in numerator and denominator, each
    with a few of the rescalings; in bf16 every exponential of the product is rounded (2^-8), and the result is."""
    each = 2 * 2.0 ** -24 * (67 * bound + count + 8)
    each = each.repeat_interleave(64, dim=1)
    return mag * (each + (HALF["bf16"] if dtype == "bf16" else 0.0)) + HALF[dtype] * ref.abs()
