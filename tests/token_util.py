"""Plain 64-bit forms of the operators over a token cache, by positions, and the rounding bounds that their tests use."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # a rounding is off by at most this, relative to the value
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}   # ... or by this, below the type's normal range


def row_of(p, n_sink, ring):
    return p if p < n_sink else n_sink + (p - n_sink) % ring


def norm_rope(x, gain, pos, inv_freq, eps, interleaved):
    """x [T, heads, d] float64, pos [T]; returns (y, |pair|): the result and the size of what each of its values comes from."""
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    half = 0 if inv_freq is None else inv_freq.shape[0]
    size = y.abs()
    if half:
        ang = pos.double()[:, None] * inv_freq.double()
        cos, sin = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        a, b = y[..., i].clone(), y[..., j].clone()
        y[..., i], y[..., j] = a * cos - b * sin, b * cos + a * sin
        size[..., i] = size[..., j] = a.abs() + b.abs()
    return y, size


def attention(q, k, v, positions, at, n_sink, window, scale):
    """q [T, H, d] at positions `at`; k, v [Hkv, n, d] at `positions`, all float64.  Returns out, sum_p w |v| / sum_p w, and the largest
    bound on |error of a score| per unit roundoff: scale * sum |q_i k_i|."""
    T, H, d = q.shape
    G = H // k.shape[0]
    p, a = positions[None, :], at[:, None]
    seen = (p <= a) & ((p < n_sink) | (p > a - window))
    out, mag, worst = torch.empty_like(q), torch.empty_like(q), 0.0
    for h in range(k.shape[0]):
        for g in range(G):
            qq = q[:, h * G + g]
            # rows that a token does not see take no part, whatever they hold
            kk, vv = k[h], v[h]
            s = (qq @ torch.nan_to_num(kk, 0, 0, 0).T) * scale
            odd = ~torch.isfinite(kk).all(1)
            for c in torch.nonzero(odd).flatten().tolist():
                s[:, c] = (qq * kk[c]).sum(1) * scale
            worst = max(worst, float((qq.abs() @ torch.nan_to_num(kk, 0, 0, 0).abs().T).masked_fill(~seen, 0).max()) * scale)
            w = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
            o = torch.where(seen[..., None], w[..., None] * vv, torch.zeros((), dtype=q.dtype, device=q.device)).sum(1) if not torch.isfinite(vv).all() else w @ vv
            out[:, h * G + g] = o
            mag[:, h * G + g] = w @ torch.nan_to_num(vv, 0, 0, 0).abs()
    return out, mag, worst


def attention_bound(out, mag, worst, n_keys, d, dtype, chunk):
    """How far a kernel's output may be off: its own rounding (half a step); in calls of several tokens the rounding of every numerator
    (half a step of each weight; in fp16 also 2^-25 of the largest, for every key); and fp32 inside: a score is a sum of d products
    (d + 8 roundings of 2^-23, the matrix unit truncates), the exponent's argument another two, exp2 2^-22, the two sums n_keys roundings of 2^-24 and 2^-23."""
    score = worst * (d + 10) * 2.0 ** -23
    inner = 2 * score + 2.0 ** -21 + n_keys * 2.0 ** -22
    bound = HALF[dtype] * out.abs() * (1 + inner) + inner * mag + TINY[dtype]
    if not chunk:      # (the numerators as two halves: what the second one's rounding leaves)
        return bound + HALF[dtype] ** 2 * mag + (n_keys * 2.0 ** -25 * mag.amax(-1, keepdim=True) if dtype == torch.float16 else 0)
    return bound + HALF[dtype] * mag + (n_keys * 2.0 ** -25 * mag.amax(-1, keepdim=True) if dtype == torch.float16 else 0)
