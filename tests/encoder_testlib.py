"""64-bit forms of attention over encoder states and over the paged 8-bit cache, with bounds for the kernels' roundings."""
import math

import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def attention(q, k, v, sees, scale):
    """q [n, H, d], k, v [m, G, d] (64 bits), row i sees the first sees[i] keys.  Returns (O, sum_j a_j |V_j|, sum_j |V_j|)."""
    n, H, d = q.shape
    o, spread, plain = (torch.zeros(n, H, d, dtype=torch.float64) for _ in range(3))
    for h in range(H):
        g = h // (H // k.shape[1])
        for i in range(n):
            m = int(sees[i])
            if m <= 0:
                continue
            a = torch.softmax(k[:m, g] @ q[i, h] * scale, 0)
            o[i, h], spread[i, h], plain[i, h] = a @ v[:m, g], a @ v[:m, g].abs(), v[:m, g].abs().sum(0)
    return o, spread, plain


def bound(o, spread, plain, q, k, scale, out_type, weight_type):
    """How far a kernel's O may be off: the output's rounding; each weight's rounding to `weight_type` for the product; the weight's
    error in 32 bits, which is that of its exponent: a dot product of d terms (d roundings of at most 2^-24 of the sum of its
    terms' sizes, twice that for the accumulator's order and the scale), an exponential good to 2^-21, sums over the keys (a running sum of
    up to 2^14 terms in 32 bits or more: 2^-20 at the sizes here); weights below the smallest normal fp16 are off by
    at most 2^-25 of the largest."""
    d = q.shape[-1]
    logit = (q.abs().amax() * k.abs().amax() * d * abs(scale)).item() if k.numel() else 0.0
    fp32 = 2 * math.log2(math.e) * logit * (d + 4) * 2.0 ** -24 + 2.0 ** -20
    tiny = 2.0 ** -25 if weight_type == torch.float16 else 0.0
    return HALF_STEP[out_type] * (o.abs() + HALF_STEP[weight_type] * spread) + (HALF_STEP[weight_type] + fp32) * spread + tiny * plain + 2.0 ** -24


def check(got, ref, limit):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    off = (got - ref).abs()
    worst = (off - limit).argmax()
    assert (off <= limit).all(), f"off by {off.flatten()[worst]:.3e}, allowed {limit.flatten()[worst]:.3e}"
