"""Attention in 64 bits on the GPU with a bound, element by element, for what the kernels round."""
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def attend(q, k, v, sees, scale, out, weight, v_scale=None):
    """q [n, H, d], k and v [m, G, d] in 64 bits on the GPU, row i sees the first sees[i] keys (a list or a number); v_scale [m, G] are
    the scales in v, whose kernels multiply codes.  Returns O and how far a result of type `out` may be off whose weights were
    rounded to `weight` for the product:

    * the output's half step;
    * each weight's: sum_j a_j |V_j|; fp16 weights below 2^-14 of the reference are off by up to 2^-25 of it, absolutely.  The
      reference is at most the largest a_j s_j, and what is rounded belongs to V_j / s_j;
    * each exponent's: d products and sums of 2^-24 of the terms' sizes each, twice for their order; scale and reference take four
      more roundings, of the largest score's size.  bf16 queries over codes go to fp16 after a power of two: 2^-25 of the row's largest
      feature each.  An exponent's error is a weight's relative one, in the sum of the weights too;
    * 2^-20 for exponentials and for sums, which are held in 32 bits."""
    n, H, d = q.shape
    m, G = k.shape[0], k.shape[1]
    o, limit = torch.zeros_like(q), torch.full_like(q, 2.0 ** -24)
    if not n or not m:
        return o, limit
    sees = torch.as_tensor(sees, device=q.device).expand(n)
    hidden = torch.arange(m, device=q.device)[None] >= sees[:, None]
    some = (sees > 0)[:, None]
    for h in range(H):
        g = h // (H // G)
        kk, vv = k[:, g], v[:, g]
        t = (q[:, h] @ kk.T * scale).masked_fill(hidden, float("-inf"))
        a = torch.where(some, torch.softmax(t, -1), 0.0)
        size = q[:, h].abs() @ kk.abs().T * abs(scale)
        if v_scale is not None and out == torch.bfloat16:
            size = size + q[:, h].abs().amax(1, keepdim=True) * kk.abs().sum(1)[None] * abs(scale) / 4
        top = torch.where(hidden, 0.0, t.abs()).amax(1, keepdim=True)
        rel = a * (2.0 ** -24 * ((2 * d + 8) * size + 4 * top) + 2.0 ** -20)
        r = a @ vv
        off = (a * HALF_STEP[weight] + rel) @ vv.abs() + rel.sum(1, keepdim=True) * r.abs()
        if weight == torch.float16:
            s = torch.ones(m, dtype=q.dtype, device=q.device) if v_scale is None else v_scale[:, g]
            w = a * s
            most = w.amax(1, keepdim=True)
            small = torch.where(s > 0, 2.0 ** -25 / s, 0.0)[:, None] * vv.abs()
            off = off + most * (((w < 2.0 ** -13 * most) & ~hidden).to(q.dtype) @ small)
        o[:, h] = r
        limit[:, h] += HALF_STEP[out] * (r.abs() + off) + off
    return o, limit


def check(got, want):
    ref, limit = want
    got = got.double()
    assert got.shape == ref.shape
    if not got.numel():
        return
    assert torch.isfinite(got).all()
    over = (got - ref).abs() - limit
    worst = over.argmax()
    assert over.flatten()[worst] <= 0, f"off by {(got - ref).abs().flatten()[worst]:.3e}, allowed {limit.flatten()[worst]:.3e}"
