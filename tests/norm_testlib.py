"""64-bit forms of the group norm, of its codes and of the products of few rows, with bounds for the kernels' roundings."""
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def norm(x, n_groups, gamma, beta, eps, silu, add=None):
    """x [B, P, C] of any type.  Returns (v, y, c) in 64 bits on the CPU: the result, what the activation is applied to, and the part of y
    that is the same for a whole channel (with the addend inside the sums it is beta - mean * factor)."""
    x = x.detach().cpu().double()
    B, P, C = x.shape
    e = torch.zeros(B, C, dtype=torch.float64) if add is None else add.detach().cpu().double()
    u = (x + e[:, None]).reshape(B, P, n_groups, C // n_groups)
    mean = u.mean((1, 3), keepdim=True)
    var = ((u - mean) ** 2).mean((1, 3), keepdim=True)
    factor = (1 / torch.sqrt(var + eps)).expand(B, 1, n_groups, C // n_groups).reshape(B, 1, C)
    mean = mean.expand(B, 1, n_groups, C // n_groups).reshape(B, 1, C)
    g = torch.ones(C, dtype=torch.float64) if gamma is None else gamma.detach().cpu().double()
    b = torch.zeros(C, dtype=torch.float64) if beta is None else beta.detach().cpu().double()
    y = (u.reshape(B, P, C) - mean) * factor * g + b
    const = (e[:, None] - mean) * factor * g + b
    return (y * torch.sigmoid(y) if silu else y), y, const.expand(B, P, C)


def norm_bound(v, y, const, dtype):
    """How far a value may be off: its own rounding; 32-bit arithmetic behind the statistics, which is one fused multiply-add of a rounded
    factor and addend (2^-23 of |y| + |addend|) and the activation (an exponential and a reciprocal of two units in the last place, its
    slope at most 1.1: 2.2 * 2^-22 |y| + 0.6 * 2^-22 |addend|); statistics good to 2^-21 of the deviation (sums in 32 bits of at most a few
    hundred terms each, joined in 64): 2^-21 (|y - beta| + 1), where |y - beta| <= |y| + |beta| is counted with the addend."""
    return HALF_STEP[dtype] * v.abs() + 2.0 ** -20 * (y.abs() + const.abs() + 1) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def check(got, ref, limit):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape
    assert torch.isfinite(got).all()
    off = (got - ref).abs()
    worst = (off - limit).argmax()
    assert (off <= limit).all(), f"off by {off.flatten()[worst]:.3e}, allowed {limit.flatten()[worst]:.3e}"


def codes(v, ex, bits, timestep, centred):
    """Codes [B * P, K_pad] (as bytes) of values v [B, P, C] (64 bits) with an exported grouping."""
    B, P, C = v.shape
    perm, col = torch.from_numpy(ex["perm"]).long(), torch.from_numpy(ex["col_group"]).long()
    row = torch.from_numpy(ex["row_group"]).long()
    row = row[torch.arange(B * P) % row.numel()]
    off = torch.from_numpy(ex["group_off"]).long()
    of = torch.searchsorted(off, torch.arange(perm.numel()), right=True) - 1
    of = torch.where(perm >= 0, col[perm.clamp(min=0)], of)
    inv = (1.0 / torch.from_numpy(ex["scale"][timestep])).double()[row][:, of]  # the table's numbers are fp32
    z = torch.from_numpy(ex["zp"][timestep]).double()[row][:, of]
    top = 2 ** bits - 1
    q = (torch.round(v.reshape(B * P, C)[:, perm.clamp(min=0)] * inv) + z).nan_to_num(nan=0.0, posinf=1e30, neginf=-1e30).clamp(0, top)
    q = torch.where(perm < 0, z.clamp(0, top), q)
    return ((q - z) if centred else q).long() & 255


def few(x, wq, scales, group, silu, bias):
    """(Y, sum of the sizes of its terms) in 64 bits; x [M, K]."""
    x = x.detach().cpu().double()
    if silu:
        x = x * torch.sigmoid(x)
    w = wq.detach().cpu().double() * scales.detach().cpu().double().repeat_interleave(group, 1)[:, :wq.shape[1]]
    b = torch.zeros(w.shape[0], dtype=torch.float64) if bias is None else bias.detach().cpu().double()
    return x @ w.T + b, x.abs() @ w.abs().T + b.abs()


def few_bound(y, size, dtype, silu, k):
    """The output's rounding; sums in 32 bits: the products are exact, each is part of at most k / 16 + 30 additions of its chain, of a group's
    scale and of the warps' parts, whose rounding (or, inside the matrix instruction, cutting) is at most 2^-23 of the sizes' sum; a SiLU's
    error in 32 bits (2^-20 of it) and the rounding of what its first 16-bit part leaves (half a step of half a step, and in fp16 2^-25 where
    that part is below the smallest normal number, which 2^-20 of the sizes' sum covers where the rows are about 1)."""
    t = HALF_STEP[dtype] * y.abs() + (k / 16 + 30) * 2.0 ** -23 * size + 2.0 ** -25
    return t + (HALF_STEP[dtype] ** 2 + 2.0 ** -19) * size * (1 if silu else 0)
