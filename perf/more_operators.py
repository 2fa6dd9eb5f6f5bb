"""Group normalisation of channels-last maps, as values and as a layer's codes, and products of few rows with 4-bit weights.

What a UNet's residual block has around its quantized convolutions, each as a user's program calls it (`own`) and in its
plain form:

  norm    group norm with an optional addend per image and channel (the time embedding) and an optional SiLU, 16 bits in
          and out;
  codes   the same, straight into the codes that the next quantized layer reads: the channels permuted into its groups,
          each padded, quantized with the layer's table;
  few     products of few 16-bit rows with 4-bit weights that share a scale in groups of input channels: time embeddings
          and single tokens.

A code is the whole number that 64-bit arithmetic gives from the 16-bit inputs, so the plain form of `codes` computes in
64 bits.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
_SILU_LOW = -0.2784645  # the smallest value of y * sigmoid(y)


# ------------------------------------------------------------------------------------------ cases
def _norm(name, batch, pixels, c, groups, dtype, silu, add, wide, eps=1e-5):
    """wide: the rows are a slice of rows that many channels longer (the buffer of a skip connection)."""
    return dict(name=name, kind="norm", batch=batch, pixels=pixels, c=c, groups=groups, dtype=dtype, silu=silu, add=add, wide=wide, eps=eps)


def _codes(name, batch, pixels, c, groups, dtype, silu, add, bits, n_ranges, row_ranges, eps=1e-5):
    """n_ranges channel groups of the next layer (row_ranges 2: the outlier pixels have ranges of their own); codes of up to
    7 bits are stored less their zero-point, as the convolutions read them."""
    return dict(name=name, kind="codes", batch=batch, pixels=pixels, c=c, groups=groups, dtype=dtype, silu=silu, add=add, bits=bits,
                n_ranges=n_ranges, row_ranges=row_ranges, eps=eps)


def _few(name, rows, k, n, group, dtype, silu, bias):
    return dict(name=name, kind="few", rows=rows, k=k, n=n, group=group, dtype=dtype, silu=silu, bias=bias)


def listed():
    return [
        # First norm of the 8x8 middle block at batch 2 (classifier-free guidance): the smallest map.
        _norm("norm_2x64x1280_silu_f16", 2, 64, 1280, 32, "f16", True, False, 0),
        # Second norm of the 64x64 level's residual block, the time embedding added on the way in.
        _norm("norm_2x4096x320_silu_add_f16", 2, 4096, 320, 32, "f16", True, True, 0),
        # In front of a transformer block of the 32x32 level at batch 8: no activation; rows cut out of a wider buffer.
        _norm("norm_8x1024x640_wide_bf16", 8, 1024, 640, 32, "bf16", False, False, 320, 1e-6),
        # Decoder of the latents at 512x512 pixels, 128 channels: the largest map.
        _norm("norm_1x262144x128_silu_f16", 1, 262144, 128, 32, "f16", True, False, 0, 1e-6),
        # 8x8 level into the codes of a 6-bit convolution, 16 ranges: where latency counts.
        _codes("codes_2x64x1280_silu_6bit", 2, 64, 1280, 32, "f16", True, True, 6, 16, 1),
        # 64x64 level into the 6-bit convolution of 320 channels.
        _codes("codes_2x4096x320_silu_add_6bit", 2, 4096, 320, 32, "f16", True, True, 6, 16, 1),
        # In front of the first projection of a transformer block, 8 bits, pixel and channel ranges.
        _codes("codes_8x1024x640_8bit_bf16", 8, 1024, 640, 32, "bf16", False, False, 8, 8, 2, 1e-6),
        # 64x64 level behind a skip connection at batch 8: 960 channels, groups of 30, the largest map of the UNet.
        _codes("codes_8x4096x960_silu_6bit", 8, 4096, 960, 32, "f16", True, False, 6, 16, 1),
        # Time embedding of two images onto the 320 channels of a residual block: the smallest product.
        _few("few_2x1280_320_silu_f16", 2, 1280, 320, 64, "f16", True, True),
        # One token through a projection.
        _few("few_1x4096_4096_bf16", 1, 4096, 4096, 128, "bf16", False, False),
        # Seven tokens, odd sizes: a reduction that no group size divides and an odd number of outputs.
        _few("few_7x5000_10007_f16", 7, 5000, 10007, 32, "f16", False, True),
        # 32 tokens through the widest layer: the largest weight.
        _few("few_32x8192_28672_bf16", 32, 8192, 28672, 128, "bf16", False, False),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    """One more case: half the widths are the UNet's own channel counts, the others any multiple of 8; maps of any number of
    pixels, any number of groups that divides the channels."""
    kind = rng.choice(["norm"] * 4 + ["codes"] * 4 + ["few"] * 4)
    dtype = rng.choice(["f16", "bf16"])
    if kind == "few":
        while True:
            k = rng.choice([320, 640, 768, 1280, 2048, 4096, 5120, 8192]) if rng.random() < 0.4 else _log_int(rng, 32, 8192, 8)
            n = rng.choice([320, 640, 1280, 2560, 4096, 10240]) if rng.random() < 0.4 else _log_int(rng, 8, 28672)
            rows = 1 if rng.random() < 0.25 else _log_int(rng, 1, 32)
            if k * n <= 8192 * 28672:
                c = _few("", rows, k, n, rng.choice([32, 64, 128]), dtype, rng.random() < 0.4, rng.random() < 0.5)
                del c["name"]
                return c
    top = 262144 * 128 if kind == "norm" else 8 * 4096 * 960
    while True:
        ch = rng.choice([320, 640, 960, 1280, 1920, 2560, 128, 256, 512]) if rng.random() < 0.5 else _log_int(rng, 8, 2560, 8)
        few = [g for g in range(1, ch + 1) if ch % g == 0]
        groups = 32 if ch % 32 == 0 and rng.random() < 0.7 else rng.choice(few)
        pixels = rng.choice([64, 256, 1024, 4096, 16384]) if rng.random() < 0.4 else _log_int(rng, 1, 262144 if kind == "norm" else 16384)
        batch = _log_int(rng, 1, 8)
        if batch * pixels * ch <= top and pixels * ch // groups > 1:
            break
    silu, add, eps = rng.random() < 0.6, rng.random() < 0.5, rng.choice([1e-5, 1e-6])
    if kind == "norm":
        c = _norm("", batch, pixels, ch, groups, dtype, silu, add, 8 * rng.randint(1, 80) if rng.random() < 0.3 and pixels < 32768 else 0, eps)
    else:
        c = _codes("", batch, pixels, ch, groups, dtype, silu, add, rng.choice([8, 6, 6, 4]), min(ch, rng.choice([1, 4, 8, 16])), rng.choice([1, 1, 2]), eps)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _ranges(c, gain, spread, gamma, beta, row_gain, table):
    """The next layer's groups and table, as a calibration on such maps would leave them: channels sorted by their range and cut
    into n_ranges groups of nearly the same size, a scale and a zero-point for each pixel group and channel group."""
    C, G, R, bits = c["c"], c["n_ranges"], c["row_ranges"], c["bits"]
    std = np.repeat(spread, C // c["groups"])
    wide = np.abs(gamma) * gain / std
    lo, hi = beta - 4 * wide, beta + 4 * wide
    if c["silu"]:
        lo, hi = np.maximum(lo, _SILU_LOW), np.maximum(hi, 0.1)
    order = np.argsort(hi - lo, kind="stable")
    col = np.empty(C, dtype=np.int32)
    for g, part in enumerate(np.array_split(order, G)):
        col[part] = g
    row = (row_gain > 1).astype(np.int32) if R == 2 else np.zeros(c["pixels"], dtype=np.int32)
    scale, zp = np.empty((1, R, G), dtype=np.float32), np.empty((1, R, G), dtype=np.int32)
    for r in range(R):
        more = 4.0 if r else 1.0
        for g in range(G):
            a, b = lo[col == g].min() * (1.0 if c["silu"] else more), hi[col == g].max() * more
            scale[0, r, g] = (b - a) / 2 ** bits
            zp[0, r, g] = int(np.clip(np.rint(-a / scale[0, r, g]), 0, 2 ** bits - 1))
    perm = []
    for g in range(G):
        mine = np.nonzero(col == g)[0].tolist()
        perm += mine + [-1] * (-(-(len(mine) + 8) // 32) * 32 - len(mine))
    inv = (np.float32(1.0) / scale).astype(np.float32)
    of = np.repeat(np.arange(G), [-(-(int((col == g).sum()) + 8) // 32) * 32 for g in range(G)])
    table.update(col=col, row=row, scale=scale, zp=zp, bits=bits, centred=bits <= 7, perm=torch.tensor(perm, device="cuda"), of=torch.tensor(of, device="cuda"),
                 inv=torch.from_numpy(inv[0]).cuda(), z=torch.from_numpy(zp[0]).cuda(), rows=torch.from_numpy(row).cuda().long())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    order = np.random.RandomState(int(seed) % (2 ** 32))
    kind, t = case["kind"], _TYPES[case["dtype"]]
    s = dict(kind=kind, silu=case["silu"])
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    if kind == "few":
        m, k, n, group = (case[x] for x in ("rows", "k", "n", "group"))
        s.update(x=randn(m, k).to(t), codes=torch.randint(-7, 8, (n, k), generator=gen, device="cuda", dtype=torch.int8), group=group,
                 scales=randn(n, -(-k // group)).mul_(0.2).exp_().mul_(0.25 / math.sqrt(k)).half(), bias=randn(n).mul_(0.1).to(t) if case["bias"] else None)
        if own:
            from paper_2501_04304_b200 import binding as b
            s["weight"] = b.few_weight_from_codes(s["codes"], s["scales"], group)
        return s
    B, P, C, G = (case[x] for x in ("batch", "pixels", "c", "groups"))
    # normal maps with a few wide channels and, where the map is large enough, a few wide pixels
    gain, row_gain = np.ones(C, dtype=np.float32), np.ones(P, dtype=np.float32)
    gain[order.permutation(C)[:-(-C // 100)]] = 8.0
    row_gain[order.permutation(P)[:P // 200]] = 4.0
    x = torch.empty(B, P, C + case.get("wide", 0), dtype=t, device="cuda")
    s["x"] = x[:, :, :C]
    for b in range(B):
        s["x"][b] = randn(P, C).mul_(torch.from_numpy(gain).cuda()).mul_(torch.from_numpy(row_gain).cuda()[:, None]).add_(0.3)
    gamma, beta = (1 + 0.1 * order.randn(C)).astype(np.float32), (0.1 * order.randn(C)).astype(np.float32)
    s.update(gamma=torch.from_numpy(gamma).cuda(), beta=torch.from_numpy(beta).cuda(), groups=G, eps=case["eps"],
             add=randn(B, C).mul_(0.5).to(t) if case["add"] else None)
    if kind == "codes":
        _ranges(case, gain, np.sqrt((gain.reshape(G, -1) ** 2).mean(1)), gamma, beta, row_gain, s)
        if own:
            from paper_2501_04304_b200 import binding as b
            s["handle"] = b.groups_from_host(C, P, case["bits"], s["col"], s["row"], s["scale"], s["zp"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_values(s, bits):
    """The normalised map in 32 or 64 bits."""
    x = s["x"].to(bits)
    B, P, C = x.shape
    if s["add"] is not None:
        x = x + s["add"].to(bits)[:, None, :]
    x = x.view(B, P, s["groups"], C // s["groups"])
    x = x - x.mean((1, 3), keepdim=True)
    var = (x * x).mean((1, 3), keepdim=True)
    y = (x / torch.sqrt(var + s["eps"])).view(B, P, C) * s["gamma"].to(bits) + s["beta"].to(bits)
    return y / (1 + torch.exp(-y)) if s["silu"] else y


def _plain_codes(s):
    """The permuted, padded codes: padding carries the zero-point."""
    v = _plain_values(s, torch.float64)
    B, P, C = v.shape
    perm, of, top = s["perm"], s["of"], 2 ** s["bits"] - 1
    inv, z = s["inv"].double()[s["rows"]][:, of], s["z"][s["rows"]][:, of]
    q = (torch.round(v[:, :, perm.clamp(min=0)] * inv) + z).clamp(0, top)
    q = torch.where(perm < 0, z.double().clamp(0, top), q)
    return ((q - z) if s["centred"] else q).to(torch.int64).to(torch.uint8).view(B * P, -1)


def _plain_few(s):
    x = s["x"].float()
    if s["silu"]:
        x = x / (1 + torch.exp(-x))
    n, k = s["codes"].shape
    w = s["codes"].float() * s["scales"].float().repeat_interleave(s["group"], 1)[:, :k]
    y = torch.matmul(x, w.T)
    return (y if s["bias"] is None else y + s["bias"].float()).to(s["x"].dtype)


def run(state):
    s = state
    if own:
        from paper_2501_04304_b200 import binding as b
        act = b.ACT_SILU if s["silu"] else b.ACT_NONE
        if s["kind"] == "norm":
            return b.group_norm(s["x"], s["groups"], s["gamma"], s["beta"], eps=s["eps"], act=act, add=s["add"])
        if s["kind"] == "codes":
            return b.group_norm_quantize(s["handle"], s["x"], s["groups"], s["gamma"], s["beta"], eps=s["eps"], act=act, add=s["add"],
                                         layout=b.CODES_S8_CENTRED if s["centred"] else b.CODES_U8)
        return b.linear_few(s["weight"], s["x"], bias=s["bias"], act=act)
    if s["kind"] == "norm":
        return _plain_values(s, torch.float32).to(s["x"].dtype)
    return _plain_codes(s) if s["kind"] == "codes" else _plain_few(s)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "few":
        m, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": n * k / 2 + 2 * n * -(-k // case["group"]) + 2 * m * (k + n), "flops": 2 * m * n * k}
    B, P, C = case["batch"], case["pixels"], case["c"]
    small = 8 * C + (2 * B * C if case["add"] else 0)
    if case["kind"] == "norm":
        return {"bytes": 4 * B * P * C + small, "flops": 10 * B * P * C}
    sizes = [len(p) for p in np.array_split(np.arange(C), case["n_ranges"])]
    return {"bytes": B * P * (2 * C + sum(-(-(n + 8) // 32) * 32 for n in sizes)) + small + 4 * C, "flops": 12 * B * P * C}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "few":
        x = s["x"].double()
        x = x * torch.sigmoid(x) if s["silu"] else x
        y = torch.zeros(x.shape[0], s["codes"].shape[0], dtype=torch.float64, device="cuda")
        for g in range(s["scales"].shape[1]):
            at = slice(g * s["group"], (g + 1) * s["group"])
            y += (x[:, at] @ s["codes"][:, at].double().T) * s["scales"][:, g].double()
        return y if s["bias"] is None else y + s["bias"].double()
    x, C = s["x"], case["c"]
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    step = C // s["groups"]
    for b in range(x.shape[0]):
        v = x[b].double() if s["add"] is None else x[b].double() + s["add"][b].double()
        per = v.T.reshape(s["groups"], -1)
        var, mean = torch.var_mean(per, 1, correction=0)
        v = (v - mean.repeat_interleave(step)) / (var + s["eps"]).sqrt().repeat_interleave(step)
        v = v * s["gamma"].double() + s["beta"].double()
        out[b] = v * torch.sigmoid(v) if s["silu"] else v
    if s["kind"] == "norm":
        return out
    codes, top = torch.zeros(x.shape[0] * x.shape[1], s["perm"].numel(), dtype=torch.int64, device="cuda"), 2 ** s["bits"] - 1
    rows = s["rows"].repeat(x.shape[0])
    for p, (c, g) in enumerate(zip(s["perm"].tolist(), s["of"].tolist())):
        z = s["z"][rows, g].long()
        q = z.clamp(0, top) if c < 0 else (torch.round(out[:, :, c].reshape(-1) * s["inv"][rows, g].double()).long() + z).clamp(0, top)
        codes[:, p] = q - z if s["centred"] else q
    return codes.to(torch.uint8)
