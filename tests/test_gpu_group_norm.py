"""Group norm of channels-last maps, as values and as codes, against 64 bits."""
import numpy as np
import pytest
import torch

import norm_testlib as nl
from dgq_testlib import gpu
from paper_2501_04304_b200 import binding as b

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def make(seed, B, P, C, dtype, add=True, shift=0.3):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, P, C)).astype(np.float32) + np.float32(shift)
    x[:, :, rng.permutation(C)[:max(1, C // 50)]] *= 8
    t = torch.from_numpy(x).to(dtype).cuda()
    gamma = torch.from_numpy((1 + 0.2 * rng.standard_normal(C)).astype(np.float32)).cuda()
    beta = torch.from_numpy((0.2 * rng.standard_normal(C)).astype(np.float32)).cuda()
    e = torch.from_numpy(rng.standard_normal((B, C)).astype(np.float32)).to(dtype).cuda() if add else None
    return t, gamma, beta, e


def against(x, groups, gamma, beta, eps, silu, e, y):
    v, u, c = nl.norm(x, groups, gamma, beta, eps, silu, e)
    nl.check(y, v, nl.norm_bound(v, u, c, x.dtype))


# B, P, C, groups: one pixel, one channel a group, one group, groups of 10, 30, 40 and 60 channels, groups that start inside eight
# channels, the widest, many images, maps that one block holds, that several share and that none does
SHAPES = [(1, 1, 8, 1), (2, 1, 64, 8), (3, 2, 8, 8), (1, 37, 24, 8), (2, 64, 1280, 32), (1, 4096, 320, 32), (2, 333, 320, 32), (1, 1000, 960, 32),
          (2, 77, 1920, 32), (1, 257, 72, 24), (1, 129, 40, 40), (2, 50, 4096, 1), (1, 30, 4096, 4096), (1, 300, 2568, 321), (9, 100, 128, 32), (70, 5, 56, 7),
          (1, 70001, 8, 2), (1, 90000, 128, 32), (1, 5000, 640, 1), (40, 260, 64, 4), (2, 1030, 1000, 5), (1, 16, 3000, 3000)]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,P,C,groups", SHAPES)
def test_values(B, P, C, groups, dtype):
    gpu()
    if P * C // groups == 1:
        pytest.skip("a group of one value")
    x, gamma, beta, e = make(B + P + C, B, P, C, dtype, add=P % 2 == 0)
    silu = C % 3 != 0
    y = b.group_norm(x, groups, gamma, beta, eps=1e-5, act=b.ACT_SILU if silu else b.ACT_NONE, add=e)
    assert y.dtype == dtype and y.shape == x.shape
    against(x, groups, gamma, beta, 1e-5, silu, e, y)


def test_one_value_a_group():
    """Its variance is 0: the result is beta."""
    gpu()
    x, gamma, beta, _ = make(5, 2, 1, 16, F16, add=False)
    y = b.group_norm(x, 16, gamma, beta)
    assert torch.equal(y, beta.half().expand(2, 1, 16))


@pytest.mark.parametrize("P", [64, 5000, 40000, 150000])
def test_defaults_and_constant_maps(P):
    gpu()
    x = torch.full((2, P, 64), 3.25, dtype=F16, device="cuda")
    assert (b.group_norm(x, 4).abs() <= 1e-4).all()
    x[1] = 0
    assert (b.group_norm(x, 4)[1] == 0).all()


@pytest.mark.parametrize("P", [100, 3000, 60000, 300000])
def test_far_mean_and_one_outlier(P):
    """Values around 1000 of deviation 1, in one image; zeros with one large value in front, in the other."""
    gpu()
    rng = np.random.default_rng(P)
    x = torch.zeros(2, P, 32, dtype=F16)
    x[0] = torch.from_numpy((1000 + rng.standard_normal((P, 32))).astype(np.float32)).half()
    x[1, 0, 0] = 1000.0
    x = x.cuda()
    y = b.group_norm(x, 4)
    v, u, c = nl.norm(x, 4, None, None, 1e-5, False)
    nl.check(y, v, nl.norm_bound(v, u, c, F16))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("P", [60, 4000])
def test_strides(P, dtype):
    """Slices of wider rows, in and out, an addend that all images share, images in reverse order of memory left to torch."""
    gpu()
    wide, gamma, beta, _ = make(7, 3, P, 960, dtype, add=False)
    e = torch.randn(1, 320, device="cuda").to(dtype).expand(3, 320)
    x = wide[:, :, 320:640]
    out = torch.full((3, P, 400), 7.0, dtype=dtype, device="cuda")
    y = b.group_norm(x, 32, gamma[:320], beta[:320], act=b.ACT_SILU, add=e, out=out[:, :, 64:384])
    assert y.data_ptr() == out[:, :, 64:384].data_ptr()
    against(x, 32, gamma[:320], beta[:320], 1e-5, True, e, y)
    assert (out[:, :, :64] == 7).all() and (out[:, :, 384:] == 7).all()
    swapped = wide.transpose(0, 1).contiguous().transpose(0, 1)  # pixels outermost
    assert torch.equal(b.group_norm(swapped, 32, gamma, beta), b.group_norm(wide, 32, gamma, beta))


def test_maps_of_rows_and_columns():
    gpu()
    x, gamma, beta, _ = make(8, 2, 15 * 21, 64, F16, add=False)
    flat = b.group_norm(x, 8, gamma, beta)
    assert torch.equal(b.group_norm(x.view(2, 15, 21, 64), 8, gamma, beta), flat.view(2, 15, 21, 64))
    assert torch.equal(b.group_norm(x.view(2, 15, 21, 64)[:, :, :1], 8).view(2, 15, 64), b.group_norm(x.view(2, 15, 21, 64)[:, :, 0].contiguous(), 8))
    with pytest.raises(ValueError):
        b.group_norm(x.view(2, 15, 21, 64)[:, :, :20], 8)


@pytest.mark.parametrize("shape", [(2, 64, 1280), (2, 4096, 320), (1, 100000, 128)])
def test_in_place(shape):
    gpu()
    x, gamma, beta, e = make(9, *shape, F16)
    y = b.group_norm(x, 32, gamma, beta, act=b.ACT_SILU, add=e)
    assert b.group_norm(x, 32, gamma, beta, act=b.ACT_SILU, add=e, out=x) is x
    assert torch.equal(x, y)


@pytest.mark.parametrize("shape", [(3, 70, 64), (3, 5000, 320), (2, 120000, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_not_finite(shape, bad):
    """The group is NaN, the others are what they were."""
    gpu()
    x, gamma, beta, _ = make(10, *shape, F16, add=False)
    clean = b.group_norm(x, 32, gamma, beta)
    x[1, shape[1] // 2, 5] = bad
    y = b.group_norm(x, 32, gamma, beta)
    n = shape[2] // 32
    at = 5 // n
    assert torch.isnan(y[1, :, at * n:(at + 1) * n]).all()
    y[1, :, at * n:(at + 1) * n] = clean[1, :, at * n:(at + 1) * n]
    assert torch.equal(y, clean)


def test_large_and_small_bf16():
    gpu()
    x, gamma, beta, _ = make(11, 2, 500, 64, BF16, add=False)
    for f in (1e30, 1e-12):
        big = (x.double() * f).to(BF16)
        against(big, 8, gamma, beta, 1e-30, False, None, b.group_norm(big, 8, gamma, beta, eps=1e-30))


# ------------------------------------------------------------------ codes
def grouping(seed, C, P, bits, G, R, silu, z=None, T=1):
    rng = np.random.default_rng(seed)
    col = rng.integers(0, G, C)
    row = rng.integers(0, R, P)
    scale = np.exp(rng.uniform(-0.5, 0.5, (T, R, G))).astype(np.float32) * np.float32(8.0 / 2 ** bits)
    zp = np.full((T, R, G), z) if z is not None else rng.integers(0, 2 ** bits // (4 if silu else 1), (T, R, G))
    return b.groups_from_host(C, P, bits, col, row, scale, zp)


def codes_against(g, x, groups, gamma, beta, silu, e, timestep, centred, got, eps=1e-5):
    v, _, _ = nl.norm(x, groups, gamma, beta, eps, silu, e)
    ref = nl.codes(v, g.export(), g.bits, timestep, centred)
    assert torch.equal(got.cpu().long(), ref)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,P,C,groups", [s for s in SHAPES if s[1] * s[2] // s[3] > 1 and s[3] <= 2048] + [(1, 40, 4096, 2048)])
@pytest.mark.parametrize("bits,G,R,centred", [(6, 16, 1, True), (8, 5, 2, False), (4, 1, 1, False), (6, 3, 3, True), (2, 32, 1, True), (8, 32, 32, False)])
def test_codes(B, P, C, groups, dtype, bits, G, R, centred):
    gpu()
    if B * P * C > 1 << 21 and (bits, R) != (6, 1):
        pytest.skip("the large maps once")
    x, gamma, beta, e = make(B + P + C, B, P, C, dtype, add=P % 2 == 0)
    silu = C % 3 != 0
    g = grouping(P, C, P, bits, min(G, C), R, silu)
    q = b.group_norm_quantize(g, x, groups, gamma, beta, act=b.ACT_SILU if silu else b.ACT_NONE, add=e,
                              layout=b.CODES_S8_CENTRED if centred else b.CODES_U8)
    codes_against(g, x, groups, gamma, beta, silu, e, 0, centred, q)


def test_codes_of_a_timestep_and_another_period():
    """Row 1 of the table; pixel positions repeat with the grouping's own period, not with the map's."""
    gpu()
    x, gamma, beta, _ = make(3, 3, 50, 96, F16, add=False)
    g = grouping(4, 96, 35, 6, 4, 3, False, T=2)
    q = b.group_norm_quantize(g, x, 8, gamma, beta, timestep=1, layout=b.CODES_S8_CENTRED)
    codes_against(g, x, 8, gamma, beta, False, None, 1, True, q)


@pytest.mark.parametrize("z", [0, 255, -3, 300, -70000, 70000, 2 ** 21, -2 ** 30])
def test_codes_of_far_zero_points(z):
    gpu()
    x, gamma, beta, e = make(4, 2, 90, 64, F16)
    beta = beta - 0.05 * z if abs(z) < 1000 else beta
    g = grouping(5, 64, 90, 8, 3, 1, False, z=z)
    q = b.group_norm_quantize(g, x, 8, gamma, beta, add=e)
    codes_against(g, x, 8, gamma, beta, False, e, 0, False, q)


def test_codes_next_to_borders():
    """Scales so fine that a 32-bit value leaves the code open for most values, and tables whose steps are the map's own."""
    gpu()
    x, gamma, beta, _ = make(6, 1, 400, 64, F16, add=False)
    n = 64
    scale = np.full((1, 1, 2), 2.0 ** -18, np.float32)
    v, _, _ = nl.norm(x, 8, gamma, beta, 1e-5, True)
    zp = np.full((1, 1, 2), -int(v.median() * 2 ** 18) + 128)
    g = b.groups_from_host(n, 400, 8, np.arange(n) % 2, np.zeros(400), scale, zp)
    q = b.group_norm_quantize(g, x, 8, gamma, beta, act=b.ACT_SILU)
    codes_against(g, x, 8, gamma, beta, True, None, 0, False, q)


@pytest.mark.parametrize("centred", [True, False])
def test_codes_of_values_that_are_not_finite(centred):
    gpu()
    x, gamma, beta, _ = make(12, 2, 300, 64, F16, add=False)
    x[0, 7, 3], x[1, 8, 40] = float("inf"), float("nan")
    g = grouping(9, 64, 300, 6, 4, 1, False)
    q = b.group_norm_quantize(g, x, 8, gamma, beta, layout=b.CODES_S8_CENTRED if centred else b.CODES_U8)
    codes_against(g, x, 8, gamma, beta, False, None, 0, centred, q)


def test_codes_feed_the_layer():
    """The codes are dgq_quantize_act's on the same values, up to the values' rounding to 16 bits, and in its layout."""
    gpu()
    x, gamma, beta, _ = make(13, 2, 256, 320, F16, add=False)
    g = grouping(10, 320, 256, 8, 6, 2, True)
    a = b.group_norm_quantize(g, x, 32, gamma, beta, act=b.ACT_SILU)
    y = b.group_norm(x, 32, gamma, beta, act=b.ACT_SILU)
    c, _, _ = b.quantize_act(g, y.view(-1, 320))
    d = (a.int() - c.int()).abs()
    assert d.max() <= 1 and (d > 0).float().mean() < 0.05
    pad = torch.from_numpy(g.export()["perm"] < 0)
    assert torch.equal(a[:, pad.cuda()], c[:, pad.cuda()])


# ------------------------------------------------------------------ streams, graphs, memory
@pytest.mark.parametrize("shape", [(2, 64, 1280), (2, 4096, 320), (1, 100000, 128)])
def test_another_stream_and_graphs(shape):
    """On a side stream, then as two graphs with workspaces of their own replayed in turn, with other inputs in the same place."""
    gpu()
    x, gamma, beta, e = make(14, *shape, F16)
    g = grouping(11, shape[2], shape[1], 6, 8, 1, True)
    want = [b.group_norm(x, 32, gamma, beta, add=e), b.group_norm_quantize(g, x, 32, gamma, beta, act=b.ACT_SILU, add=e)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [b.group_norm(x, 32, gamma, beta, add=e, stream=side), b.group_norm_quantize(g, x, 32, gamma, beta, act=b.ACT_SILU, add=e, stream=side)]
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graphs = []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = b.group_norm(x, 32, gamma, beta, add=e) if k == 0 else b.group_norm_quantize(g, x, 32, gamma, beta, act=b.ACT_SILU, add=e)
        graphs.append((graph, out))
    x.copy_(torch.flip(x, (1,)) * 0.5)
    want = [b.group_norm(x, 32, gamma, beta, add=e), b.group_norm_quantize(g, x, 32, gamma, beta, act=b.ACT_SILU, add=e)]
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, (_, q) in zip(want, graphs))


def test_two_streams_at_once():
    gpu()
    made = [(make(30 + i, *s, F16), n) for i, (s, n) in enumerate((((2, 4096, 320), 32), ((1, 100000, 128), 32)))]
    g = [grouping(20 + i, x.shape[2], x.shape[1], 6, 8, 1, True) for i, ((x, *_), _) in enumerate(made)]
    call = lambda i, **k: (b.group_norm(made[i][0][0], made[i][1], *made[i][0][1:3], add=made[i][0][3], **k),
                           b.group_norm_quantize(g[i], made[i][0][0], made[i][1], *made[i][0][1:3], act=b.ACT_SILU, **k))
    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[call(i, stream=streams[i]) for _ in range(5)] for i in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            assert all(torch.equal(p, q) for p, q in zip(want[i], out))


def test_many_calls_in_a_row_and_a_workspace_of_the_callers():
    gpu()
    shapes = [(2, 64, 1280), (1, 300, 64), (2, 4096, 320), (1, 90000, 128), (3, 7, 24)]
    made = [make(20 + i, *s, F16) for i, s in enumerate(shapes)]
    n_groups = [32, 8, 32, 32, 3]
    size = max(b.group_norm_workspace_bytes(*s, n) for s, n in zip(shapes, n_groups))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert size > 0
    want = [b.group_norm(x, n, g, c, add=e) for (x, g, c, e), n in zip(made, n_groups)]
    for _ in range(5):
        ws.fill_(255)
        got = [b.group_norm(x, n, g, c, add=e, workspace=ws) for (x, g, c, e), n in zip(made, n_groups)]
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_more_elements_than_31_bits():
    """Two images 2^31 elements apart."""
    gpu()
    x, gamma, beta, _ = make(15, 2, 100, 64, F16, add=False)
    far = torch.empty((1 << 31) + 64 * 100, dtype=F16, device="cuda").as_strided((2, 100, 64), (1 << 31, 64, 1))
    far.copy_(x)
    assert torch.equal(b.group_norm(far, 8, gamma, beta), b.group_norm(x, 8, gamma, beta))
    g = grouping(12, 64, 100, 6, 4, 1, False)
    assert torch.equal(b.group_norm_quantize(g, far, 8, gamma, beta), b.group_norm_quantize(g, x, 8, gamma, beta))


def test_refusals_of_the_binding():
    gpu()
    x, gamma, beta, e = make(16, 2, 10, 64, F16)
    for call in (lambda: b.group_norm(x.float(), 8), lambda: b.group_norm(x[0], 8), lambda: b.group_norm(x, 8, gamma[:32]),
                 lambda: b.group_norm(x, 8, gamma.half()), lambda: b.group_norm(x, 8, add=e[:1]), lambda: b.group_norm(x, 8, add=e.float()),
                 lambda: b.group_norm(x, 8, out=x[:, :5]), lambda: b.group_norm(x.transpose(1, 2), 8), lambda: b.group_norm(x.cpu(), 8),
                 lambda: b.group_norm_quantize(grouping(1, 32, 10, 6, 2, 1, False), x, 8)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.group_norm(x, 7), lambda: b.group_norm(x, 8, eps=0.0), lambda: b.group_norm(x, 8, act=2),
                 lambda: b.group_norm_quantize(grouping(1, 64, 10, 6, 2, 1, False), x, 8, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(b.DgqError):
            call()
    wide = torch.zeros(1, 2, 4096, dtype=F16, device="cuda")
    with pytest.raises(b.DgqError) as refused:
        b.group_norm_quantize(grouping(1, 4096, 2, 6, 2, 1, False), wide, 4096)
    assert refused.value.status == 3
    empty = b.group_norm(x[:0], 8)
    assert empty.shape == (0, 10, 64) and b.group_norm(x[:, :0], 8).shape == (2, 0, 64)


def test_codes_of_the_widest_table():
    """Cells, statistics and channels that leave shared memory room for one set of a row's words, over more rows than one round of blocks has."""
    gpu()
    C, P = 4096, 600
    x, gamma, beta, e = make(17, 1, P, C, F16)
    rng = np.random.default_rng(18)
    scale = np.exp(rng.uniform(-0.5, 0.5, (1, 32, 32))).astype(np.float32) / np.float32(32)
    g = b.groups_from_host(C, P, 8, np.arange(C) % 32, np.arange(P) % 32, scale, rng.integers(0, 256, (1, 32, 32)))
    for silu in (False, True):
        q = b.group_norm_quantize(g, x, 2048, gamma, beta, act=b.ACT_SILU if silu else b.ACT_NONE, add=e)
        codes_against(g, x, 2048, gamma, beta, silu, e, 0, False, q)


# ------------------------------------------------------------------ bf16 maps up to the type's end
def far_map(kind, B, P, C, groups):
    """outlier: two values of 3e38 among those around -3e38; wide: deviations of 1e38; addend: the sums with the addend leave 32 bits; mixed: every
    second group has deviations of 1e38, the others of 1."""
    rng = np.random.default_rng(B + P + C)
    n = np.clip(rng.standard_normal((B, P, C)).astype(np.float32), -3, 3)
    e = None
    if kind == "outlier":
        n = np.float32(-3e38) * (1 + np.float32(0.01) * n)
        n[0, 0, 0] = n[-1, P // 2, C // 2] = 3e38
    elif kind == "mixed":
        n[:, :, np.arange(C) // (C // groups) % 2 == 1] *= np.float32(1e38)
    else:
        n *= np.float32(1e38)
        if kind == "addend":
            e = torch.from_numpy(np.clip(rng.standard_normal((B, C)).astype(np.float32) * 3, -3, 3) * np.float32(1e38)).to(BF16).cuda()
    gamma = torch.from_numpy((1 + 0.2 * rng.standard_normal(C)).astype(np.float32)).cuda()
    beta = torch.from_numpy((0.2 * rng.standard_normal(C)).astype(np.float32)).cuda()
    x = torch.from_numpy(n).to(BF16).cuda()
    assert torch.isfinite(x).all()
    return x, gamma, beta, e


FAR_KINDS = ["outlier", "wide", "addend", "mixed"]


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("bits,R,centred", [(8, 1, False), (6, 1, True), (8, 3, False), (6, 3, True)])
@pytest.mark.parametrize("B,P,C,groups", [(2, 500, 64, 8), (1, 333, 24, 8), (1, 4096, 96, 8)])
@pytest.mark.parametrize("kind", FAR_KINDS)
def test_codes_of_far_bf16(kind, B, P, C, groups, bits, R, centred, silu):
    gpu()
    x, gamma, beta, e = far_map(kind, B, P, C, groups)
    rng = np.random.default_rng(bits + R)
    scale = np.exp(rng.uniform(-0.5, 0.5, (1, R, 4))).astype(np.float32) * np.float32(128.0 / 2 ** bits)  # an outlier's code is none of the ends
    g = b.groups_from_host(C, P, bits, np.arange(C) % 4, np.arange(P) % R, scale, rng.integers(0, 2 ** bits // 4, (1, R, 4)))
    q = b.group_norm_quantize(g, x, groups, gamma, beta, act=b.ACT_SILU if silu else b.ACT_NONE, add=e,
                              layout=b.CODES_S8_CENTRED if centred else b.CODES_U8)
    codes_against(g, x, groups, gamma, beta, silu, e, 0, centred, q)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("B,P,C,groups", [(2, 500, 64, 8), (1, 333, 24, 8), (1, 1000, 96, 8), (2, 4096, 320, 32), (1, 2, 8, 1), (1, 90000, 128, 32),
                                          (1, 70001, 8, 2), (1, 150000, 24, 8)])
@pytest.mark.parametrize("kind", FAR_KINDS)
def test_values_of_far_bf16(kind, B, P, C, groups, silu):
    gpu()
    x, gamma, beta, e = far_map(kind, B, P, C, groups)
    against(x, groups, gamma, beta, 1e-5, silu, e, b.group_norm(x, groups, gamma, beta, act=b.ACT_SILU if silu else b.ACT_NONE, add=e))


@pytest.mark.parametrize("P", [64, 150000])
def test_far_bf16_with_a_large_eps_and_far_constants(P):
    """An eps of ten times the variance counts; equal values give beta, also where 32 bits do not hold them."""
    gpu()
    x, gamma, beta, _ = far_map("wide", 1, P, 64, 8)
    x = (x.double() * 1e-20).to(BF16)
    against(x, 8, gamma, beta, 1e37, False, None, b.group_norm(x, 8, gamma, beta, eps=1e37))
    x.fill_(3e38)
    e = torch.full((1, 64), 2e38, dtype=BF16, device="cuda")
    for add in (None, e):
        assert torch.equal(b.group_norm(x, 8, gamma, beta, add=add), beta.to(BF16).expand(1, P, 64))


@pytest.mark.parametrize("size", [1e12, 1e22, 1e30])
@pytest.mark.parametrize("P", [300, 150000])
def test_silu_of_far_values(P, size):
    """Factors so large that a SiLU's argument is far out: it is the argument or, below, at most 2^-60 of it (and its rounding)."""
    gpu()
    x, gamma, beta, _ = make(19, 1, P, 24, BF16, add=False)
    gamma = gamma * size
    y = b.group_norm(x, 8, gamma, beta, act=b.ACT_SILU)
    v, u, c = nl.norm(x, 8, gamma, beta, 1e-5, True)
    nl.check(y, v, nl.norm_bound(v, u, c, BF16))
    assert (y.cpu().double().abs() <= 2.0 ** -59 * u.abs())[u < -100].all()


@pytest.mark.parametrize("size", [1e12, 1e16, 1e22, 1e30])
@pytest.mark.parametrize("R", [1, 2])
def test_codes_of_far_silus(R, size):
    gpu()
    x, gamma, beta, _ = make(20, 1, 300, 64, F16, add=False)
    x[:, 150:] = -x[:, :150]  # a mean of 0, so that nothing but the factor is large
    gamma = gamma * size
    for bits, centred in ((8, False), (6, True)):
        g = grouping(13, 64, 300, bits, 4, R, True)
        q = b.group_norm_quantize(g, x, 8, gamma, beta, act=b.ACT_SILU, layout=b.CODES_S8_CENTRED if centred else b.CODES_U8)
        codes_against(g, x, 8, gamma, beta, True, None, 0, centred, q)


@pytest.mark.parametrize("P", [300, 150000])
def test_silu_of_far_values_f16(P):
    gpu()
    x, gamma, beta, _ = make(19, 1, P, 24, F16, add=False)
    gamma = gamma * 1e22
    y = b.group_norm(x, 8, gamma, beta, act=b.ACT_SILU).cpu().double()
    _, u, _ = nl.norm(x, 8, gamma, beta, 1e-5, True)
    assert torch.isposinf(y[u > 1e6]).all()
    assert (y.abs() <= 2.0 ** -59 * u.abs())[u < -1e6].all()


@pytest.mark.parametrize("R", [1, 2])
@pytest.mark.parametrize("value", [7.0, 9984.0, 222 * 2.0 ** 60, 222 * 2.0 ** 120])
@pytest.mark.parametrize("P,groups", [(333, 8), (75, 24), (25, 8), (77, 24)])
def test_codes_of_constant_maps(P, groups, value, R):
    """Equal values, 75 of them (whose sum times the reciprocal of 75 need not be them) among others: the code of beta, however far out they are."""
    gpu()
    x, gamma, beta, _ = make(21, 1, P, 24, BF16, add=False)
    x.fill_(value)
    assert (x.double() == value).all()
    g = grouping(14, 24, P, 8, 3, R, False)
    q = b.group_norm_quantize(g, x, groups, gamma, beta)
    codes_against(g, x, groups, gamma, beta, False, None, 0, False, q)


def test_images_apart_and_overlapping():
    """Every distance of images and of pixels up to 13 times eight channels: what does not overlap is written as it is asked for, all else refused."""
    gpu()
    B, P, C = 3, 4, 16
    x, gamma, beta, _ = make(23, B, P, C, F16, add=False)
    want = b.group_norm(x, 2, gamma, beta)
    refused = 0
    for batch in range(0, 104, 8):
        for token in range(0, 104, 8):
            buf = torch.full((4096,), 7.0, dtype=F16, device="cuda")
            out = buf.as_strided((B, P, C), (batch, token, 1))
            places = (torch.arange(B)[:, None, None] * batch + torch.arange(P)[:, None] * token + torch.arange(C)).flatten()
            if places.unique().numel() < B * P * C:
                refused += 1
                with pytest.raises(b.DgqError) as e:
                    b.group_norm(x, 2, gamma, beta, out=out)
                assert e.value.status == 1 and (buf == 7).all()
            else:
                b.group_norm(x, 2, gamma, beta, out=out)
                left = torch.full_like(buf, 7.0)
                left[places.cuda()] = want.flatten()
                assert torch.equal(buf, left)
    assert 80 < refused < 160


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,P,C,groups", [(2, 64, 1280, 32), (1, 333, 320, 32), (1, 257, 72, 24), (3, 37, 24, 8)])
@pytest.mark.parametrize("bits,G,R,centred,z", [(8, 5, 1, True, 128), (8, 5, 3, True, 128), (7, 4, 1, True, None), (7, 4, 3, True, None), (7, 4, 1, False, None),
                                                (5, 3, 2, True, None), (3, 3, 1, True, None), (3, 2, 4, False, None)])
def test_codes_of_other_widths(B, P, C, groups, dtype, bits, G, R, centred, z):
    """Zero-centred codes of 8 bits (their zero-point is 128), of 7, the most that leave a bit free, and of odd widths."""
    gpu()
    x, gamma, beta, e = make(B + P + C + bits, B, P, C, dtype, add=P % 2 == 0)
    for silu in (False, True):
        g = grouping(P + bits, C, P, bits, G, R, silu, z=z)
        q = b.group_norm_quantize(g, x, groups, gamma, beta, act=b.ACT_SILU if silu else b.ACT_NONE, add=e,
                                  layout=b.CODES_S8_CENTRED if centred else b.CODES_U8)
        codes_against(g, x, groups, gamma, beta, silu, e, 0, centred, q)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape", [(3, 70, 64), (2, 5000, 320), (2, 120000, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_addends_that_are_not_finite(shape, bad, dtype):
    """The group of that image is NaN, and its codes are 0; the others are what they were."""
    gpu()
    x, gamma, beta, e = make(22, *shape, dtype)
    n = shape[2] // 16
    at = slice(5 // n * n, 5 // n * n + n)
    g = grouping(15, shape[2], shape[1], 8, 4, 1, False)
    place = torch.from_numpy(np.argsort(np.where((p := g.export()["perm"]) < 0, 1 << 20, p), kind="stable")[:shape[2]]).cuda()  # of every channel
    clean, codes = b.group_norm(x, 16, gamma, beta, add=e), b.group_norm_quantize(g, x, 16, gamma, beta, add=e)
    e[1, 5] = bad
    y, q = b.group_norm(x, 16, gamma, beta, add=e), b.group_norm_quantize(g, x, 16, gamma, beta, add=e)
    assert torch.isnan(y[1, :, at]).all()
    y[1, :, at] = clean[1, :, at]
    assert torch.equal(y, clean)
    rows = slice(shape[1], 2 * shape[1])
    assert (q[rows][:, place[at]] == 0).all()
    q[rows][:, place[at]] = codes[rows][:, place[at]]
    assert torch.equal(q, codes)
