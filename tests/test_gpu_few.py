"""Products of few rows with 4-bit weights in groups, against 64 bits."""
import numpy as np
import pytest
import torch

import norm_testlib as nl
from dgq_testlib import gpu
from paper_2501_04304_b200 import binding as b

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def make(seed, M, K, N, group, dtype, bias=True):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dtype).cuda()
    wq = torch.from_numpy(rng.integers(-8, 8, (N, K)).astype(np.int8)).cuda()
    scales = torch.from_numpy(np.exp(0.3 * rng.standard_normal((N, -(-K // group)))).astype(np.float32) * 0.02).half().cuda()
    c = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).to(dtype).cuda() if bias else None
    return x, wq, scales, c


def against(x, wq, scales, group, silu, c, y):
    ref, size = nl.few(x, wq, scales, group, silu, c)
    nl.check(y, ref, nl.few_bound(ref, size, x.dtype, silu, x.shape[1]))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 8, 1), (2, 1280, 320), (1, 4096, 4096), (7, 5000, 1007), (8, 72, 16), (9, 136, 17), (16, 640, 1280), (17, 1000, 33),
                                   (24, 96, 100), (31, 2048, 250), (32, 320, 640), (33, 128, 48), (100, 768, 320), (3, 10240, 1280), (1, 200, 5000),
                                   (4, 64, 20001), (5, 8192, 15), (12, 4096, 1600), (32, 1024, 6150), (20, 520, 12500), (45, 1288, 3100),
                                   (16, 8192, 800), (9, 712, 6300), (33, 4160, 3000)])
def test_products(M, K, N, group, dtype):
    gpu()
    x, wq, scales, c = make(M + K + N, M, K, N, group, dtype, bias=N % 2 == 0)
    w = b.few_weight_from_codes(wq, scales, group)
    for silu in (False, True):
        y = b.linear_few(w, x, bias=c, act=b.ACT_SILU if silu else b.ACT_NONE)
        assert y.shape == (M, N) and y.dtype == dtype
        against(x, wq, scales, group, silu, c, y)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_code_is_at_its_place(group):
    """Unit rows give the weights themselves, exactly."""
    gpu()
    K, N = 328, 37
    _, wq, scales, _ = make(1, 1, K, N, group, F16)
    w = b.few_weight_from_codes(wq, scales, group)
    y = b.linear_few(w, torch.eye(K, dtype=F16, device="cuda"))
    want = (wq.float() * scales.float().repeat_interleave(group, 1)[:, :K]).half().T
    assert torch.equal(y, want)
    codes, s = w.export()
    assert np.array_equal(codes, wq.cpu().numpy()) and np.array_equal(s, scales.cpu().numpy())


def test_weights_that_start_anywhere():
    """Codes and fp16 weights one element behind an aligned place."""
    gpu()
    _, wq, scales, _ = make(9, 1, 200, 21, 32, F16)
    want = b.few_weight_from_codes(wq, scales, 32).export()
    buf = torch.zeros(21 * 200 + 1, dtype=torch.int8, device="cuda")
    buf[1:] = wq.flatten()
    got = b.few_weight_from_codes(buf[1:].view(21, 200), scales, 32).export()
    assert all(np.array_equal(p, q) for p, q in zip(got, want))
    W = torch.randn(21, 200, device="cuda").half()
    want = b.few_weight_prepare(W, 64).export()
    buf = torch.zeros(21 * 200 + 1, dtype=F16, device="cuda")
    buf[1:] = W.flatten()
    got = b.few_weight_prepare(buf[1:].view(21, 200), 64).export()
    assert all(np.array_equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(40, 328), (16, 128), (5, 1000), (1, 8)])
def test_round_to_nearest(N, K, group):
    gpu()
    rng = np.random.default_rng(N + K)
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    W[0, :8] = 0
    if N > 4:
        W[4] = 0                  # a row of nothing
        W[3] *= np.float16(1e-3)  # scales below the smallest normal fp16
        W[2, ::7] = 60000         # and the largest
    w = b.few_weight_prepare(torch.from_numpy(W).cuda(), group)
    codes, scales = w.export()
    n = -(-K // group)
    wide = np.zeros((N, n * group), np.float64)
    wide[:, :K] = W
    top = np.abs(wide.reshape(N, n, group)).max(2)
    s = scales.astype(np.float64)
    # the smallest fp16 that is not below top / 7
    assert (s >= top / 7).all()
    below = np.nextafter(scales, np.float16(-np.inf)).astype(np.float64)
    assert (below[top > 0] < (top / 7 * (1 + 2.0 ** -23))[top > 0]).all() and (s[top == 0] == 0).all()
    with np.errstate(divide="ignore", invalid="ignore"):
        t = np.where(top[..., None] > 0, wide.reshape(N, n, group) / s[..., None], 0).reshape(N, -1)[:, :K]
    assert np.abs(codes).max() <= 7
    assert (np.abs(codes - t) <= 0.5 + 2.0 ** -20).all()


def test_strides_and_outputs():
    gpu()
    K, N = 640, 333
    x, wq, scales, c = make(2, 6, K, N, 64, F16)
    w = b.few_weight_from_codes(wq, scales, 64)
    want = b.linear_few(w, x, bias=c)
    wide = torch.zeros(6, 1000, dtype=F16, device="cuda")
    wide[:, 64:64 + K] = x
    assert torch.equal(b.linear_few(w, wide[:, 64:64 + K], bias=c), want)
    out = torch.full((6, 500), 9.0, dtype=F16, device="cuda")
    assert torch.equal(b.linear_few(w, x, bias=c, out=out[:, 7:7 + N]), want)
    assert (out[:, :7] == 9).all() and (out[:, 7 + N:] == 9).all()
    assert torch.equal(b.linear_few(w, x[:1].expand(6, K), bias=c), want[:1].expand(6, N))
    assert b.linear_few(w, x[:0]).shape == (0, N)


def test_rows_do_not_meet():
    """A row's result does not depend on the others, not even on NaN in them."""
    gpu()
    for M in (8, 20, 40):
        x, wq, scales, c = make(3, M, 400, 100, 128, BF16)
        w = b.few_weight_from_codes(wq, scales, 128)
        want = b.linear_few(w, x, bias=c)
        x[M // 2] = float("nan")
        got = b.linear_few(w, x, bias=c)
        assert torch.isnan(got[M // 2]).all()
        got[M // 2] = want[M // 2]
        assert torch.equal(got, want)


def test_short_rows_do_not_read_on():
    """What lies behind a row's K channels may be anything."""
    gpu()
    K, N = 200, 64
    x, wq, scales, _ = make(4, 3, K, N, 128, F16)
    w = b.few_weight_from_codes(wq, scales, 128)
    wide = torch.full((3, 256), float("nan"), dtype=F16, device="cuda")
    wide[:, :K] = x
    assert torch.equal(b.linear_few(w, wide[:, :K]), b.linear_few(w, x))


@pytest.mark.parametrize("silu", [False, True])
def test_large_values(silu):
    gpu()
    x, wq, scales, _ = make(5, 4, 256, 32, 64, BF16, bias=False)
    x *= 1e30
    w = b.few_weight_from_codes(wq, scales, 64)
    y = b.linear_few(w, x, act=b.ACT_SILU if silu else b.ACT_NONE)
    ref, size = nl.few(x, wq, scales, 64, silu, None)
    nl.check(y, ref, nl.few_bound(ref, size, BF16, silu, 256))


def test_another_stream_and_graphs():
    gpu()
    x, wq, scales, c = make(6, 2, 1280, 320, 64, F16)
    w = b.few_weight_from_codes(wq, scales, 64)
    want = b.linear_few(w, x, bias=c, act=b.ACT_SILU)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = b.linear_few(w, x, bias=c, act=b.ACT_SILU, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graphs = []
    for act in (b.ACT_SILU, b.ACT_NONE):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = b.linear_few(w, x, bias=c, act=act)
        graphs.append((graph, out))
    x.mul_(-0.5)
    want = [b.linear_few(w, x, bias=c, act=a) for a in (b.ACT_SILU, b.ACT_NONE)]
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, (_, q) in zip(want, graphs))


def test_refusals():
    gpu()
    x, wq, scales, c = make(7, 2, 64, 32, 64, F16)
    w = b.few_weight_from_codes(wq, scales, 64)
    for call in (lambda: b.linear_few(w, x.float()), lambda: b.linear_few(w, x[:, :56]), lambda: b.linear_few(w, x, bias=c.bfloat16()),
                 lambda: b.linear_few(w, x, bias=c[:8]), lambda: b.linear_few(w, x, out=torch.empty(2, 31, dtype=F16, device="cuda")),
                 lambda: b.linear_few(w, x.t().contiguous().t()), lambda: b.few_weight_from_codes(wq, scales, 48),
                 lambda: b.few_weight_from_codes(wq, scales[:16], 64), lambda: b.few_weight_from_codes(wq.int(), scales, 64),
                 lambda: b.few_weight_prepare(x.float())):
        with pytest.raises(ValueError):
            call()
    bad = wq.clone()
    bad[31, 63] = 8
    inf = scales.clone()
    inf[3, 0] = float("inf")
    nan = torch.zeros(8, 64, dtype=F16, device="cuda")
    nan[7, 63] = float("nan")
    for call in (lambda: b.few_weight_from_codes(bad, scales, 64), lambda: b.few_weight_from_codes(wq, inf, 64), lambda: b.few_weight_prepare(nan),
                 lambda: b.linear_few(w, x, act=2)):
        with pytest.raises(b.DgqError) as e:
            call()
        assert e.value.status == 1
    with pytest.raises(b.DgqError):  # rows of 60 channels do not start on 16 bytes
        b.linear_few(b.few_weight_from_codes(wq[:, :56].contiguous(), scales, 64), torch.zeros(2, 60, dtype=F16, device="cuda")[:, :56])


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("M", [1, 8, 12, 30, 70])
def test_infinities_and_silu(M, group, dtype):
    """silu(inf) is inf: the outputs are infinities of the codes' signs; the other rows are what they were."""
    gpu()
    K, N = 712, 100
    x, wq, scales, c = make(10 + M, M, K, N, group, dtype)
    at = [3, K - 1, 300]
    sign = torch.where(torch.arange(N, device="cuda") % 3 == 0, -1, 1).to(torch.int8)
    for k in at:
        wq[:, k] = sign * (1 + k % 7)
    w = b.few_weight_from_codes(wq, scales, group)
    want = b.linear_few(w, x, bias=c, act=b.ACT_SILU)
    rows = sorted({0, M // 2, M - 1})
    for i, m in enumerate(rows):
        x[m, at[i]] = float("inf")
        want[m] = sign.to(dtype) * float("inf")
    assert torch.equal(b.linear_few(w, x, bias=c, act=b.ACT_SILU), want)
    assert torch.equal(b.linear_few(w, x, bias=c)[rows], want[rows])


@pytest.mark.parametrize("M", [2, 12, 30])
@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-5])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_silu_of_small_rows(dtype, size, M):
    """A SiLU's results are good to 2^-20 of them and 2^-25 (fp16), 2^-15 of them and 2^-119 (bf16): a part each of the sum of the terms' sizes and of the
    weights'.  Beside them the output's rounding and the sums' (as in few_bound)."""
    gpu()
    K, N, group = 320, 64, 64
    x, wq, scales, _ = make(20 + M, M, K, N, group, dtype, bias=False)
    x = (x.double() * size).to(dtype)
    y = b.linear_few(b.few_weight_from_codes(wq, scales, group), x, act=b.ACT_SILU)
    ref, terms = nl.few(x, wq, scales, group, True, None)
    _, weights = nl.few(torch.ones_like(x), wq, scales, group, False, None)
    part, least = (2.0 ** -20, 2.0 ** -25) if dtype == F16 else (2.0 ** -15, 2.0 ** -119)
    limit = nl.HALF_STEP[dtype] * ref.abs() + 2.0 ** -25 * (dtype == F16) + ((K / 16 + 30) * 2.0 ** -23 + part) * terms + least * weights
    nl.check(y, ref, limit)
