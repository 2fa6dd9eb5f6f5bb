"""dgq_encoder_attn against attention in 64 bits: types, head sizes and groups, lengths from none to several key blocks,
views, masked rubbish, streams and graphs."""
import math

import pytest
import torch

from dgq_testlib import gpu
from encoder_testlib import attention, bound, check

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def make(B, nq, nk, H, G, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(dtype) for s in ((B, nq, H, d), (B, nk, G, d), (B, nk, G, d))]


def compare(O, q, k, v, lens, scale=None):
    B, nq, H, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    for b in range(B):
        n = k.shape[1] if lens is None else min(max(int(lens[b]), 0), k.shape[1])
        qq, kk, vv = q[b].double(), k[b, :n].double(), v[b, :n].double()
        o, spread, plain = attention(qq, kk, vv, [n] * nq, scale)
        check(O[b], o, bound(o, spread, plain, qq, kk, scale, q.dtype, q.dtype))


CASES = [
    # B, nq, nk, H, G, d, lens
    (1, 1, 1, 1, 1, 8, None),
    (2, 130, 77, 2, 2, 40, None),
    (3, 5, 9, 2, 1, 64, [0, 9, 1]),
    (2, 129, 300, 2, 1, 64, [300, 129]),
    (2, 257, 129, 2, 2, 48, [128, 129]),
    (1, 40, 513, 4, 2, 128, [385]),
    (2, 131, 260, 2, 1, 160, [260, 131]),
    (1, 70, 200, 2, 2, 80, [193]),
    (1, 33, 150, 2, 2, 104, [150]),
    (2, 300, 140, 1, 1, 16, [1, 140]),
    # few rows: one query a request, grouped heads
    (3, 1, 1000, 4, 4, 64, [1000, 517, 0]),
    (2, 1, 700, 8, 1, 128, [700, 3]),
    (1, 2, 1300, 10, 5, 40, [1289]),
    (2, 4, 333, 16, 2, 80, [333, 100]),
    (1, 3, 270, 20, 2, 160, [266]),
    (1, 1, 130, 48, 1, 24, [129]),
    (1, 17, 400, 2, 1, 96, [399]),
    (1, 65, 1100, 2, 2, 64, [1030]),
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_against_64_bits(case, dtype):
    _, b = gpu()
    B, nq, nk, H, G, d, lens = case
    q, k, v = make(B, nq, nk, H, G, d, dtype)
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    O = b.encoder_attn(q.cuda(), k.cuda(), v.cuda(), kv_lens=n)
    assert b.device_status() == 0
    compare(O, q, k, v, lens)


def on_gpu(q, k, v, n, scale):
    """Attention of one request in 64 bits on the GPU, all rows alike: (O, sum of a |V|, sum of |V|)."""
    H, G, d = q.shape[1], k.shape[1], q.shape[2]
    kk, vv = (x[:n].double().repeat_interleave(H // G, 1).transpose(0, 1) for x in (k, v))
    a = torch.softmax(q.double().transpose(0, 1) @ kk.transpose(1, 2) * scale, -1)
    return [x.transpose(0, 1).cpu() for x in (a @ vv, a @ vv.abs(), vv.abs().sum(1, keepdim=True).expand(-1, q.shape[0], -1))]


@pytest.mark.parametrize("B,nq,nk,H,G,d,lens", [
    # enough heads that a block walks several tiles of queries over keys that stay in shared memory
    (8, 1100, 77, 16, 16, 40, [77, 1, 16, 17, 64, 0, 65, 76]), (6, 1000, 192, 20, 5, 64, None), (6, 1000, 185, 20, 20, 64, [185, 96, 97, 180, 33, 160]),
    (6, 900, 128, 20, 10, 128, [128, 127, 1, 64, 65, 100]), (6, 900, 100, 20, 20, 72, None),
    # long keys over many blocks, every kernel class of head sizes
    (1, 700, 1500, 4, 2, 64, [1490]), (1, 700, 1500, 4, 4, 128, None), (1, 300, 900, 4, 1, 160, [895]),
])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_many_rows(B, nq, nk, H, G, d, lens, dtype):
    _, b = gpu()
    q, k, v = (t.cuda() for t in make(B, nq, nk, H, G, d, dtype, seed=6))
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    O = b.encoder_attn(q, k, v, kv_lens=n)
    assert b.device_status() == 0
    for i in range(B):
        m = nk if lens is None else lens[i]
        if m == 0:
            assert not O[i].any()
            continue
        ref = on_gpu(q[i], k[i], v[i], m, d ** -0.5)
        check(O[i], ref[0], bound(*ref, q[i].double(), k[i].double(), d ** -0.5, dtype, dtype))


@pytest.mark.parametrize("nq", [1, 3, 200])
@pytest.mark.parametrize("nk,lens", [(300, [0, 1, 128, 237]), (150, [0, 1, 128, 137])])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_rubbish_behind_the_lengths(dtype, nk, lens, nq):
    """NaN, infinities and the type's extremes in keys and values that no row sees."""
    _, b = gpu()
    q, k, v = make(4, nq, nk, 2, 1, 64, dtype, seed=1)
    for i, n in enumerate(lens):
        for t in (k, v):
            t[i, n:] = torch.tensor([float("nan"), float("inf"), float("-inf"), torch.finfo(dtype).min])[torch.arange(nk - n) % 4].to(dtype)[:, None, None]
    O = b.encoder_attn(q.cuda(), k.cuda(), v.cuda(), kv_lens=torch.tensor(lens, dtype=torch.int32).cuda())
    compare(O, q, k, v, lens)
    assert not O[0].any()


@pytest.mark.parametrize("nq", [1, 12, 150])
@pytest.mark.parametrize("nk,d", [(90, 40), (300, 40), (90, 64), (260, 24), (300, 104), (200, 144)])
def test_a_key_that_scores_minus_infinity(nk, d, nq):
    """One feature of one key is -inf where every query is positive: its weight is 0, whichever pieces of a row a lane has."""
    _, b = gpu()
    q, k, v = make(1, nq, nk, 2, 1, d, F16, seed=7)
    q[..., 0] = 1.0
    k[0, 5, :, 0] = float("-inf")
    O = b.encoder_attn(q.cuda(), k.cuda(), v.cuda())
    rest = [i for i in range(nk) if i != 5]
    compare(O, q, k[:, rest], v[:, rest], None)


def test_lengths_outside_the_range_are_clamped():
    _, b = gpu()
    q, k, v = make(3, 20, 50, 1, 1, 40, F16, seed=2)
    lens = [-5, 70, 2 ** 31 - 1]
    O = b.encoder_attn(q.cuda(), k.cuda(), v.cuda(), kv_lens=torch.tensor(lens, dtype=torch.int32).cuda())
    compare(O, q, k, v, lens)


@pytest.mark.parametrize("nq", [1, 150])
@pytest.mark.parametrize("nk,d", [(600, 64), (600, 128), (90, 64), (150, 40)])
def test_large_logits_and_scale(nq, nk, d):
    """Rows whose maximum moves far from block to block, negative scale, zero scale."""
    _, b = gpu()
    q, k, v = make(1, nq, nk, 2, 2, d, BF16, seed=3)
    k = (k * torch.linspace(0.1, 12, nk)[None, :, None, None]).to(BF16)
    for scale in (0.125, -0.5, 0.0):
        O = b.encoder_attn(q.cuda(), k.cuda(), v.cuda(), scale=scale)
        compare(O, q, k, v, None, scale)


@pytest.mark.parametrize("nq", [1, 140])
def test_views(nq):
    """Keys and values as slices of one projection, queries stored head by head, an output inside a larger tensor, states shared by
    the whole batch."""
    torch_, b = gpu()
    g = torch.Generator().manual_seed(4)
    B, nk, H, G, d = 2, 150, 4, 2, 40
    q = torch.randn(B, H, nq, d, generator=g).half().cuda().transpose(1, 2)
    kv = torch.randn(B, nk, 2, G, d, generator=g).half().cuda()
    big = torch.full((B, nq + 3, H + 1, d + 8), 7.0, dtype=F16, device="cuda")
    out = big[:, 1:nq + 1, :H, :d]
    r = b.encoder_attn(q, kv[:, :, 0], kv[:, :, 1], out=out)
    assert r is out
    compare(out, q.cpu(), kv[:, :, 0].cpu(), kv[:, :, 1].cpu(), None)
    rest = big.clone()
    rest[:, 1:nq + 1, :H, :d] = 7.0
    assert (rest == 7.0).all()
    one = kv[:1].expand(B, nk, 2, G, d)
    O = b.encoder_attn(q, one[:, :, 0], one[:, :, 1])
    compare(O, q.cpu(), one[:, :, 0].cpu(), one[:, :, 1].cpu(), None)
    heads = kv[:, :, :, :1].expand(B, nk, 2, H, d)
    O = b.encoder_attn(q, heads[:, :, 0], heads[:, :, 1])
    compare(O, q.cpu(), heads[:, :, 0].cpu(), heads[:, :, 1].cpu(), None)


@pytest.mark.parametrize("nq,nk", [(2, 400), (260, 400), (260, 180)])
def test_same_bits_again_in_a_graph_and_on_a_stream(nq, nk):
    _, b = gpu()
    q, k, v = (t.cuda() for t in make(2, nq, nk, 4, 2, 64, F16, seed=5))
    lens = torch.tensor([nk, 111], dtype=torch.int32).cuda()
    O = b.encoder_attn(q, k, v, kv_lens=lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = b.encoder_attn(q, k, v, kv_lens=lens, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, on_side)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.encoder_attn(q, k, v, kv_lens=lens, out=out)
    lens.copy_(torch.tensor([100, 0], dtype=torch.int32))
    graph.replay()
    want = b.encoder_attn(q, k, v, kv_lens=lens)
    assert torch.equal(out, want) and not out[1].any()


def test_sizes_of_zero():
    _, b = gpu()
    q, k, v = (t.cuda() for t in make(2, 3, 4, 2, 2, 40, F16))
    assert not b.encoder_attn(q, k[:, :0], v[:, :0]).any()
    assert b.encoder_attn(q[:, :0], k, v).shape == (2, 0, 2, 40)


def test_refusals():
    _, b = gpu()
    q, k, v = (t.cuda() for t in make(2, 3, 4, 2, 2, 40, F16))
    with pytest.raises(b.DgqError):  # heads that no key head divides
        b.encoder_attn(torch.cat([q, q[:, :, :1]], 2), k, v)
    for bad in (lambda: b.encoder_attn(q.float(), k.float(), v.float()), lambda: b.encoder_attn(q, k.bfloat16(), v), lambda: b.encoder_attn(q, k[:1], v[:1]),
                lambda: b.encoder_attn(q, k, v[:, :3]), lambda: b.encoder_attn(q, k, v, kv_lens=torch.zeros(2, device="cuda")),
                lambda: b.encoder_attn(q, k, v, kv_lens=torch.zeros(3, dtype=torch.int32, device="cuda")),
                lambda: b.encoder_attn(q, k, v, kv_lens=torch.zeros(2, dtype=torch.int32)), lambda: b.encoder_attn(q, k, v, out=q[:, :2]),
                lambda: b.encoder_attn(q, k.cpu(), v.cpu())):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros(2, 3, 2, 41, dtype=F16, device="cuda")
    with pytest.raises(b.DgqError) as e:  # strides of 41
        b.encoder_attn(wide[..., :40], k, v)
    assert e.value.status == 2
    with pytest.raises(b.DgqError) as e:
        b.encoder_attn(q, k, v, scale=float("nan"))
    assert e.value.status == 1
    with pytest.raises(b.DgqError) as e:  # an output that broadcasts
        b.encoder_attn(q, k, v, out=torch.empty(1, 3, 2, 40, dtype=F16, device="cuda").expand(2, 3, 2, 40))
    assert e.value.status == 1
