"""One residual block of a UNet as the calls stand in it: the time embedding's product, norm into codes, 3x3 convolution, norm with the embedding
added into codes, second convolution; against the same steps in 64 bits."""
import numpy as np
import pytest
import torch

import norm_testlib as nl
from dgq_testlib import gpu
from paper_2501_04304_b200 import binding as b

pytestmark = pytest.mark.gpu


def conv64(q, wq, sw, scale, col):
    """q [B, H, W, C] codes less their zero-points (64 bits), wq [N, 3, 3, C]: the de-quantized 3x3 convolution."""
    v = q * scale[col]
    w = wq.double() * sw.double()[:, None, None, None]
    return torch.nn.functional.conv2d(v.permute(0, 3, 1, 2), w.permute(0, 3, 1, 2), padding=1).permute(0, 2, 3, 1)


def test_residual_block():
    gpu()
    B, H, C, E = 2, 16, 64, 128
    rng = np.random.default_rng(1)
    f16 = lambda *s, k=1.0: torch.from_numpy((k * rng.standard_normal(s)).astype(np.float16)).cuda()
    x, temb, bias = f16(B, H, H, C), f16(B, E), f16(C, k=0.1)
    norms = [(torch.from_numpy((1 + 0.1 * rng.standard_normal(C)).astype(np.float32)).cuda(),
              torch.from_numpy((0.1 * rng.standard_normal(C)).astype(np.float32)).cuda()) for _ in range(2)]
    few = b.few_weight_prepare(f16(C, E, k=0.1), 32)
    groups, weights = [], []
    for _ in range(2):
        col = rng.integers(0, 4, C)
        scale = (0.06 * np.exp(0.2 * rng.standard_normal((1, 1, 4)))).astype(np.float32)
        g = b.groups_from_host(C, H * H, 6, col, np.zeros(H * H), scale, np.full((1, 1, 4), 5))
        groups.append(g)
        weights.append(b.weight_prepare(g, f16(C, 3, 3, C, k=0.05), 4, conv=(B, H, H, C)))

    def block(x):
        e = b.linear_few(few, temb, bias=bias, act=b.ACT_SILU)
        q = b.group_norm_quantize(groups[0], x, 32, *norms[0], act=b.ACT_SILU, layout=b.CODES_S8_CENTRED)
        h = b.linear(groups[0], weights[0], q, layout=b.CODES_S8_CENTRED, conv=(B, H, H, C)).view(B, H, H, C)
        q2 = b.group_norm_quantize(groups[1], h, 32, *norms[1], act=b.ACT_SILU, add=e, layout=b.CODES_S8_CENTRED)
        return e, q, h, q2, b.linear(groups[1], weights[1], q2, layout=b.CODES_S8_CENTRED, conv=(B, H, H, C)).view(B, H, H, C)

    e, q, h, q2, y = block(x)
    # every step against 64 bits on the inputs that it got
    codes, scales = few.export()
    ref, size = nl.few(temb, torch.from_numpy(codes), torch.from_numpy(scales), 32, True, bias)
    nl.check(e, ref, nl.few_bound(ref, size, torch.float16, True, E))
    for step, (src, add, got, out) in enumerate(((x, None, q, h), (h, e, q2, y))):
        ex = groups[step].export()
        v, _, _ = nl.norm(src.view(B, H * H, C), 32, *norms[step], 1e-5, True, add)
        assert torch.equal(got.cpu().long(), nl.codes(v, ex, 6, 0, True))
        col = torch.from_numpy(ex["col_group"]).long()
        scale = torch.from_numpy(ex["scale"][0, 0]).double()
        z = torch.from_numpy(ex["zp"][0, 0]).double()
        code = (torch.round(v * (1 / torch.from_numpy(ex["scale"][0, 0])).double()[col]) + z[col]).clamp(0, 63) - z[col]
        wq, sw = weights[step].export()
        ref = conv64(code.view(B, H, H, C), torch.from_numpy(wq).view(C, 3, 3, C), torch.from_numpy(sw), scale, col)
        nl.check(out, ref, 2.0 ** -11 * ref.abs() + 2.0 ** -20 * ref.abs().max() + 2.0 ** -25)
    # the same as a graph, on another map
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = block(x)
    x.copy_(x.flip(1))
    want = block(x)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, r) for p, r in zip(outs, want))
