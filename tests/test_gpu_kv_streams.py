"""The cache's calls on a stream of their own and in captured graphs, and the log-quantized attention over what is read back."""
import numpy as np
import pytest
import torch

from dgq_testlib import gpu
from test_gpu_attention import _compare
from test_gpu_kv_cache import dev, plan_reference, quantize_reference, random_cache

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
HEADS, D, PAGE, WIDE = 2, 64, 16, 8


class Server:
    """The buffers of three requests that a program with captured graphs keeps, and one step over them."""

    def __init__(self, b, dtype, seed):
        self.b, self.dtype = b, dtype
        g = torch.Generator().manual_seed(seed)
        self.cache = random_cache(b, 30, HEADS, PAGE, D, seed)
        self.lens, self.new, self.table = dev([0, 0, 0]), dev([0, 0, 0]), dev(np.full((3, WIDE), -1))
        self.free = dev(np.random.RandomState(seed).permutation(30))
        self.k, self.v = (torch.randn(64, HEADS, D, generator=g).to(dtype).cuda() for _ in range(2))
        self.q = torch.randn(3, 2, 2 * HEADS, D, generator=g).to(dtype).cuda()

    def step(self, stream=None):
        b = self.b
        start, lens, slots, used = b.kv_plan(self.lens, self.new, self.free, self.table, PAGE, 64, stream=stream)
        b.kv_write(self.cache, self.k, self.v, slots, stream=stream)
        k, v = b.kv_read(self.cache, slots, self.dtype, stream=stream)
        return start, lens, slots, used, k, v, b.cached_attn(self.q, self.cache, self.table, lens, stream=stream)

    def state(self):
        c = self.cache
        return [x.clone() for x in (self.table, c.k, c.v, c.k_scale, c.v_scale)]

    def begin(self, lens, new):
        """Lengths of the next step; the table and the free pages start again."""
        need = -(-np.asarray(lens) // PAGE)
        table = np.full((3, WIDE), -1)
        table[np.arange(WIDE)[None] < need[:, None]] = np.arange(need.sum())
        for t, x in ((self.lens, lens), (self.new, new), (self.table, table), (self.free, np.roll(np.arange(30), -int(need.sum())))):
            t.copy_(dev(x))


STEPS = [([0, 0, 0], [33, 16, 1]), ([33, 16, 1], [1, 1, 1]), ([77, 0, 90], [0, 64, 0])]


def same(got, want, n_new):
    """Equal outputs of a step; rows behind the last new one are zeros."""
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert not got[4][n_new:].any() and not got[5][n_new:].any()


@TYPES
def test_on_a_stream_of_their_own(dtype):
    """The same bits as on the current stream; the stream waits only where the program says so, outputs are dropped while it runs."""
    _, b = gpu()
    here, there = Server(b, dtype, 1), Server(b, dtype, 1)
    side = torch.cuda.Stream()
    for lens, new in STEPS:
        here.begin(lens, new)
        there.begin(lens, new)
        want = here.step()
        side.wait_stream(torch.cuda.current_stream())
        got = there.step(side)
        there.b.kv_read(there.cache, got[2], dtype, stream=side)  # dropped at once
        torch.full((64, HEADS, D), 9.0, dtype=dtype, device="cuda")
        torch.cuda.current_stream().wait_stream(side)
        same(got, want, sum(new))
        assert all(torch.equal(x, y) for x, y in zip(there.state(), here.state()))
    assert b.device_status() == 0


@TYPES
def test_two_graphs_in_turn(dtype):
    """Steps captured once and replayed with other lengths, two programs' graphs between each other, against eager steps."""
    _, b = gpu()
    graphs = []
    for seed in (2, 3):
        s = Server(b, dtype, seed)
        s.begin(*STEPS[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = s.step()
        graphs.append((s, Server(b, dtype, seed), graph, out))
    for lens, new in STEPS * 2:
        for s, eager, graph, out in graphs:
            for x in (s, eager):
                x.begin(lens, new)
            graph.replay()
        for s, eager, graph, out in graphs:
            same(out, eager.step(), sum(new))
            assert all(torch.equal(x, y) for x, y in zip(s.state(), eager.state()))
    assert b.device_status() == 0


@TYPES
def test_a_step_against_its_definition(dtype):
    """One step's plan, codes and values, with requests that grow into a page they have begun."""
    _, b = gpu()
    s = Server(b, dtype, 4)
    lens, new = STEPS[1]
    s.begin(lens, new)
    codes = [x.cpu() for x in s.state()[1:]]
    table, start, total, slots, used = plan_reference(lens, new, s.free.cpu().numpy(), s.table.cpu().numpy(), PAGE, 64)
    got = s.step()
    assert np.array_equal(s.table.cpu(), table) and got[0].tolist() == start and got[1].tolist() == total
    assert got[2].tolist() == slots and got[3].item() == used
    for x, c, scale, now, now_scale in ((s.k, codes[0], codes[2], s.cache.k, s.cache.k_scale), (s.v, codes[1], codes[3], s.cache.v, s.cache.v_scale)):
        want = quantize_reference(x.cpu(), slots, c, scale, PAGE)
        assert torch.equal(now.cpu(), want[0]) and torch.equal(now_scale.cpu(), want[1])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d", [40, 64])
def test_log_quantized_attention_over_values_read_back(d, bits):
    """Keys and values of two prompts through the cache and into dgq_cross_attn_logq: the oracle's result for the values that the codes
    stand for."""
    torch_, b = gpu()
    g = torch.Generator().manual_seed(5)
    B, H, nk = 2, 2, 77
    c = b.KvCache.empty(12, H, PAGE, d)
    k, v = (torch.randn(B * nk, H, d, generator=g).half() for _ in range(2))
    table = dev(np.full((B, 5), -1))
    _, lens, slots, _ = b.kv_plan(dev([0, 0]), dev([nk, nk]), dev(np.random.RandomState(6).permutation(12)), table, PAGE, B * nk)
    b.kv_write(c, k.cuda(), v.cuda(), slots)
    rk, rv = b.kv_read(c, slots)
    at = slots.long().cpu()
    for x, codes, scale in ((rk, c.k, c.k_scale), (rv, c.v, c.v_scale)):
        value = codes.cpu()[at // PAGE, :, at % PAGE, :d].float() * scale.cpu()[at // PAGE][..., None]
        assert torch.equal(x.cpu(), value.half())
    q = torch.randn(B, 130, H, d, generator=g).half()
    _compare(torch_, b, q.numpy(), rk.view(B, nk, H, d).cpu().numpy(), rv.view(B, nk, H, d).cpu().numpy(), bits)
