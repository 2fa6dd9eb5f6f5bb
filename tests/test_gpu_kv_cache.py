"""The paged 8-bit cache: plans, rows in, values out and attention over it, each against its definition in plain code, and a run of
them together as a server uses them."""
import math

import numpy as np
import pytest
import torch

from dgq_testlib import gpu
from encoder_testlib import HALF_STEP, attention, bound, check

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def plan_reference(lens, new, free, table, page, n_tokens):
    table, slots, taken, starts = table.copy(), [], 0, [0]
    for b, (n, m) in enumerate(zip(lens, new)):
        have, need = -(-n // page), -(-(n + m) // page)
        table[b, have:need] = free[taken:taken + need - have]
        taken += need - have
        slots += [table[b, p // page] * page + p % page for p in range(n, n + m)]
        starts.append(len(slots))
    return table, starts, [n + m for n, m in zip(lens, new)], slots + [-1] * (n_tokens - len(slots)), taken


@pytest.mark.parametrize("B,page,top,new", [(1, 16, 0, 1), (8, 16, 77, 77), (9, 128, 500, 3), (300, 32, 200, 40), (700, 64, 1, 0)])
def test_plan(B, page, top, new):
    _, b = gpu()
    rng = np.random.RandomState(B)
    lens, add = rng.randint(0, top + 1, B), rng.randint(0, new + 1, B)
    max_pages = -(-(top + new) // page) + 1
    free = rng.permutation(B * max_pages * 2).astype(np.int32)
    table = np.full((B, max_pages), -7, np.int32)
    held = np.arange(max_pages)[None, :] < -(-lens // page)[:, None]
    table[held] = free[-held.sum():] if held.any() else 0
    n_tokens = int(add.sum()) + 5
    want = plan_reference(lens, add, free, table, page, n_tokens)
    t = dev(table)
    start, kv, slots, used = b.kv_plan(dev(lens), dev(add), dev(free), t, page, n_tokens)
    assert np.array_equal(t.cpu(), want[0]) and start.tolist() == want[1] and kv.tolist() == want[2]
    assert slots.tolist() == want[3] and used.item() == want[4] and b.device_status() == 0


def test_plan_that_does_not_fit():
    _, b = gpu()
    # the second request lacks a page, the third's lengths are beyond the table, the fourth's negative
    t = dev(np.full((4, 2), -1))
    start, kv, slots, used = b.kv_plan(dev([0, 0, 30, -3]), dev([16, 16, 9, 1]), dev([5]), t, 16, 40)
    assert b.device_status() == 1
    assert t.tolist()[:2] == [[5, -1], [-1, -1]] and start.tolist() == [0, 16, 32, 34, 35] and kv.tolist() == [16, 16, 32, 1]
    assert slots.tolist() == list(range(80, 96)) + [-1] * 24 and used.item() == 1
    # room for fewer tokens than there are
    start, kv, slots, used = b.kv_plan(dev([0]), dev([20]), dev([1, 0]), dev([[-1, -1]]), 16, 18)
    assert b.device_status() == 1 and slots.tolist() == list(range(16, 32)) + [0, 1]


def quantize_reference(x, slots, codes, scale, page):
    """kv_write of one tensor in the arithmetic that the header states, page by page."""
    codes, scale, d = codes.clone(), scale.clone(), x.shape[2]
    by_page = {}
    for t, s in enumerate(slots):
        if s >= 0:
            by_page.setdefault(s // page, []).append((s % page, t))
    for p, rows in by_page.items():
        at, new = [r for r, _ in rows], x[[t for _, t in rows]].float()
        first = min(at)
        top = new.abs().amax((0, 2))
        s = torch.where(top > 0, torch.clamp(top * torch.tensor(1.0 / 127.0), min=2.0 ** -126), torch.zeros(()))
        if first:
            s = torch.maximum(s, scale[p])
        if first:
            old = codes[p, :, :first].float()
            codes[p, :, :first] = torch.where((s > scale[p])[:, None, None], (old * scale[p][:, None, None] / s[:, None, None]).round(), old).to(torch.int8)
        q = torch.where(s[None, :, None] > 0, new / s[None, :, None], torch.zeros(())).round().to(torch.int8)
        for i, r in enumerate(at):
            codes[p, :, r, :d] = q[i]
            codes[p, :, r, d:] = 0
        scale[p] = s
    return codes, scale


def random_cache(b, n_pages, heads, page, d, seed):
    g = torch.Generator().manual_seed(seed)
    c = b.KvCache.empty(n_pages, heads, page, d)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes[..., :d] = torch.randn(n_pages, heads, page, d, generator=g).mul_(32).round_().clamp_(-127, 127).to(torch.int8).cuda()
        scale.copy_(torch.rand(n_pages, heads, generator=g) * 0.03 + 0.01)
    return c


WRITES = [
    # heads, d, page, slots
    (1, 8, 16, [0]),
    (2, 40, 16, list(range(16, 16 + 77))),
    (3, 64, 32, [37, 38, 39, 64, 65, 5, 200, -1, -1]),
    (2, 128, 64, list(range(70, 128)) + list(range(256, 300)) + [3]),
    (2, 160, 128, list(range(1, 128)) + list(range(384, 512))),
    (5, 104, 16, [p * 16 + p % 16 for p in range(30)]),
]


@TYPES
@pytest.mark.parametrize("heads,d,page,slots", WRITES, ids=[f"{w[0]}x{w[1]}_page{w[2]}" for w in WRITES])
def test_write_and_read(heads, d, page, slots, dtype):
    _, b = gpu()
    c = random_cache(b, 40, heads, page, d, seed=d)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(len(slots), heads, d, generator=g).to(dtype) * f for f in (1.0, 3.0))
    want = [quantize_reference(x, slots, codes.cpu(), scale.cpu(), page) for x, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale))]
    b.kv_write(c, k.cuda(), v.cuda(), dev(slots))
    # bit for bit: both sides round the same 32-bit quotients
    assert torch.equal(c.k.cpu(), want[0][0]) and torch.equal(c.k_scale.cpu(), want[0][1])
    assert torch.equal(c.v.cpu(), want[1][0]) and torch.equal(c.v_scale.cpu(), want[1][1])
    rk, rv = b.kv_read(c, dev(slots), dtype)
    assert b.device_status() == 0
    for r, (codes, scale), x in ((rk, want[0], k), (rv, want[1], v)):
        for t, s in enumerate(slots):
            if s < 0:
                assert not r[t].any()
                continue
            value = codes[s // page, :, s % page, :d].float() * scale[s // page][:, None]
            assert torch.equal(r[t].cpu(), value.to(dtype))
            # half a code's step, and both sides' roundings to `dtype`
            limit = 0.5001 * scale[s // page][:, None] + 2 * HALF_STEP[dtype] * x[t].float().abs()
            assert ((r[t].cpu().float() - x[t].float()).abs() <= limit).all()


def test_write_zeros_and_views():
    _, b = gpu()
    c = b.KvCache.empty(4, 2, 16, 40)
    fused = torch.randn(20, 3, 2, 40, generator=torch.Generator().manual_seed(2)).half().cuda()
    fused[:, 2, 1] = 0
    slots = list(range(16, 36))
    b.kv_write(c, fused[:, 1], fused[:, 2], dev(slots))
    k, v = b.kv_read(c, dev(slots))
    assert not v[:, 1].any() and not c.v_scale[1:3, 1].any()
    assert (k.float() - fused[:, 1].float()).abs().max() <= 0.51 * c.k_scale.max() + 2 * 2.0 ** -11 * 5
    out = torch.full((20, 2, 2, 40), 5.0, dtype=F16, device="cuda")
    b.kv_read(c, dev(slots), out=(out[:, 0], out[:, 1]))
    assert torch.equal(out[:, 0], k) and torch.equal(out[:, 1], v)
    # a page whose rows are all zero takes the scale of what comes next
    b.kv_write(c, fused[:4, 1], fused[:4, 1], dev([36, 37, 38, 39]))
    assert (c.v_scale[2, 1] > 0).item()


@TYPES
def test_codes_near_borders(dtype):
    """Rows full of odd multiples of half a scale, up to the type's rounding: the quotient in 32 bits decides."""
    _, b = gpu()
    c = b.KvCache.empty(300, 1, 16, 64)
    top = (torch.rand(300, generator=torch.Generator().manual_seed(15)) * 60 + 0.01).to(dtype)
    x = (top.float()[:, None] * (2 * torch.arange(64) + 1) / 254).to(dtype)
    x[:, 63], x[:, 31], x[:, 30] = top, top / 2, -top / 2
    slots = [16 * i for i in range(300)]
    b.kv_write(c, x[:, None].cuda(), (-x[:, None]).cuda(), dev(slots))
    codes, scale = quantize_reference(x[:, None], slots, torch.zeros(300, 1, 16, 64, dtype=torch.int8), torch.zeros(300, 1), 16)
    assert torch.equal(c.k.cpu(), codes) and torch.equal(c.v.cpu(), -codes) and torch.equal(c.k_scale.cpu(), scale)


def test_slots_beyond_the_cache():
    _, b = gpu()
    c = random_cache(b, 3, 2, 16, 64, seed=3)
    before = c.k.clone(), c.k_scale.clone()
    x = torch.ones(3, 2, 64, dtype=F16, device="cuda")
    b.kv_write(c, x, x, dev([48, -5, 2 ** 31 - 1]))
    assert b.device_status() == 1
    assert torch.equal(c.k, before[0]) and torch.equal(c.k_scale, before[1])
    k, _ = b.kv_read(c, dev([48, -5, 2 ** 31 - 1]))
    assert not k.any() and b.device_status() == 1


def values(codes, scale, d):
    return codes[..., :d].double().cpu() * scale.double().cpu()[..., None, None]


def compare(O, q, c, table, lens, starts, causal, scale=None):
    """O, q packed [rows, H, d]."""
    d, page = c.d, c.page
    scale = 1 / math.sqrt(d) if scale is None else scale
    k, v = values(c.k, c.k_scale, d), values(c.v, c.v_scale, d)
    for b, n in enumerate(lens):
        n = min(max(n, 0), len(table[b]) * page)
        pages = torch.tensor([int(p) for p in table[b][:-(-n // page)]], dtype=torch.long)
        kk, vv = (x[pages].transpose(1, 2).reshape(-1, x.shape[1], d)[:n] for x in (k, v))
        rows = slice(starts[b], starts[b + 1])
        nq = starts[b + 1] - starts[b]
        if nq == 0:
            continue
        sees = [min(n, max(0, n - nq + i + 1)) if causal else n for i in range(nq)]
        qq = q[rows].double().cpu()
        o, spread, plain = attention(qq, kk, vv, sees, scale)
        # a key's value is code * scale, its weight is rounded times the page's scale: the smallest weights are off by 2^-25 of
        # the largest such product
        check(O[rows], o, bound(o, spread, plain * 256, qq, kk, scale, q.dtype, F16))


CACHED = [
    # B, H, G, d, page, lens, queries, causal
    (1, 1, 1, 8, 16, [1], [1], False),
    (3, 4, 4, 64, 16, [300, 0, 17], [1, 1, 1], False),
    (3, 8, 2, 128, 64, [1000, 64, 65], [1, 1, 1], False),
    (2, 10, 5, 40, 32, [511, 33], [2, 2], False),
    (2, 8, 1, 160, 128, [700, 129], [3, 3], True),
    (4, 4, 2, 80, 16, [100, 5, 0, 31], [7, 0, 2, 130], False),
    (3, 2, 2, 40, 16, [77, 20, 154], [300, 1, 129], False),
    (2, 4, 1, 64, 64, [400, 290], [200, 290], True),
    (2, 2, 1, 128, 128, [385, 130], [131, 140], True),
    (1, 2, 2, 160, 32, [260], [129], True),
    (2, 2, 2, 104, 64, [200, 140], [33, 40], False),
    (1, 40, 1, 96, 16, [333], [1], False),
    (1, 2, 1, 64, 16, [1500], [70], True),
]


def cached_case(b, B, H, G, d, page, lens, nq, dtype, seed=0, spare=3):
    need = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(need) + spare
    order = np.random.RandomState(seed).permutation(n_pages)
    table = np.full((B, max(1, max(need))), -1, np.int64)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    c = random_cache(b, n_pages, G, page, d, seed)
    q = torch.randn(sum(nq), H, d, generator=torch.Generator().manual_seed(seed + 1)).to(dtype).cuda()
    return c, table, q, np.concatenate([[0], np.cumsum(nq)]).tolist()


@TYPES
@pytest.mark.parametrize("case", CACHED, ids=lambda c: "x".join(map(str, c[:5])))
def test_cached_attention(case, dtype):
    _, b = gpu()
    B, H, G, d, page, lens, nq, causal = case
    c, table, q, starts = cached_case(b, B, H, G, d, page, lens, nq, dtype)
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=max(nq), causal=causal)
    assert b.device_status() == 0
    compare(O, q, c, table, lens, starts, causal)
    if len(set(nq)) == 1:
        four = q.view(B, nq[0], H, d)
        assert torch.equal(b.cached_attn(four, c, dev(table), dev(lens), causal=causal).view_as(O), O)


@TYPES
@pytest.mark.parametrize("G,H,d,page,lens,nq", [
    (16, 16, 40, 16, [154, 20, 0, 33, 154, 97, 16, 160], [1500, 1100, 200, 1024, 1, 129, 128, 900]),
    (5, 20, 64, 64, [190, 64, 130, 7], [700, 300, 1000, 1000]), (10, 20, 128, 32, [128, 33, 70, 96], [600, 900, 31, 32]),
    (2, 4, 128, 16, [1000, 500], [300, 257]), (2, 2, 160, 64, [700, 90], [300, 100]),
])
def test_many_rows(G, H, d, page, lens, nq, dtype):
    """Several tiles of packed queries a block, requests that end inside a tile, blocks of keys that are codes."""
    _, b = gpu()
    c, table, q, starts = cached_case(b, len(lens), H, G, d, page, lens, nq, dtype, seed=14)
    more = torch.cat([q, q[:50]])
    out = torch.full_like(more, 3.0)
    b.cached_attn(more, c, dev(table), dev(lens), q_start=dev(starts), max_nq=max(nq), out=out)
    assert b.device_status() == 0 and (out[len(q):] == 3.0).all()
    for i, n in enumerate(lens):
        rows = slice(starts[i], starts[i + 1])
        if n == 0:
            assert not out[rows].any()
            continue
        pages = torch.as_tensor(table[i, :-(-n // page)]).cuda()
        k, v = ((x[pages][..., :d].double() * s[pages].double()[..., None, None]).transpose(1, 2).reshape(-1, G, d)[:n].repeat_interleave(H // G, 1).transpose(0, 1)
                for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        a = torch.softmax(q[rows].double().transpose(0, 1) @ k.transpose(1, 2) * d ** -0.5, -1)
        ref = [x.transpose(0, 1).cpu() for x in (a @ v, a @ v.abs(), v.abs().sum(1, keepdim=True).expand(-1, nq[i], -1))]
        check(out[rows], ref[0], bound(ref[0], ref[1], ref[2] * 256, q[rows].double(), k, d ** -0.5, dtype, F16))


@pytest.mark.parametrize("nq,lens", [(1, [200, 77]), (140, [200, 77]), (140, [160, 77])])
def test_queries_of_any_size(nq, lens):
    """bf16 queries far outside fp16's range: a power of two in the queries and its inverse in the scale change no bit."""
    _, b = gpu()
    c, table, q, starts = cached_case(b, 2, 4, 2, 64, 16, lens, [nq, nq], BF16, seed=16)
    four = q.view(2, nq, 4, 64)
    O = b.cached_attn(four, c, dev(table), dev(lens), scale=0.125)
    compare(O.view(-1, 4, 64), q, c, table, lens, starts, False)
    for e in (60, -60):
        assert torch.equal(b.cached_attn((four.float() * 2.0 ** e).bfloat16(), c, dev(table), dev(lens), scale=0.125 * 2.0 ** -e), O)
    # the outputs in the queries' place
    same = four.clone()
    b.cached_attn(same, c, dev(table), dev(lens), scale=0.125, out=same)
    assert torch.equal(same, O)


@pytest.mark.parametrize("nq", [1, 2, 150])
def test_scales_far_apart(nq):
    """Pages of zeros, and pages whose values are 2^14 times smaller than others' in front of those with the large weights."""
    _, b = gpu()
    lens = [200, 177]
    c, table, q, starts = cached_case(b, 2, 4, 2, 64, 16, lens, [nq, nq], F16, seed=7)
    c.v_scale[table[0, 3]] = 0
    c.v[table[0, 3]] = 0
    c.k_scale[table[1, 2]] = 0
    c.v_scale[table[1, :10]] *= 2.0 ** -14
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=nq)
    compare(O, q, c, table, lens, starts, False)


@pytest.mark.parametrize("nq", [1, 150])
def test_small_pages_with_all_the_weight(nq):
    """Keys that take all the weight lie on pages whose values are 2^-12 of the others': their weights must not sink below
    what fp16 holds."""
    _, b = gpu()
    lens = [160]
    c, table, q, starts = cached_case(b, 1, 2, 2, 64, 16, lens, [nq], F16, seed=8)
    c.k_scale.mul_(0.02)
    q[:, :, 0] = 8.0
    page = table[0, 4]
    c.k_scale[page] = 0.25
    c.k[page] = 0
    c.k[page, :, :, 0] = 100
    c.v_scale[page] *= 2.0 ** -12
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=nq)
    v = values(c.v, c.v_scale, 64)[page].mean(1)  # every row sees the page's sixteen keys alike
    # sixteen equal weights, exact in fp16 up to one rounding; the rest of the keys weigh less than e^-20 each
    limit = (2.0 ** -10 * v.abs() + 2.0 ** -10 * values(c.v, c.v_scale, 64)[page].abs().mean(1) + 144 * math.exp(-20) * 4 + 2.0 ** -24)[None]
    assert ((O.double().cpu() - v[None]).abs() <= limit).all()


def test_rows_outside_requests_and_bad_tables():
    _, b = gpu()
    for nq in (1, 140):
        lens = [100, 90]
        c, table, q, starts = cached_case(b, 2, 2, 1, 64, 16, lens, [nq, nq], BF16, seed=9)
        more = torch.cat([q, q, q])
        out = torch.full_like(more, 3.0)
        begin = [nq + s for s in starts]
        b.cached_attn(more, c, dev(table), dev(lens), q_start=dev(begin), max_nq=nq, out=out)
        assert b.device_status() == 0
        compare(out[nq:], more[nq:], c, table, lens, starts, False)
        assert (out[:nq] == 3.0).all() and (out[3 * nq:] == 3.0).all()
        # an entry outside the cache: its tokens count as absent
        bad = table.copy()
        bad[0, 2], bad[1, 0] = c.k.shape[0], -1
        O = b.cached_attn(q, c, dev(bad), dev(lens), q_start=dev(starts), max_nq=nq)
        assert b.device_status() == 1
        k, v = (values(x, s, 64) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        for i, gap in ((0, 2), (1, 0)):
            keep = [j for j in range(lens[i]) if j // 16 != gap]
            kk, vv = (torch.stack([x[bad[i, j // 16], :, j % 16] for j in keep]) for x in (k, v))
            qq = q[i * nq:(i + 1) * nq].double().cpu()
            o, spread, plain = attention(qq, kk, vv, [len(keep)] * nq, 0.125)
            check(O[i * nq:(i + 1) * nq], o, bound(o, spread, plain * 256, qq, kk, 0.125, BF16, F16))


def test_more_queries_than_said():
    _, b = gpu()
    lens = [50, 60]
    c, table, q, starts = cached_case(b, 2, 2, 2, 40, 16, lens, [5, 3], F16, seed=10)
    out = torch.full_like(q, 2.0)
    b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=3, out=out)
    assert b.device_status() == 1
    assert (out[3:5] == 2.0).all() and (out[5:] != 2.0).any() and (out[:3] != 2.0).any()
    out.fill_(2.0)
    b.cached_attn(q, c, dev(table), dev(lens), q_start=dev([6, 8, 12]), max_nq=4, out=out)
    assert b.device_status() == 1 and (out[:6] == 2.0).all()


def test_offsets_beyond_32_bits():
    """A cache of 2.3 GB of keys: the last page begins behind 2^31 codes."""
    _, b = gpu()
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    c = b.KvCache.empty(9000, 16, 128, 128)
    last = 8999
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(200, 16, 128, generator=g).half().cuda() for _ in range(2))
    slots = list(range(last * 128, last * 128 + 128)) + list(range(8000 * 128, 8000 * 128 + 72))
    b.kv_write(c, k, v, dev(slots))
    rk, rv = b.kv_read(c, dev(slots))
    assert (rk - k).abs().max() < 0.03 and (rv - v).abs().max() < 0.03
    for nq in (1, 130):
        q = torch.randn(1, nq, 16, 128, generator=g).half().cuda()
        O = b.cached_attn(q, c, dev([[last, 8000]]), dev([200]))
        want = b.encoder_attn(q, rk[None], rv[None])
        # the cache's values against the same rounded to fp16: half a step each in keys and values
        assert (O - want).abs().max() < 8 * 2.0 ** -11 * 4
    assert b.device_status() == 0


@TYPES
def test_a_server_step_by_step(dtype):
    """Prompts of different lengths enter the cache, two requests grow by a token at a time across a page's border, every step
    attends to it; one step is captured in a graph and replayed with other lengths; the log-quantized attention takes what is read back."""
    _, b = gpu()
    B, H, G, d, page, max_pages = 3, 4, 2, 64, 16, 6
    g = torch.Generator().manual_seed(12)
    c = b.KvCache.empty(20, G, page, d)
    table, lens = dev(np.full((B, max_pages), -1)), dev([0, 0, 0])
    free = dev(np.random.RandomState(1).permutation(20))
    keys, vals = [[] for _ in range(B)], [[] for _ in range(B)]
    taken = 0
    for new in ([77, 15, 32], [1, 1, 0], [1, 1, 0], [0, 3, 1]):
        T = sum(new)
        k, v = (torch.randn(T, G, d, generator=g).to(dtype) for _ in range(2))
        start, lens, slots, used = b.kv_plan(lens, dev(new), free[taken:], table, page, T + 3)
        taken += used.item()
        pad = torch.zeros(3, G, d, dtype=dtype)
        b.kv_write(c, torch.cat([k, pad]).cuda(), torch.cat([v, pad]).cuda(), slots)
        s = start.tolist()
        for i in range(B):
            keys[i].append(k[s[i]:s[i + 1]])
            vals[i].append(v[s[i]:s[i + 1]])
        q = torch.randn(B, 2, H, d, generator=g).to(dtype).cuda()
        O = b.cached_attn(q, c, table, lens)
        assert b.device_status() == 0
        starts = [0, 2, 4, 6]
        compare(O.view(-1, H, d), q.view(-1, H, d), c, table.cpu().numpy(), lens.tolist(), starts, False)
    # every value is within half a step of its page's scale, and half another one for each time the scale grew (at most three times)
    for i in range(B):
        n = int(lens[i])
        at = table[i].long().cpu()[torch.arange(n) // page] * page + torch.arange(n) % page
        rk, rv = b.kv_read(c, dev(at), dtype)
        for r, x, scale in ((rk, torch.cat(keys[i]), c.k_scale), (rv, torch.cat(vals[i]), c.v_scale)):
            step = scale[at // page].cpu()[..., None]
            assert ((r.cpu().float() - x.float()).abs() <= 2.001 * step + 2 * HALF_STEP[dtype] * x.float().abs()).all()
    q1 = torch.randn(B, 1, H, d, generator=g).to(dtype).cuda()
    out = torch.empty_like(q1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.cached_attn(q1, c, table, lens, out=out)
    lens.copy_(torch.tensor([3, 0, 20], dtype=torch.int32))
    graph.replay()
    assert torch.equal(out, b.cached_attn(q1, c, table, lens)) and not out[1].any()
    if dtype == F16:
        rk, rv = (x.view(1, 77, G, d) for x in b.kv_read(c, dev(table[0].cpu().numpy().repeat(page)[:77] * page + np.arange(77) % page)))
        q = torch.randn(1, 130, G, d, generator=g).half().cuda()
        O, _, _ = b.cross_attn_logq(q, rk, rv, 8)
        assert torch.isfinite(O).all()


@pytest.mark.parametrize("nq", [1, 150])
def test_on_another_stream(nq):
    _, b = gpu()
    lens = [500, 200]
    c, table, q, starts = cached_case(b, 2, 4, 2, 128, 32, lens, [nq, nq], BF16, seed=13)
    t, n, s = dev(table), dev(lens), dev(starts)
    O = b.cached_attn(q, c, t, n, q_start=s, max_nq=nq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = b.cached_attn(q, c, t, n, q_start=s, max_nq=nq, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, other)


def test_refusals():
    _, b = gpu()
    c, table, q, starts = cached_case(b, 2, 4, 2, 64, 16, [20, 20], [1, 1], F16)
    t, n = dev(table), dev([20, 20])
    four = q.view(2, 1, 4, 64)
    for bad in (lambda: b.cached_attn(four.float(), c, t, n), lambda: b.cached_attn(q, c, t, n), lambda: b.cached_attn(four, c, t, n[:1]),
                lambda: b.cached_attn(four, c, t.long(), n), lambda: b.cached_attn(four, c, t, n.cpu()), lambda: b.cached_attn(four, c, t, n, max_nq=2),
                lambda: b.cached_attn(q, c, t, n, q_start=dev([0, 1])), lambda: b.cached_attn(four[..., :56], c, t, n),
                lambda: b.kv_write(c, q[:, :1], q[:, :1], dev([1, 2])), lambda: b.kv_write(c, q[:, :2], q[:, :2], dev([1])),
                lambda: b.kv_write(c, q[:, :2].float(), q[:, :2].float(), dev([1, 2])), lambda: b.kv_read(c, dev([1, 2]).long()),
                lambda: b.kv_read(c, dev([1, 2]), torch.float32), lambda: b.kv_read(c, dev([1]), out=(q[:1, :2], q[:2, :2])),
                lambda: b.kv_plan(n, dev([1]), dev([1]), t, 16, 2), lambda: b.kv_plan(n, n, dev([1]), t, 16, -1),
                lambda: b.kv_plan(n, n, dev([1]), t[:, ::2], 16, 2),
                lambda: b.cached_attn(four, b.KvCache(c.k, c.v[:1], c.k_scale, c.v_scale, 64), t, n),
                lambda: b.cached_attn(four, b.KvCache(c.k, c.v, c.k_scale, c.v_scale.half(), 64), t, n),
                lambda: b.cached_attn(four[..., :40], b.KvCache(c.k, c.v, c.k_scale, c.v_scale, 40), t, n)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(b.DgqError):
        b.cached_attn(four[:, :, :3], c, t, n)
    with pytest.raises(b.DgqError):
        b.kv_plan(n, n, dev([1, 2]), t, 24, 40)
    odd = b.KvCache.empty(4, 2, 24, 64)
    with pytest.raises(b.DgqError):
        b.cached_attn(four, odd, t, n)
