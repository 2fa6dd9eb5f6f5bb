"""dgq_kv_write where the rows of a page do not follow one another: rows left out, skipped tokens, slots that do not ascend."""
import pytest
import torch

from dgq_testlib import gpu
from test_gpu_kv_cache import dev, quantize_reference, random_cache

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
FAR = 2 ** 31 - 1


def accepted(slots, page, n_slots):
    """The slots with -1 for those that are skipped, and whether any of these is recorded: one beyond the cache, or not above all
    of its page's in the same run."""
    out, at, top, recorded = [], None, -1, False
    for s in slots:
        if 0 <= s < n_slots and s // page != at:
            at, top = s // page, -1
        good = 0 <= s < n_slots and s % page > top
        recorded |= not good and s >= 0
        if good:
            top = s % page
        out.append(s if good else -1)
    return out, recorded


def every(step, first, last):
    return list(range(first, last, step))


GAPS = [
    # heads, d, page, slots
    (2, 64, 16, [32, 34]),
    (2, 40, 16, [5, 7, 16, 18]),
    (1, 64, 16, [5, -1, 6]),
    (3, 64, 16, [16, 17, -1, 19]),
    (2, 8, 16, [0, 2, 4, 33, 47]),
    # a page of zeros' rows between, more skipped tokens than a warp looks at in one read, in the run and behind it
    (2, 128, 16, [3] + [-1] * 300 + [9] + [-3] * 1000 + [64, 65] + [-1] * 700),
    (1, 40, 16, [-1, 3, -2 ** 31, 4, 5] + [-2 ** 31] * 2500 + [7] + [-1] * 1024 + [48, 50] + [-1] * 5001),
    (1, 64, 64, [70] + [-1] * 1087 + [71] + [-1] * 4096 + [73, 74] + [-1] * 127 + [75] + [-1] * 300),
    (2, 64, 32, [-1] * 1500 + [40] + [-1] * 31 + [41, 43] + [-1] * 600 + [64]),
    (1, 160, 32, every(2, 33, 128)),
    (5, 104, 16, every(3, 1, 600)),
    # runs that the whole block has, more rows than stay in registers
    (2, 128, 64, every(1, 70, 100) + every(1, 101, 128) + [256, 299]),
    (2, 160, 128, every(2, 1, 128) + [-1] * 40 + every(3, 128, 300)),
    (1, 8, 128, every(1, 5, 100) + [-1] + every(1, 100, 128)),
    # slots beyond the cache inside a run, slots that do not ascend, one twice
    (2, 64, 16, [5, 6, 40 * 16, 7, FAR, 9]),
    (2, 64, 16, [5, 3, 6, 16, 16, 18]),
    (2, 64, 128, [5, 7, 7, 6, 9, 127, 0, 128]),
    # runs that begin inside a warp's window of tokens, and in front of it
    (4, 8, 16, [s for s in range(16 * 500) if s % 5]),
    (16, 8, 16, [s for s in range(16 * 500) if s % 5]),
    (8, 8, 32, [s if s % 7 else -1 for s in range(32 * 250)]),
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("heads,d,page,slots", GAPS, ids=[f"{i}_{g[0]}x{g[1]}_page{g[2]}" for i, g in enumerate(GAPS)])
def test_rows_with_gaps(heads, d, page, slots, dtype):
    _, b = gpu()
    pages = max(40, -(-len(slots) * 2 // page)) if page < 64 and len(slots) > 2500 else 40
    c = random_cache(b, pages, heads, page, d, seed=d)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(len(slots), heads, d, generator=g).to(dtype) * f for f in (1.0, 3.0))
    v[:, 0] = 0  # one head's pages keep their scale, or get none
    real, recorded = accepted(slots, page, pages * page)
    want = [quantize_reference(x, real, codes.cpu(), scale.cpu(), page) for x, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale))]
    before = [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    for offset in range(4 if -1 in slots else 1):  # a slot map may begin at any multiple of four bytes
        for x, y in zip((c.k, c.v, c.k_scale, c.v_scale), before):
            x.copy_(y)
        b.kv_write(c, k.cuda(), v.cuda(), dev([5] * offset + slots)[offset:])
        assert torch.equal(c.k.cpu(), want[0][0]) and torch.equal(c.k_scale.cpu(), want[0][1])
        assert torch.equal(c.v.cpu(), want[1][0]) and torch.equal(c.v_scale.cpu(), want[1][1])
        assert b.device_status() == int(recorded)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("d,page,slots", [
    (64, 16, list(range(16, 60))), (40, 32, list(range(5, 90))), (128, 64, [70, 71, 128, 200]), (160, 128, list(range(1, 128)) + list(range(256, 300))),
    (64, 16, [33, 35, 36, 48, 50]), (64, 128, list(range(7, 120, 2))),
], ids=lambda x: None if isinstance(x, list) else str(x))
def test_values_that_are_not_finite(d, page, slots, dtype):
    """Such a value counts as 0 and is recorded; other rows, pages and heads are as without it."""
    _, b = gpu()
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(len(slots), 3, d, generator=g).to(dtype) for _ in range(2))
    clean = [k.clone(), v.clone()]
    for x, z, places in ((k, clean[0], [(1, 0, 0, "nan"), (3, 0, d - 1, "inf")]), (v, clean[1], [(2, 1, 5, "-inf"), (0, 1, 1, "-nan")])):
        for t, h, i, value in places:
            x[t, h, i], z[t, h, i] = float(value), 0.0
    v[:, 2], clean[1][:, 2] = float("nan"), 0.0  # a head without a finite value
    c = random_cache(b, 40, 3, page, d, seed=d)
    want = [quantize_reference(x, slots, codes.cpu(), scale.cpu(), page) for x, codes, scale in zip(clean, (c.k, c.v), (c.k_scale, c.v_scale))]
    b.kv_write(c, k.cuda(), v.cuda(), dev(slots))
    assert b.device_status() == 1
    assert torch.equal(c.k.cpu(), want[0][0]) and torch.equal(c.k_scale.cpu(), want[0][1])
    assert torch.equal(c.v.cpu(), want[1][0]) and torch.equal(c.v_scale.cpu(), want[1][1])


@pytest.mark.parametrize("page", [16, 128])
def test_skipped_rows_hold_anything(page):
    _, b = gpu()
    slots = [16, 17, -1, 19, -2, 40 * page, page * 3 - 1]
    g = torch.Generator().manual_seed(3)
    x = torch.randn(len(slots), 2, 64, generator=g).half()
    x[[2, 4, 5]] = torch.tensor([float("nan"), float("inf"), float("-inf")]).half()[:, None, None]
    c = random_cache(b, 40, 2, page, 64, seed=4)
    want = quantize_reference(x, [s if s < 40 * page else -1 for s in slots], c.k.cpu(), c.k_scale.cpu(), page)
    b.kv_write(c, x[:5].cuda(), x[:5].cuda(), dev(slots[:5]))
    assert b.device_status() == 0
    c = random_cache(b, 40, 2, page, 64, seed=4)
    b.kv_write(c, x.cuda(), x.cuda(), dev(slots))
    assert b.device_status() == 1  # the slot beyond the cache
    assert torch.equal(c.k.cpu(), want[0]) and torch.equal(c.k_scale.cpu(), want[1])
