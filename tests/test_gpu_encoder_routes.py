"""Attention over encoder states and over the cache where the launch rules change: clusters of two and of sixteen blocks, requests dealt out
longest first, blocks of keys whose maxima grow, rows without keys, rows of several requests in one launch.  148 SMs are meant."""
import numpy as np
import pytest
import torch

from attention_testlib import attend, check
from dgq_testlib import gpu
from test_gpu_kv_cache import cached_case, dev

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])


def lengths(B, top, seed=0):
    """Lengths of all kinds, several alike: zero, one, negative, beyond the keys, any."""
    g = np.random.RandomState(seed)
    kinds = [top, top * 2 // 3, 0, 1, top, -4, top + 9, top // 2, top // 2]
    return [int(kinds[i]) if i < len(kinds) else int(g.randint(0, top + 1)) for i in g.permutation(B)]


def encoder_case(B, nq, nk, H, G, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda").to(dtype) for s in ((B, nq, H, d), (B, nk, G, d), (B, nk, G, d))]


def check_encoder(O, q, k, v, lens, scale=None):
    B, nq, H, d = q.shape
    for b in range(B):
        n = k.shape[1] if lens is None else min(max(lens[b], 0), k.shape[1])
        check(O[b], attend(q[b].double(), k[b, :n].double(), v[b, :n].double(), n, d ** -0.5 if scale is None else scale, q.dtype, q.dtype))


def check_cached(O, q, c, table, lens, starts, causal, scale=None):
    """O, q packed [rows, H, d]."""
    d, page = c.d, c.page
    for b, n in enumerate(lens):
        n = min(max(n, 0), table.shape[1] * page)
        rows = slice(starts[b], starts[b + 1])
        nq = starts[b + 1] - starts[b]
        pages = torch.as_tensor(table[b, :-(-n // page)]).cuda()
        k, v = ((x[pages][..., :d].double() * s[pages].double()[..., None, None]).transpose(1, 2).reshape(-1, x.shape[1], d)[:n]
                for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        v_scale = c.v_scale[pages].double().repeat_interleave(page, 0)[:n]
        sees = torch.arange(nq, device="cuda").add_(n - nq + 1).clamp_(0, n) if causal else n
        check(O[rows], attend(q[rows].double(), k, v, sees, d ** -0.5 if scale is None else scale, q.dtype, F16, v_scale))


FEW = [
    # B, H, G, nq, keys (16 bits), d: one block a request and head, 640 to 800 of them
    (100, 8, 8, 1, 100, 64), (128, 5, 5, 2, 70, 128), (129, 5, 5, 1, 70, 40), (90, 14, 7, 1, 60, 160),
    # clusters of two, with more than 592 blocks and with fewer
    (80, 16, 8, 2, 530, 64), (10, 16, 16, 1, 600, 128), (10, 16, 16, 1, 600, 160),
    # clusters of sixteen; 8, 16 and 32 columns
    (3, 4, 2, 1, 4200, 64), (3, 8, 2, 3, 4200, 128), (2, 8, 2, 8, 4200, 64), (2, 8, 2, 8, 4200, 128), (2, 4, 2, 4, 4200, 160), (1, 8, 2, 6, 4200, 160),
]


@TYPES
@pytest.mark.parametrize("B,H,G,nq,nk,d", FEW, ids=lambda x: str(x))
def test_few_rows_over_states(B, H, G, nq, nk, d, dtype):
    _, b = gpu()
    q, k, v = encoder_case(B, nq, nk, H, G, d, dtype)
    lens = lengths(B, nk)
    O = b.encoder_attn(q, k, v, kv_lens=dev(lens))
    assert b.device_status() == 0
    check_encoder(O, q, k, v, lens)


@TYPES
@pytest.mark.parametrize("B,H,G,nq,nk,d", FEW, ids=lambda x: str(x))
def test_few_rows_over_codes(B, H, G, nq, nk, d, dtype):
    """Steps of 32 keys (of 16 for heads of 160) where 16-bit states have 16: twice the keys for the same clusters."""
    _, b = gpu()
    top = nk if d > 128 else 2 * nk
    lens = lengths(B, top)
    page = 64 if top > 500 else 16
    c, table, q, starts = cached_case(b, B, H, G, d, page, [min(max(n, 0), top) for n in lens], [nq] * B, dtype, seed=1)
    lens = [min(n, top) for n in lens]  # the table may be wider than the longest request
    O = b.cached_attn(q.view(B, nq, H, d), c, dev(table), dev(lens))
    assert b.device_status() == 0
    check_cached(O.view(-1, H, d), q, c, table, lens, starts, False)
    assert torch.equal(b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=nq).view_as(O), O)


@TYPES
@pytest.mark.parametrize("d", [64, 128, 160])
def test_many_rows_longest_first(d, dtype):
    """More tiles than places, requests of different, equal and no length."""
    _, b = gpu()
    B, H, G, nq, nk = 9, 16, 4, 500, 300
    q, k, v = encoder_case(B, nq, nk, H, G, d, dtype, seed=2)
    lens = lengths(B, nk, seed=2)
    O = b.encoder_attn(q, k, v, kv_lens=dev(lens))
    assert b.device_status() == 0
    check_encoder(O, q, k, v, lens)
    lens = [300, 0, 129, 128, 300, 1, 257, 299]
    rows = [500, 400, 270, 1, 0, 300, 129, 500]
    for causal in (False, True):
        c, table, q, starts = cached_case(b, 8, H, G, d, 32, lens, rows, dtype, seed=3)
        O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=max(rows), causal=causal)
        assert b.device_status() == 0
        check_cached(O, q, c, table, lens, starts, causal)


@TYPES
@pytest.mark.parametrize("scale", [0.125, -0.25])
@pytest.mark.parametrize("d", [64, 128, 160])
def test_growing_maxima_by_tiles(d, scale, dtype):
    """A row's largest score is far above the one before in every block of keys; more than 256 rows, which are never split."""
    _, b = gpu()
    nq, nk = 300, 700
    q, k, v = encoder_case(1, nq, nk, 2, 1, d, dtype, seed=4)
    k = (k.float() * torch.linspace(0.05, 6, nk, device="cuda")[None, :, None, None]).to(dtype)
    check_encoder(b.encoder_attn(q, k, v, scale=scale), q, k, v, None, scale)
    lens, rows = [690, 530], [300, 290]
    for causal in (False, True):
        c, table, q, starts = cached_case(b, 2, 4, 2, d, 32, lens, rows, dtype, seed=5)
        for i, n in enumerate(lens):
            pages = torch.as_tensor(table[i, :-(-n // 32)]).cuda()
            c.k_scale[pages] *= torch.linspace(0.05, 6, len(pages), device="cuda")[:, None]
        O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=300, causal=causal, scale=scale)
        assert b.device_status() == 0
        check_cached(O, q, c, table, lens, starts, causal, scale)


@TYPES
@pytest.mark.parametrize("d,page", [(40, 16), (64, 64), (128, 128), (160, 32)])
def test_causal_rows_without_keys(d, page, dtype):
    """More rows than keys: the first ones see nothing, in tiles that other rows keep alive."""
    _, b = gpu()
    lens, rows = [300, 40, 700, 0, 257], [400, 300, 5, 270, 258]
    c, table, q, starts = cached_case(b, 5, 4, 2, d, page, lens, rows, dtype, seed=6)
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=400, causal=True)
    assert b.device_status() == 0
    assert not O[:100].any() and not O[400:660].any() and not O[705:975].any() and not O[975].any()
    check_cached(O, q, c, table, lens, starts, True)
    # the same by the kernel for few rows
    rows = [16, 3, 1, 5, 0]
    c, table, q, starts = cached_case(b, 5, 4, 2, d, page, [9, 3, 700, 0, 257], rows, dtype, seed=7)
    O = b.cached_attn(q, c, dev(table), dev([9, 3, 700, 0, 257]), q_start=dev(starts), max_nq=16, causal=True)
    assert not O[:7].any()
    check_cached(O, q, c, table, [9, 3, 700, 0, 257], starts, True)


@TYPES
@pytest.mark.parametrize("d", [40, 64, 128, 160])
@pytest.mark.parametrize("causal", [False, True])
def test_requests_of_one_and_of_many_rows(d, causal, dtype):
    """Up to 128 columns of a key head, most of which most requests do not have; the default of max_nq."""
    _, b = gpu()
    lens, rows = [500, 33, 0, 1300, 64, 1], [16, 1, 7, 1, 0, 9]
    c, table, q, starts = cached_case(b, 6, 16, 2, d, 64, lens, rows, dtype, seed=8)
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=16, causal=causal)
    assert b.device_status() == 0
    check_cached(O, q, c, table, lens, starts, causal)
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), causal=causal)
    assert b.device_status() == 0
    check_cached(O, q, c, table, lens, starts, causal)


@TYPES
@pytest.mark.parametrize("case", [(2, 130, 77, 2, 2, 40), (2, 300, 400, 4, 2, 64), (1, 300, 400, 2, 1, 128), (3, 1, 3000, 4, 2, 128), (1, 40, 90, 2, 1, 160)], ids=str)
def test_states_within_the_roundings(case, dtype):
    _, b = gpu()
    B, nq, nk, H, G, d = case
    q, k, v = encoder_case(B, nq, nk, H, G, d, dtype, seed=9)
    check_encoder(b.encoder_attn(q, k, v), q, k, v, None)


@TYPES
@pytest.mark.parametrize("H,G,d,page,lens,rows", [
    (4, 4, 64, 16, [300, 0, 17], [1, 1, 1]), (8, 2, 128, 64, [3000, 64, 65], [1, 1, 1]), (2, 2, 40, 16, [77, 20, 154], [300, 1, 129]),
    (4, 2, 64, 64, [1500, 290], [300, 290]), (2, 1, 128, 128, [385, 130], [300, 140]), (2, 2, 160, 32, [260], [129]),
], ids=str)
def test_codes_within_the_roundings(H, G, d, page, lens, rows, dtype):
    _, b = gpu()
    c, table, q, starts = cached_case(b, len(lens), H, G, d, page, lens, rows, dtype, seed=10)
    O = b.cached_attn(q, c, dev(table), dev(lens), q_start=dev(starts), max_nq=max(rows))
    assert b.device_status() == 0
    check_cached(O, q, c, table, lens, starts, False)


@pytest.mark.parametrize("nq,n", [(1, 300), (1, 40), (150, 90), (300, 300)])
def test_value_scales_far_apart(nq, n):
    """Pages of values 2^78 and more from one another, and pages of zeros: the row's sum has the weights of all of them.  Every row sees
    the zeros' keys about as much as the others', so that a weight that is lost from the sum shows."""
    _, b = gpu()
    c, table, q, starts = cached_case(b, 1, 2, 2, 64, 16, [n], [nq], BF16, seed=11)
    pages = torch.as_tensor(table[0, :-(-n // 16)]).cuda()
    c.k_scale.mul_(0.02)
    scales = torch.tensor([2.0 ** -40, 2.0 ** 38, 0.0, 2.0 ** 38]).cuda()
    c.v_scale[pages] = scales[torch.arange(len(pages), device="cuda") % 4][:, None]
    c.v[pages[2::4]] = 0
    O = b.cached_attn(q, c, dev(table), dev([n]), q_start=dev(starts), max_nq=nq)
    assert b.device_status() == 0
    check_cached(O, q, c, table, [n], starts, False)
