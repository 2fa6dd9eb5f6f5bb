"""Integer arguments of the native binding that 32 bits do not hold are refused: cut, they would be other sizes."""
import pytest
import torch

from dgq_testlib import gpu
from paper_2501_04304_b200 import binding as b

BIG = [2 ** 31, 2 ** 32 + 16, -2 ** 31 - 1, 2 ** 63 - 1]


@pytest.mark.parametrize("value", BIG)
@pytest.mark.parametrize("name", ["page", "n_tokens", "timestep"])
def test_refused_before_anything_else(name, value):
    """No tensor is looked at before, so no GPU is needed."""
    if name == "timestep":
        call = lambda: b.native().quantize_act(0, 32, 1, value, 0, 0, None, None, None, None, 0, None)
    else:
        sizes = dict(page=16, n_tokens=8)
        sizes[name] = value
        call = lambda: b.kv_plan(None, None, None, None, **sizes)
    with pytest.raises(ValueError, match="32 bits"):
        call()


@pytest.mark.gpu
@pytest.mark.parametrize("value", BIG)
def test_most_queries_of_a_request(value):
    gpu()
    c = b.KvCache.empty(2, 1, 16, 64)
    q = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        b.cached_attn(q, c, ints(0).view(1, 1), ints(1), q_start=ints(0, 1), max_nq=value)
