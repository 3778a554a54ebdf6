"""Numbers at the ends of their types in the KV-cache operators.  The plain implementations and the bounds are those of test_gpu_kv.py."""
import pytest
import torch

from test_gpu_kv import BF, E4, check_decode, gen, make_cache, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [3, 12])
@pytest.mark.parametrize("power", [126, 121, -110, -126])
def test_queries_at_the_ends_of_bf16_next_to_an_8_bit_cache(power, group):
    """Every finite query has a power of two that makes it f16: the largest, 2^128 less one step, and the smallest normal ones."""
    g = gen(13)
    table, pages = tables(g, [300, 17], 16)
    c = make_cache(g, pages, 16, 1, 64, E4, "nhd", (0.0625, 0.0625))
    lens = torch.tensor([300, 17], dtype=torch.int32, device="cuda")
    f = 2.0 ** power
    q = (torch.randn(2, group, 64, generator=g, device="cuda").clamp(-3.9, 3.9) * f).to(BF)
    if power == 126:
        q[0, 0, 5], q[1, 2, 63] = torch.finfo(BF).max, -torch.finfo(BF).max
    check_decode(c, q, table, lens, scale=0.25 / f)
    check_decode(c, q, table, lens, scale=0.25 / f, weight=False)
