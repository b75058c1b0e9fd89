"""sm_scale far from the usual: tiny ones over large products, zero over products near the end of the range."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import check_attention, fill, heads, make_batch

pytestmark = pytest.mark.gpu


def setup(bits, q_len, up):
    """Queries and keys (their scales, over codes) that are 2^up times the usual."""
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    cache = hbl.KvCache.empty(20, 16, 2, 64, bits)
    fill(g, cache)
    kv = q_len + 80
    batch, tables = make_batch(g, cache, [q_len], [kv])
    q = heads(g, q_len, 4, 64) * 2.0 ** up
    (cache.k if bits == 16 else cache.k_scale).mul_(2.0 ** up)
    return cache, batch, tables, q, kv


@pytest.mark.parametrize("bits", [3, 8, 16])
@pytest.mark.parametrize("q_len", [1, 40])
@pytest.mark.parametrize("up", [30, 50, 56])
def test_a_tiny_scale_over_large_products(bits, q_len, up):
    """The scores are the usual ones: the factors of two cancel."""
    cache, batch, tables, q, kv = setup(bits, q_len, up)
    for sign in (1, -1):
        check_attention(cache, batch, tables, [q_len], [kv], q, sm_scale=sign * 2.0 ** (-2 * up - 3))


@pytest.mark.parametrize("bits", [3, 8, 16])
@pytest.mark.parametrize("q_len", [1, 40])
def test_a_scale_of_zero_over_large_products(bits, q_len):
    cache, batch, tables, q, kv = setup(bits, q_len, 56)
    check_attention(cache, batch, tables, [q_len], [kv], q, sm_scale=0.0)
