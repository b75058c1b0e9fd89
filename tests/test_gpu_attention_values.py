"""Values and scales of a cache of codes that are not finite, or at the end of their range: whose rows they reach."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, heads, make_batch

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def setup(seed, q_lens, kv_lens, H, KH, D, bits, page):
    g = gen(seed)
    cache = hbl.KvCache.empty(sum(-(-x // page) for x in kv_lens) + 2, page, KH, D, bits)
    fill(g, cache)
    batch, tables = make_batch(g, cache, q_lens, kv_lens)
    return cache, batch, tables, heads(g, sum(q_lens), H, D)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("q_len", [100, 700])
def test_a_value_scale_that_is_not_finite_marks_the_rows_that_see_its_key_and_no_others(bits, q_len, D):
    """Every tile of keys brings its marks along; tiles with and without any take turns in every stage, and the key heads
    (more of them than blocks that run at once) each have their own."""
    H, page = 170, 64
    kv = q_len + 900
    cache, batch, tables, q = setup(1, [q_len], [kv], H, H, D, bits, page)
    cpu = torch.Generator().manual_seed(q_len)
    # the last key of a few tiles among the call's own tokens, another place for every head; every fourth head is clean
    first = torch.full((H,), q_len)
    for h in range(H):
        if h % 4 == 3:
            continue
        at = torch.randint(0, q_len, (3,), generator=cpu).tolist()
        for n in at:
            n += kv - q_len
            cache.v_scale[tables[0][n // page], h, n % page] = (float("nan"), float("inf"), -float("inf"))[n % 3]
        first[h] = min(at)
    for _ in range(3):
        out = hbl.hbl_attention(cache, batch, q)
        bad = torch.isnan(out).cpu()
        seen = torch.arange(q_len)[:, None] >= first[None]
        assert torch.equal(bad.all(-1), seen) and torch.equal(bad.any(-1), seen)
        assert torch.isfinite(out).cpu()[~seen].all()
    assert hbl.hbl_check_status() == 0
