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


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("q_len,group", [(1, 1), (5, 2), (16, 1), (17, 1), (200, 1)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("back", [1, 3, 60, 400])
def test_a_value_scale_alone_that_is_not_finite(bits, q_len, group, what, back):
    """The keys' scales are sound: a row that sees the value is NaN in all its elements, whichever kernel computes it."""
    kv, page = q_len + 450, 16
    cache, batch, tables, q = setup(2, [q_len], [kv], 2 * group, 2, 64, bits, page)
    clean = hbl.hbl_attention(cache, batch, q)
    n = kv - back
    cache.v_scale[tables[0][n // page], 1, n % page] = what
    out = hbl.hbl_attention(cache, batch, q)
    first = max(0, q_len - back)                                              # the first token that sees it
    assert torch.isnan(out[first:, group:]).all()
    assert torch.equal(out[:first], clean[:first]) and torch.equal(out[:, :group], clean[:, :group])
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("q_len", [1, 40])
def test_a_first_token_whose_value_scale_is_not_finite(bits, q_len):
    kv = q_len + 90
    g = gen(3)
    cache = hbl.KvCache.empty(12, 16, 2, 64, bits, 2)
    fill(g, cache)
    batch, _ = make_batch(g, cache, [q_len], [kv], slots=[1])
    q = heads(g, q_len, 2, 64)
    clean = hbl.hbl_attention(cache, batch, q)
    cache.bos_v_scale[1, 0] = float("inf")
    out = hbl.hbl_attention(cache, batch, q)
    assert torch.isnan(out[:, 0]).all() and torch.equal(out[:, 1], clean[:, 1])
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("q_len", [1, 6, 17, 300])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("back", [1, 5, 250])
def test_a_bf16_value_that_is_not_finite(q_len, what, back):
    """Its element is not finite in a row that sees it; the row's other elements are as without it, or the whole row is NaN."""
    kv, D, e = q_len + 280, 128, 37
    cache, batch, tables, q = setup(4, [q_len], [kv], 2, 2, D, 16, 32)
    clean = hbl.hbl_attention(cache, batch, q)
    n = kv - back
    cache.v[tables[0][n // 32], 1, n % 32, e] = what
    out = hbl.hbl_attention(cache, batch, q)
    first = max(0, q_len - back)
    assert torch.equal(out[:first], clean[:first]) and torch.equal(out[:, 0], clean[:, 0])
    rows, was = out[first:, 1], clean[first:, 1]
    assert not torch.isfinite(rows[:, e]).any()
    other = torch.arange(D, device="cuda") != e
    assert (torch.isnan(rows).all(-1) | (rows == was)[:, other].all(-1)).all()
    assert hbl.hbl_check_status() == 0
