"""A row number in q_start that makes no sense: reported, and the sequences it does not belong to are computed all the same."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, heads, make_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("start", [1_000_000, -7])
def test_sequences_with_sound_starts_are_whole(bits, start):
    """The rows that a senseless pair of starts would have must not take the place of another sequence's."""
    q_lens, kv_lens = [20, 20, 20, 580], [50, 60, 70, 580]
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    cache = hbl.KvCache.empty(60, 16, 2, 64, bits)
    fill(g, cache)
    batch, _ = make_batch(g, cache, q_lens, kv_lens)
    q = heads(g, 640, 2, 64)
    good = hbl.hbl_attention(cache, batch, q)
    batch.q_start[2] = start                                                  # the end of sequence 1 and the start of sequence 2
    out = hbl.hbl_attention(cache, batch, q, out=torch.full_like(q, 5.0))
    assert hbl.hbl_check_status() == 12 and hbl.hbl_check_status() == 0
    assert torch.equal(out[:20], good[:20]) and torch.equal(out[60:], good[60:])
    assert (out[20:60] == 5).all()


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("start,end", [(0, 10_000), (-3, 100), (100, 0)])
def test_a_single_sequence_without_sound_starts_is_reported(bits, start, end):
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    cache = hbl.KvCache.empty(20, 16, 2, 64, bits)
    fill(g, cache)
    batch, _ = make_batch(g, cache, [100], [150])
    q = heads(g, 100, 2, 64)
    batch.q_start.copy_(torch.tensor([start, end], dtype=torch.int32))
    out = hbl.hbl_attention(cache, batch, q, out=torch.full_like(q, 5.0))
    assert hbl.hbl_check_status() == 12 and hbl.hbl_check_status() == 0
    assert (out == 5).all()
