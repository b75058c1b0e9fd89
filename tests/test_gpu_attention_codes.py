"""Attention over codes within the bound that fp16 weights give (codes_bound.py), an eighth of what bf16 weights need."""
import pytest
import torch

from codes_bound import attention_codes64
from paper_2504_18415_b200 import hbl
from states_ref import F8, fill, heads, make_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_lens,kv_lens,H,KH", [
    ([1, 1, 1, 1], [2, 3, 5, 9], 4, 2),                        # few keys: a weight's rounding is not averaged out
    ([4, 2], [6, 300], 4, 1),
    ([40, 30], [41, 33], 2, 2),                                # the same on the tiles: early rows see few keys
    ([150], [700], 2, 1),
    ([1, 1], [9000, 40], 2, 2),                                # split and joined
    ([20], [5000], 2, 2),
])
@pytest.mark.parametrize("bos", [False, True])
def test_rounding_of_the_weights(bits, D, q_lens, kv_lens, H, KH, bos):
    if bos and bits == 8:
        pytest.skip("first tokens at 8 bits belong to caches of fewer")
    g = torch.Generator(device="cuda")
    g.manual_seed(bits * D + sum(kv_lens))
    n, page = len(q_lens), 16
    cache = hbl.KvCache.empty(sum(-(-x // page) for x in kv_lens) + 2, page, KH, D, bits, n if bos else 0)
    fill(g, cache)
    slots = list(range(n)) if bos else None
    batch, tables = make_batch(g, cache, q_lens, kv_lens, slots=slots)
    q = heads(g, sum(q_lens), H, D)
    for scale in (D ** -0.5, 0.02):                            # (a small one: many keys share the weight)
        out = hbl.hbl_attention(cache, batch, q, sm_scale=scale)
        ref, tol = attention_codes64(cache, q, q_lens, kv_lens, tables, scale, slots=slots)
        err = (out.to(F8) - ref).abs()
        assert (err <= tol).all(), f"{(err / tol).max().item():.3f} of the tolerance"
    assert hbl.hbl_check_status() == 0
