"""What the binding refuses of an attention call before anything is launched."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, heads, make_batch

pytestmark = pytest.mark.gpu


def test_a_workspace_that_the_gpu_cannot_use():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    cache = hbl.KvCache.empty(64, 64, 2, 64, 4)
    fill(g, cache)
    batch, _ = make_batch(g, cache, [1], [4000])
    q = heads(g, 1, 2, 64)
    size = hbl.hbl_attention_workspace_bytes(cache, batch, 2)
    assert size > 0
    want = hbl.hbl_attention(cache, batch, q)
    launches = hbl.hbl_launch_count()
    for ws in (torch.empty(size + 1024, dtype=torch.uint8), torch.empty(size + 1024, dtype=torch.uint8).pin_memory(),
               hbl.new_workspace(4 * size)[::2]):
        with pytest.raises(ValueError):
            hbl.hbl_attention(cache, batch, q, workspace=ws)
    with pytest.raises(hbl.HblError) as short:
        hbl.hbl_attention(cache, batch, q, workspace=hbl.new_workspace(size - 1024))
    assert short.value.status == 6
    assert hbl.hbl_launch_count() == launches
    assert torch.equal(hbl.hbl_attention(cache, batch, q, workspace=hbl.new_workspace(size)), want)
    assert hbl.hbl_check_status() == 0
