"""Gradients of the gains added up within a call's one launch, at widths at which a warp's lanes take different numbers of elements."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import heads
from test_gpu_norm_rope import BF16, F32, check_backward, gain_of, gen, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,KH", [(1, 1, 0), (16, 5, 3), (40, 1, 7)])
@pytest.mark.parametrize("D,rot", [(8, 0), (24, 16), (40, 32), (72, 64), (88, 16), (104, 96), (136, 0), (200, 80), (248, 240), (160, 160)])
def test_widths_that_are_no_multiple_of_a_warp(dtype, T, H, KH, D, rot):
    g = gen(T * D)
    table = table_of(rot, 300) if rot else None
    pos = torch.randint(0, 300, (T,), device="cuda", generator=g, dtype=torch.int32) if rot else None
    x = [heads(g, T, n, D).to(dtype) for n in (H, KH) if n]
    dy = [torch.randn(*a.shape, device="cuda", generator=g).to(dtype) for a in x]
    gains = [gain_of(g, D, F32) for _ in x]
    second = dict(k=x[1], k_gain=gains[1], grad_k=dy[1]) if KH else {}
    before = hbl.hbl_launch_count()

    def call():
        return hbl.hbl_norm_rope_grad(dy[0], x[0], gains[0], pos, table, **second)

    first = call()
    assert hbl.hbl_launch_count() == before + 1
    for i in range(len(x)):
        check_backward(first[2 * i:2 * i + 2], dy[i], x[i], gains[i], table, pos, 1e-6, False)
    for _ in range(20):
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(first, call()))
    assert hbl.hbl_check_status() == 0
