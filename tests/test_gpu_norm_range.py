"""Gradients of normalised heads over fp32's range: the forward pass takes them (its statistic is fp64), so does the backward pass.

Tolerances are check_backward's.  Its count for r (23 eps of the squares' chain, 14 of r) and for the sum's terms bounds the way that
large and small heads go as well: there r is off by one eps, a term x r u by 1 + 1 + 3 + 1, and the chain is as long.  Gradients of heads
of 1e36 reach below the least normal number of fp32 and bf16, 2^-126: half a step is 2^-134 = 4.6e-41 there for bf16, 2^-150 for fp32,
below the 1e-40 that is there.  Products with elements of the smallest heads stay normal down to 1e-10 of a head's size."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import heads
from test_gpu_norm_rope import BF16, F32, check_backward, check_forward, gain_of, gen, table_of

pytestmark = pytest.mark.gpu

# sizes of heads side by side: both ends, both sides of what fp32 squares hold, ordinary ones in between
SIZES = [1e30, 1.0, 1e-28, 3e19, 1e-19, 2.0 ** 30, 2.0 ** -30, 1e9, 3e-10, 1e5, 1e-6, 1e36, 1e-22]


def sized(g, T, H, D, dtype):
    size = torch.tensor(SIZES, device="cuda", dtype=torch.float64)
    x = torch.randn(T, H, D, device="cuda", generator=g).double()
    return (x * size[(torch.arange(T, device="cuda")[:, None] + torch.arange(H, device="cuda")) % len(SIZES)][..., None]).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30])
@pytest.mark.parametrize("T,H,KH,D,rot", [(1, 3, 0, 128, 128), (26, 7, 2, 64, 32), (300, 9, 4, 80, 80), (70, 5, 3, 72, 0), (40, 4, 4, 256, 64), (1501, 32, 7, 128, 128),
                                          (2100, 24, 9, 64, 64)])
def test_heads_of_every_size(dtype, interleaved, eps, T, H, KH, D, rot):
    g = gen(T + D)
    table = table_of(rot, 500) if rot else None
    pos = torch.randint(0, 500, (T,), device="cuda", generator=g, dtype=torch.int32) if rot else None
    x = [sized(g, T, n, D, dtype) for n in (H, KH) if n]
    dy = [torch.randn(*a.shape, device="cuda", generator=g).to(dtype) for a in x]
    gains = [gain_of(g, D, BF16) for _ in x]
    second = dict(k=x[1], k_gain=gains[1]) if KH else {}
    y = hbl.hbl_norm_rope(x[0], gains[0], pos, table, norm_eps=eps, interleaved=interleaved, **second)
    d = hbl.hbl_norm_rope_grad(dy[0], x[0], gains[0], pos, table, norm_eps=eps, interleaved=interleaved, **second, **(dict(grad_k=dy[1]) if KH else {}))
    e32 = torch.tensor(eps, dtype=F32).double().item()                        # what the call is given
    for i in range(len(x)):
        check_forward(y[i], x[i], gains[i], table, pos, e32, interleaved)
        check_backward(d[2 * i:2 * i + 2], dy[i], x[i], gains[i], table, pos, e32, interleaved)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_is_beside_them_stays_as_it_is(dtype):
    """An ordinary head's gradient has the same bits whatever lies next to it; heads that are not finite, or zeros without an eps,
    are not numbers, and no others."""
    g = gen(3)
    T, H, D = 40, 8, 64
    x, dy = heads(g, T, H, D).to(dtype), torch.randn(T, H, D, device="cuda", generator=g).to(dtype)
    clean, _, _, _ = hbl.hbl_norm_rope_grad(dy, x, None, None, None, norm_eps=0.0)
    odd = torch.rand(T, H, device="cuda", generator=g) < 0.3
    other = x.clone()
    other[odd] = other[odd] * 1e25
    got, _, _, _ = hbl.hbl_norm_rope_grad(dy, other, None, None, None, norm_eps=0.0)
    assert torch.equal(got[~odd], clean[~odd])
    for bad in (float("nan"), float("inf"), 0.0):
        other = x.clone()
        if bad == 0.0:
            other[odd] = 0.0
        else:
            other[..., 5][odd] = bad
        got, _, _, _ = hbl.hbl_norm_rope_grad(dy, other, None, None, None, norm_eps=0.0)
        assert torch.isnan(got[odd]).all() and torch.equal(got[~odd], clean[~odd])
    got, dg, _, _ = hbl.hbl_norm_rope_grad(dy, torch.zeros_like(x), None, None, None, norm_eps=2.0 ** -20)
    assert torch.equal(got, dy * 2.0 ** 10) and (dg == 0).all()               # r = 2^10
