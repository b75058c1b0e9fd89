"""The bound of codes_bound.py tells weights in fp16 from weights in bf16: the products emulated, no GPU."""
import pytest
import torch

from codes_bound import bound
from states_ref import F8


def emulate(p, scale, codes, weight_type):
    """out of a row whose weights p_j vs_j go through `weight_type` against a power of two above the largest scale."""
    unit = 2.0 ** torch.ceil(torch.log2(scale.max()))
    w = (p * scale / unit * 128).float().to(weight_type).to(F8)
    return ((w[:, None] * codes).sum(0) * unit / 128 / p.sum()).to(torch.bfloat16).to(F8)


@pytest.mark.parametrize("bits", [3, 4, 8])
def test_weights_of_fewer_bits_are_told_apart(bits):
    g = torch.Generator().manual_seed(bits)
    outside = {torch.float16: 0, torch.bfloat16: 0}
    for _ in range(200):
        n = int(torch.randint(2, 12, (), generator=g))
        p = torch.exp(2 * torch.randn(n, generator=g, dtype=F8))
        p = p / p.max()
        scale = 0.5 + torch.rand(n, generator=g, dtype=F8)
        codes = torch.randint(1 - 2 ** (bits - 1), 2 ** (bits - 1), (n, 64), generator=g).to(F8)
        v = scale[:, None] * codes
        ref, A = (p[:, None] * v).sum(0) / p.sum(), (p[:, None] * v.abs()).sum(0) / p.sum()
        tol = bound(ref, A, 2.0 ** -20, n, v.abs().max())
        for t in outside:
            outside[t] += int(((emulate(p, scale, codes, t) - ref).abs() > tol).sum())
    assert outside[torch.float16] == 0
    assert outside[torch.bfloat16] > 200                        # of 12800 elements
