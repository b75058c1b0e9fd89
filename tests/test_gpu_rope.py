"""Rotary positions against the formula in 64 bits, their backward pass, and their table.

A product or sum in fp32 is off by at most 2^-24 of its value: an output of two products and a sum by at most
3 * 2^-24 (|c x1| + |s x2|); the rounding to bf16 adds 2^-8 of the value."""
import math

import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, heads, rotate64

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def table_of(rot, n_pos, **kw):
    return hbl.hbl_rope_table(hbl.hbl_rope_frequencies(rot), n_pos, **kw)


def check(y, x, table, pos, interleaved=False, backward=False):
    ref = rotate64(x, table, pos, interleaved, backward)
    size = rotate64(x.abs(), table.abs() * torch.tensor([1.0, -1.0], device="cuda"), pos, interleaved).abs() + \
        rotate64(x.abs(), table.abs(), pos, interleaved).abs()              # at least |c x1| + |s x2|
    tol = 3 * 2.0 ** -24 * size + (2.0 ** -8 * ref.abs() * 1.01 if y.dtype == torch.bfloat16 else 0)
    assert ((y.to(F8) - ref).abs() <= tol + 1e-40).all()


@pytest.mark.parametrize("first,amplitude", [(0, 1.0), (1_000_000, 1.0), (131_000, 1.1386)])
def test_table_is_the_rounded_cosine_and_sine(first, amplitude):
    freq = hbl.hbl_rope_frequencies(128)
    t = hbl.hbl_rope_table(freq, 300, first_pos=first, amplitude=amplitude)
    angle = (first + torch.arange(300, dtype=F8, device="cuda"))[:, None] * torch.tensor(freq, dtype=F8, device="cuda")
    ref = amplitude * torch.stack([angle.cos(), angle.sin()], -1)
    assert hbl.hbl_check_status() == 0
    assert ((t.to(F8) - ref).abs() <= 2.0 ** -24 * ref.abs() * (1 + 1e-6) + 1e-15).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 64), (3, 7, 128, 128), (17, 5, 128, 48), (130, 32, 128, 64), (5, 2, 256, 256), (33, 3, 72, 32),
                                       (9, 1, 16, 16), (1100, 32, 128, 128)])
@pytest.mark.parametrize("backward", [False, True])
def test_rope_matches_the_formula(dtype, interleaved, T, H, D, rot, backward):
    g = gen(T + D)
    table = table_of(rot, 5000, amplitude=1.07)
    x = heads(g, T, H, D).to(dtype)
    pos = torch.randint(0, 5000, (T,), device="cuda", generator=g, dtype=torch.int32)
    y = hbl.hbl_rope(x, pos, table, interleaved=interleaved, backward=backward)
    assert hbl.hbl_check_status() == 0
    check(y, x, table, pos, interleaved, backward)
    assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_the_fp32_evaluation_bit_for_bit(interleaved):
    g = gen(3)
    table = table_of(128, 1000)
    x = heads(g, 64, 8, 128).float()
    pos = torch.randint(0, 1000, (64,), device="cuda", generator=g, dtype=torch.int32)
    y = hbl.hbl_rope(x, pos, table, interleaved=interleaved)
    c, s = table[pos.long()][:, None].unbind(-1)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    ya, yb = (y[..., 0::2], y[..., 1::2]) if interleaved else y.chunk(2, -1)
    assert torch.equal(ya, a * c - b * s) and torch.equal(yb, b * c + a * s)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 64])
def test_rope_in_place_and_strided(interleaved, rot):
    g = gen(4)
    table = table_of(rot, 100)
    T, H, D = 37, 6, 128
    fused = heads(g, T, 3 * H, D)                                           # q | k | v of one projection
    keep = fused.clone()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    k = fused[:, H:2 * H]
    want = hbl.hbl_rope(k.contiguous(), pos, table, interleaved=interleaved)
    assert torch.equal(hbl.hbl_rope(k, pos, table, interleaved=interleaved), want)
    by_head = keep[:, :H].transpose(0, 1).contiguous().transpose(0, 1)       # [T, H, D] with the heads outermost in memory
    assert torch.equal(hbl.hbl_rope(by_head, pos, table, interleaved=interleaved), hbl.hbl_rope(keep[:, :H].contiguous(), pos, table, interleaved=interleaved))
    hbl.hbl_rope(k, pos, table, interleaved=interleaved, out=k)
    assert hbl.hbl_check_status() == 0
    assert torch.equal(k, want)
    assert torch.equal(fused[:, :H], keep[:, :H]) and torch.equal(fused[:, 2 * H:], keep[:, 2 * H:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_backward_is_the_gradient(interleaved):
    """Of a loss sum(w * rope(x)): against the autograd of the formula in 64 bits, and against differences."""
    g = gen(5)
    table = table_of(64, 200_000, amplitude=0.9)
    T, H, D = 11, 3, 128
    x = heads(g, T, H, D).float()
    w = torch.randn(T, H, D, device="cuda", generator=g)
    pos = torch.randint(0, 200_000, (T,), device="cuda", generator=g, dtype=torch.int32)
    grad = hbl.hbl_rope(w, pos, table, interleaved=interleaved, backward=True)
    leaf = x.to(F8).requires_grad_()
    half = 32
    c, s = table[pos.long()].to(F8)[:, None].unbind(-1)
    a, b = (leaf[..., 0:64:2], leaf[..., 1:64:2]) if interleaved else (leaf[..., :half], leaf[..., half:64])
    wa, wb = (w[..., 0:64:2], w[..., 1:64:2]) if interleaved else (w[..., :half], w[..., half:64])
    ((a * c - b * s) * wa + (b * c + a * s) * wb).sum().add((leaf[..., 64:] * w[..., 64:]).sum()).backward()
    assert ((grad.to(F8) - leaf.grad).abs() <= 3 * 2.0 ** -24 * 2 * w.abs().amax()).all()
    # the map is linear: a difference of step 1 is its derivative, up to the roundings of two forward passes
    f = lambda z: (hbl.hbl_rope(z, pos, table, interleaved=interleaved).to(F8) * w.to(F8)).sum().item()
    for t, h, d in [(0, 0, 0), (3, 1, 33), (10, 2, 63), (5, 0, 100)]:
        e = torch.zeros_like(x)
        e[t, h, d] = 1.0
        assert abs(f(e) - f(torch.zeros_like(x)) - grad[t, h, d].item()) <= 1e-5
    # <R x, y> = <x, R^T y>
    y = hbl.hbl_rope(x, pos, table, interleaved=interleaved)
    size = (y.to(F8).abs() * w.abs()).sum() + (x.to(F8).abs() * grad.abs()).sum()
    assert abs((y.to(F8) * w).sum() - (x.to(F8) * grad).sum()) <= 3 * 2.0 ** -24 * 2 * size


def test_positions_out_of_range_are_reported_and_left_out():
    table = table_of(64, 10)
    x = heads(gen(6), 4, 2, 64)
    out = torch.full_like(x, 5.0)
    pos = torch.tensor([3, 10, -1, 9], dtype=torch.int32, device="cuda")
    hbl.hbl_rope(x, pos, table, out=out)
    assert hbl.hbl_check_status() == 12
    assert hbl.hbl_check_status() == 0
    assert (out[1:3] == 5).all()
    check(out[[0, 3]], x[[0, 3]], table, pos[[0, 3]])


def test_no_tokens_other_stream_and_graph():
    table = table_of(128, 64)
    empty = hbl.hbl_rope(torch.empty(0, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), table)
    assert empty.shape == (0, 4, 128)
    x = heads(gen(7), 20, 4, 128)
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    want = hbl.hbl_rope(x, pos, table)
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hbl.hbl_rope(x, pos, table, out=out)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hbl.hbl_rope(x, pos, table, out=out)
    pos.add_(3)
    x.mul_(2)
    graph.replay()
    check(out, x, table, pos)
