"""Normalised and rotated heads and their gradients against the formulas in 64 bits.

eps here is 2^-24, half a step of fp32.  Forward: gain * x, the rotation's two products and its sum, the inverse root and the product
with it are rounded once each, so with S = r (|g x1 c| + |g x2 s|) an output is off by at most 3 eps S + 2 eps |o| <= 5 eps S; the
rounding to bf16 adds 2^-8 of the value.

Backward: t = R^T do is off by 2 eps T, T = |c do1| + |s do2|; u = g t by 3 eps gT.  A head's sums are chains of at most 16 + 5
additions: mean x^2 and so 1 / r^2 are off by 23 eps, r (root and division) by 14 eps; sum x u by 24 eps sum |x| g T; r^2 sum / D by
(24 + 28 + 4) eps of that; times x, subtracted, times r: dx = r u - r^3 x sum / D is off by (3 + 1 + 14 + 1) eps on the first term and
(56 + 1 + 1 + 14 + 1) eps on the second, so by less than 80 eps (r g T + r^3 |x| sum |x| g T / D).
dg: a term t x r is off by 18 eps T |x| r; a sum's chain is a thread's rows, 32 threads, and the blocks in 32 strands: below 400
additions at these sizes."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, heads, rotate64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def table_of(rot, n_pos, **kw):
    return hbl.hbl_rope_table(hbl.hbl_rope_frequencies(rot), n_pos, **kw)


def gain_of(g, D, dtype):
    return (1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(dtype)


def turn(x, table, pos, interleaved, backward=False):
    return x if table is None else rotate64(x, table, pos, interleaved, backward)


def sizes(x, table, pos, interleaved):
    """|c x1| + |s x2| (and more) of every element."""
    if table is None:
        return x.abs()
    t = table.abs()
    return rotate64(x.abs(), t * torch.tensor([1.0, -1.0], device="cuda"), pos, interleaved).abs() + rotate64(x.abs(), t, pos, interleaved).abs()


def forward64(x, gain, table, pos, eps, interleaved):
    r = 1 / (x.to(F8).square().mean(-1, keepdim=True) + eps).sqrt()
    z = x.to(F8) if gain is None else x.to(F8) * gain.to(F8)
    return r * turn(z, table, pos, interleaved), 1.01 * 5 * U * r * sizes(z, table, pos, interleaved)


def check_forward(y, x, gain, table, pos, eps, interleaved):
    ref, tol = forward64(x, gain, table, pos, eps, interleaved)
    tol = tol + (2.0 ** -8 * ref.abs() * 1.01 if y.dtype == BF16 else 0) + 1e-40
    err = (y.to(F8) - ref).abs()
    assert (err <= tol).all(), f"{(err / tol).max().item():.3f} of the tolerance"


def backward64(dy, x, gain, table, pos, eps, interleaved):
    """(dx, its tolerance, dg, its tolerance)"""
    z, D = x.to(F8), x.shape[-1]
    r = 1 / (z.square().mean(-1, keepdim=True) + eps).sqrt()
    g = torch.ones(D, dtype=F8, device="cuda") if gain is None else gain.to(F8)
    t, T = turn(dy.to(F8), table, pos, interleaved, True), sizes(dy.to(F8), table, pos, interleaved)
    u = g * t
    dx = r * (u - z * r * r * (z * u).mean(-1, keepdim=True))
    size = r * g.abs() * T + r ** 3 * z.abs() * (z.abs() * g.abs() * T).mean(-1, keepdim=True)
    return dx, 1.01 * 80 * U * size, (t * z * r).sum((0, 1)), 1.01 * (18 + 400) * U * (T * z.abs() * r).sum((0, 1)) + 1e-40


def check_backward(got, dy, x, gain, table, pos, eps, interleaved):
    dx, tol, dg, tol_g = backward64(dy, x, gain, table, pos, eps, interleaved)
    tol = tol + (2.0 ** -8 * dx.abs() * 1.01 if got[0].dtype == BF16 else 0) + 1e-40
    err = (got[0].to(F8) - dx).abs()
    assert (err <= tol).all(), f"dx: {(err / tol).max().item():.3f} of the tolerance"
    if got[1] is not None:
        err = (got[1].to(F8) - dg).abs()
        assert got[1].dtype == F32 and (err <= tol_g).all(), f"dg: {(err / tol_g).max().item():.3f} of the tolerance"


SHAPES = [  # T, H, KH, D, rot
    (1, 1, 0, 64, 64), (3, 7, 1, 128, 128), (17, 5, 5, 128, 48), (130, 32, 8, 128, 64), (5, 2, 1, 256, 256), (33, 3, 2, 80, 32), (9, 1, 1, 16, 16),
    (700, 32, 8, 128, 128), (21, 4, 2, 96, 96), (6, 3, 3, 8, 0), (40, 6, 2, 128, 0), (11, 2, 1, 256, 16), (900, 5, 9, 64, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gain", [BF16, F32, None])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,KH,D,rot", SHAPES)
def test_both_directions_match_the_formulas(dtype, gain, interleaved, T, H, KH, D, rot):
    g = gen(T + D)
    table = table_of(rot, 5000, amplitude=1.07) if rot else None
    pos = torch.randint(0, 5000, (T,), device="cuda", generator=g, dtype=torch.int32) if rot else None
    x = [heads(g, T, n, D).to(dtype) for n in (H, KH) if n]
    dy = [torch.randn(*a.shape, device="cuda", generator=g).to(dtype) for a in x]
    gains = [None if gain is None else gain_of(g, D, gain) for _ in x]
    second = dict(k=x[1], k_gain=gains[1]) if KH else {}
    y = hbl.hbl_norm_rope(x[0], gains[0], pos, table, norm_eps=2.0 ** -18, interleaved=interleaved, **second)
    d = hbl.hbl_norm_rope_grad(dy[0], x[0], gains[0], pos, table, norm_eps=2.0 ** -18, interleaved=interleaved, **second, **(dict(grad_k=dy[1]) if KH else {}))
    assert hbl.hbl_check_status() == 0
    assert (y[1] is None) == (d[2] is None) == (d[3] is None) == (KH == 0)
    for i in range(len(x)):
        assert y[i].dtype == d[2 * i].dtype == dtype
        check_forward(y[i], x[i], gains[i], table, pos, 2.0 ** -18, interleaved)
        check_backward(d[2 * i:2 * i + 2], dy[i], x[i], gains[i], table, pos, 2.0 ** -18, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_large_call(interleaved):
    """As many heads as several rounds of thread blocks take, of very different sizes; the same call gives the same bits."""
    g = gen(5)
    T, H, KH, D = 4096, 24, 8, 128
    table = table_of(D, 4096)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    q, k = heads(g, T, H, D), (heads(g, T, KH, D).float() * torch.logspace(-6, 6, T, device="cuda")[:, None, None]).to(BF16)
    gq, gk = gain_of(g, D, BF16), gain_of(g, D, BF16)
    y = hbl.hbl_norm_rope(q, gq, pos, table, k=k, k_gain=gk, norm_eps=2.0 ** -20, interleaved=interleaved)
    dq, dk = (torch.randn(*a.shape, device="cuda", generator=g).to(BF16) for a in (q, k))
    d = hbl.hbl_norm_rope_grad(dq, q, gq, pos, table, grad_k=dk, k=k, k_gain=gk, norm_eps=2.0 ** -20, interleaved=interleaved)
    for a, b, c, e, f in ((y[0], q, gq, dq, d[:2]), (y[1], k, gk, dk, d[2:])):
        check_forward(a, b, c, table, pos, 2.0 ** -20, interleaved)
        check_backward(f, e, b, c, table, pos, 2.0 ** -20, interleaved)
    again = hbl.hbl_norm_rope_grad(dq, q, gq, pos, table, grad_k=dk, k=k, k_gain=gk, norm_eps=2.0 ** -20, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(d, again))
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,KH,D,rot", [(1501, 32, 7, 128, 64), (2100, 40, 9, 64, 64), (1001, 23, 1, 256, 128), (3001, 15, 9, 96, 48), (6000, 9, 9, 80, 80)])
def test_calls_of_several_heads_to_a_thread(dtype, interleaved, T, H, KH, D, rot):
    """More heads than places for them, numbers that are no multiples of what a thread takes, every width of lanes."""
    g = gen(T)
    table = table_of(rot, 3000)
    pos = torch.randint(0, 3000, (T,), device="cuda", generator=g, dtype=torch.int32)
    fused = heads(g, T, H + KH, D).to(dtype)
    q, k = fused[:, :H], fused[:, H:]
    dy = torch.randn(T, H + KH, D, device="cuda", generator=g).to(dtype)
    gq, gk = gain_of(g, D, BF16), gain_of(g, D, BF16)
    y = hbl.hbl_norm_rope(q, gq, pos, table, k=k, k_gain=gk, interleaved=interleaved)
    d = hbl.hbl_norm_rope_grad(dy[:, :H], q, gq, pos, table, grad_k=dy[:, H:], k=k, k_gain=gk, interleaved=interleaved)
    assert hbl.hbl_check_status() == 0
    for x, w, gain, out, dx in ((q, dy[:, :H], gq, y[0], d[:2]), (k, dy[:, H:], gk, y[1], d[2:])):
        check_forward(out, x, gain, table, pos, 1e-6, interleaved)
        check_backward(dx, w, x, gain, table, pos, 1e-6, interleaved)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_forward_is_the_fp32_evaluation_bit_for_bit(dtype, interleaved):
    g = gen(3)
    table = table_of(128, 1000)
    x, gain = heads(g, 64, 8, 128).float(), gain_of(g, 128, dtype)
    pos = torch.randint(0, 1000, (64,), device="cuda", generator=g, dtype=torch.int32)
    y, _ = hbl.hbl_norm_rope(x, gain, pos, table, norm_eps=2.0 ** -20, interleaved=interleaved)
    r = (1 / (x.double().square().mean(-1, keepdim=True) + 2.0 ** -20).sqrt()).float()
    z = x * gain.float()
    c, s = table[pos.long()][:, None].unbind(-1)
    a, b = (z[..., 0::2], z[..., 1::2]) if interleaved else z.chunk(2, -1)
    ya, yb = (y[..., 0::2], y[..., 1::2]) if interleaved else y.chunk(2, -1)
    assert torch.equal(ya, (a * c - b * s) * r) and torch.equal(yb, (b * c + a * s) * r)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 32, 64])
def test_gradients_are_those_of_differences(interleaved, rot):
    """Along a direction v in x and one in the gain: (L(x + h v) - L(x - h v)) / 2h of the formula in 64 bits, L = sum w o.  Along x
    an output is (a + b t) / sqrt(q(t)) in units of a head's size: its third derivative is below 50 |w| S |v|^3 / |x|^3, and h^2 / 6 = 2e-11
    of that is far below fp32's roundings; 64 bits lose 1e-16 / h = 1e-11 of sum |w| S.  L is linear in the gain."""
    g = gen(8)
    T, H, D, h, eps = 4, 3, 64, 1e-5, 2.0 ** -10
    table = table_of(rot, 50) if rot else None
    pos = torch.randint(0, 50, (T,), device="cuda", generator=g, dtype=torch.int32) if rot else None
    x, w, v = (torch.randn(T, H, D, device="cuda", generator=g) for _ in range(3))
    gain, vg = gain_of(g, D, F32), torch.randn(D, device="cuda", generator=g)
    dx, dg, _, _ = hbl.hbl_norm_rope_grad(w, x, gain, pos, table, norm_eps=eps, interleaved=interleaved)

    def loss(at, a_gain):
        return (w.to(F8) * forward64(at, a_gain, table, pos, eps, interleaved)[0]).sum()

    _, tol, _, tol_g = backward64(w, x, gain, table, pos, eps, interleaved)
    size = (w.to(F8).abs() * forward64(x, gain, table, pos, eps, interleaved)[1]).sum() / (5 * U)
    along = (loss(x.to(F8) + h * v, gain) - loss(x.to(F8) - h * v, gain)) / (2 * h)
    assert ((dx.to(F8) * v).sum() - along).abs() <= (tol * v.abs()).sum() + 1e-8 * size
    along = (loss(x, gain.to(F8) + h * vg) - loss(x, gain.to(F8) - h * vg)) / (2 * h)
    assert ((dg.to(F8) * vg).sum() - along).abs() <= (tol_g * vg.abs()).sum() + 1e-8 * size


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 64])
def test_in_place_and_strided(interleaved, rot):
    g = gen(4)
    table = table_of(rot, 100)
    T, H, KH, D = 37, 6, 2, 128
    fused = heads(g, T, H + 2 * KH, D)                                        # q | k | v of one projection
    keep = fused.clone()
    pos = torch.randint(0, 100, (T,), device="cuda", generator=g, dtype=torch.int32)
    gq, gk = gain_of(g, D, F32), gain_of(g, D, F32)
    q, k = fused[:, :H], fused[:, H:H + KH]
    want = hbl.hbl_norm_rope(q.contiguous(), gq, pos, table, k=k.contiguous(), k_gain=gk, interleaved=interleaved)
    grads = torch.randn(T, H + KH, D, device="cuda", generator=g).to(BF16)
    gkeep = grads.clone()
    want_d = hbl.hbl_norm_rope_grad(grads[:, :H].contiguous(), q.contiguous(), gq, pos, table, grad_k=grads[:, H:].contiguous(), k=k.contiguous(), k_gain=gk,
                                    interleaved=interleaved)
    # the gradients over the gradients, then over the inputs
    d = hbl.hbl_norm_rope_grad(grads[:, :H], q, gq, pos, table, grad_k=grads[:, H:], k=k, k_gain=gk, interleaved=interleaved, dq=grads[:, :H], dk=grads[:, H:])
    assert all(torch.equal(a, b) for a, b in zip(d, want_d)) and torch.equal(fused, keep)
    other = fused.clone()
    d = hbl.hbl_norm_rope_grad(gkeep[:, :H], other[:, :H], gq, pos, table, grad_k=gkeep[:, H:], k=other[:, H:H + KH], k_gain=gk, interleaved=interleaved,
                               dq=other[:, :H], dk=other[:, H:H + KH])
    assert all(torch.equal(a, b) for a, b in zip(d, want_d)) and torch.equal(other[:, H + KH:], keep[:, H + KH:])
    hbl.hbl_norm_rope(q, gq, pos, table, k=k, k_gain=gk, interleaved=interleaved, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, H + KH:], keep[:, H + KH:])
    big = torch.full((T, H + 1, D + 8), 5.0, dtype=BF16, device="cuda")        # heads apart, written
    hbl.hbl_norm_rope(keep[:, :H], gq, pos, table, interleaved=interleaved, q_out=big[:, 1:, :D])
    assert torch.equal(big[:, 1:, :D], want[0])
    big[:, 1:, :D] = 5.0
    assert (big == 5.0).all()


def test_broadcast_inputs_and_gradients():
    g = gen(6)
    T, H, D = 50, 4, 64
    table, pos = table_of(D, 64), torch.arange(50, dtype=torch.int32, device="cuda")
    row, dy = heads(g, 1, H, D), torch.randn(1, 1, D, device="cuda", generator=g).to(BF16)
    gain = gain_of(g, D, BF16)
    x, grad = row.expand(T, H, D), dy.expand(T, H, D)
    y, _ = hbl.hbl_norm_rope(x, gain, pos, table)
    assert torch.equal(y, hbl.hbl_norm_rope(x.contiguous(), gain, pos, table)[0])
    d, e = hbl.hbl_norm_rope_grad(grad, x, gain, pos, table), hbl.hbl_norm_rope_grad(grad.contiguous(), x.contiguous(), gain, pos, table)
    assert torch.equal(d[0], e[0]) and torch.equal(d[1], e[1])
    check_backward(d[:2], grad, x, gain, table, pos, 1e-6, False)


@pytest.mark.parametrize("T", [1, 3000])
def test_positions_out_of_range_are_reported_and_left_out(T):
    g = gen(9)
    D, H = 128, 4
    table = table_of(D, 10)
    x, dy = heads(g, T, H, D), torch.randn(T, H, D, device="cuda", generator=g).to(BF16)
    gain = gain_of(g, D, F32)
    pos = torch.randint(0, 10, (T,), device="cuda", generator=g, dtype=torch.int32)
    good = pos.clone()
    bad = torch.arange(0, T, 7, device="cuda")
    pos[bad] = torch.tensor([-1, 10, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")[bad % 4]
    y = torch.full_like(x, 3.0)
    hbl.hbl_norm_rope(x, gain, pos, table, q_out=y)
    assert hbl.hbl_check_status() == 12 and hbl.hbl_check_status() == 0
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert (y[bad] == 3).all() and torch.equal(y[keep], hbl.hbl_norm_rope(x, gain, good, table)[0][keep])
    dx = torch.full_like(x, 3.0)
    _, dg, _, _ = hbl.hbl_norm_rope_grad(dy, x, gain, pos, table, dq=dx)
    assert hbl.hbl_check_status() == 12
    assert (dx[bad] == 3).all()
    ref = backward64(dy[keep], x[keep], gain, table, good[keep], 1e-6, False)
    assert ((dg.to(F8) - ref[2]).abs() <= ref[3]).all()
    assert ((dx[keep].to(F8) - ref[0]).abs() <= ref[1] + 2.0 ** -8 * ref[0].abs() * 1.01).all()


def test_zeros_infinities_and_very_large_heads():
    g = gen(10)
    D = 128
    x = heads(g, 8, 1, D)
    x[0] = 0
    x[1, 0, 5] = float("nan")
    x[2, 0, 7] = float("inf")
    x[3] *= 1e30                                                              # squares beyond fp32
    x[4] *= 1e-30
    gain = gain_of(g, D, F32)
    y, _ = hbl.hbl_norm_rope(x, gain, None, None, norm_eps=1e-6)
    assert (y[0] == 0).all() and torch.isnan(y[1]).all()
    assert torch.isnan(y[2, 0, 7]) and (y[2, 0, :7] == 0).all()               # x r with r = 0
    rest = [3, 4, 5, 6, 7]
    check_forward(y[rest], x[rest], gain, None, None, 1e-6, False)
    y, _ = hbl.hbl_norm_rope(x[[0, 3, 4, 5]], gain, None, None, norm_eps=0.0)  # the statistic is fp64: no head is too small
    assert torch.isnan(y[0]).all()
    check_forward(y[1:], x[[3, 4, 5]], gain, None, None, 0.0, False)


def test_no_tokens_and_no_gain_gradients():
    D = 64
    e = torch.empty(0, 4, D, dtype=BF16, device="cuda")
    gain = torch.ones(D, device="cuda")
    y, _ = hbl.hbl_norm_rope(e, gain, None, None)
    assert y.shape == (0, 4, D)
    _, dg, _, dk = hbl.hbl_norm_rope_grad(e, e, gain, None, None, grad_k=e[:, :2], k=e[:, :2], k_gain=gain)
    assert (dg == 0).all() and (dk == 0).all()
    x = heads(gen(1), 5, 4, D)
    dy = heads(gen(2), 5, 4, D)
    a, b = hbl.hbl_norm_rope_grad(dy, x, gain, None, None, gain_grads=False), hbl.hbl_norm_rope_grad(dy, x, gain, None, None)
    assert a[1] is None and torch.equal(a[0], b[0])
    assert hbl.hbl_check_status() == 0


def test_captured_and_on_another_stream():
    g = gen(11)
    T, H, KH, D = 300, 8, 2, 128
    table, pos = table_of(D, 512), torch.randint(0, 512, (T,), device="cuda", generator=g, dtype=torch.int32)
    q, k = heads(g, T, H, D), heads(g, T, KH, D)
    gq, gk = gain_of(g, D, BF16), gain_of(g, D, BF16)
    ws = hbl.new_workspace(hbl.hbl_norm_rope_grad_workspace_bytes(T, H, KH, D))

    def both(workspace=None):
        y = hbl.hbl_norm_rope(q, gq, pos, table, k=k, k_gain=gk)
        return *y, *hbl.hbl_norm_rope_grad(*[y[0], q, gq, pos, table], grad_k=y[1], k=k, k_gain=gk, workspace=workspace)

    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(ws)
    q.copy_(heads(g, T, H, D))
    pos.copy_(torch.randint(0, 512, (T,), device="cuda", generator=g, dtype=torch.int32))
    for _ in range(3):
        ws.fill_(255)                                                         # whatever the workspace holds
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("T,H,KH", [(1, 1, 0), (9, 8, 2), (128, 8, 3), (129, 8, 3), (4, 300, 1)])
def test_small_gradients_captured_side_by_side(T, H, KH):
    """Calls that add up the gains' gradients within one launch, around the border to those that take two; two graphs on two streams."""
    g = gen(12)
    D = 128
    table = table_of(D, 512)
    sets = []
    for _ in range(2):
        pos = torch.randint(0, 512, (T,), device="cuda", generator=g, dtype=torch.int32)
        x, w = heads(g, T, H + KH, D), torch.randn(T, H + KH, D, device="cuda", generator=g).to(BF16)
        gains = [gain_of(g, D, BF16) for _ in range(2)]
        ws = hbl.new_workspace(hbl.hbl_norm_rope_grad_workspace_bytes(T, H, KH, D))
        kw = dict(k=x[:, H:], k_gain=gains[1], grad_k=w[:, H:]) if KH else {}

        def call(x=x, w=w, gains=gains, pos=pos, kw=kw, ws=ws):
            return hbl.hbl_norm_rope_grad(w[:, :H], x[:, :H], gains[0], pos, table, workspace=ws, **kw)

        want = call()
        check_backward(want[:2], w[:, :H], x[:, :H], gains[0], table, pos, 1e-6, False)
        if KH:
            check_backward(want[2:], w[:, H:], x[:, H:], gains[1], table, pos, 1e-6, False)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        sets.append((graph, got, want, torch.cuda.Stream(), call))             # (the call holds what the graph reads)
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, _, _, stream, _ in sets:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, got, want, _, _ in sets:
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got, want))
    assert hbl.hbl_check_status() == 0
