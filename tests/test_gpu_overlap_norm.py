"""Normalised heads, their gradients and attention within a window between layers whose contraction lets the next launch begin early."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, make_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,q_lens,kv_lens", [(3, [1, 1, 1], [900, 20, 300]), (61, [60, 1], [60, 5000]), (170, [170], [1400])])
@pytest.mark.parametrize("path", [hbl.PATH_STREAM_OVERLAP, hbl.PATH_AUTO])
def test_each_waits_for_what_the_other_writes(T, q_lens, kv_lens, path):
    """q, k, v of early-releasing layers -> norms in place -> append with norms -> attention -> W_o as another such layer, and the
    norms' gradients with W_o's output as the incoming one, over and over without a wait in between, against the same calls with
    everything waited for.  (3 and 61 tokens: the gains' gradients in one launch; 170: in two.)"""
    H, D, hidden = 16, 128, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    cache = hbl.KvCache.empty(sum(-(-n // 64) for n in kv_lens) + 2, 64, H, D, 4)
    fill(g, cache)
    batch, _ = make_batch(g, cache, q_lens, kv_lens)
    W = {m: hbl.hbl_quantize_weights(torch.randn(hidden, hidden, device="cuda", generator=g) * 0.02) for m in "qkvo"}
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), max(kv_lens))
    pos = torch.randint(0, max(kv_lens), (T,), device="cuda", generator=g, dtype=torch.int32)
    gains = [(1 + 0.3 * torch.randn(D, device="cuda", generator=g)).bfloat16() for _ in range(2)]
    xs = [torch.randn(T, hidden, device="cuda", generator=g).bfloat16() for _ in range(4)]
    ws = [hbl.new_workspace(hbl.hbl_workspace_bytes(T, hidden, hidden)) for _ in range(2)]
    scratch = hbl.new_workspace(max(1, hbl.hbl_attention_window_workspace_bytes(cache, batch, H, 700, 4)))
    sums = hbl.new_workspace(hbl.hbl_norm_rope_grad_workspace_bytes(T, H, H, D))
    proj = {m: torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda") for m in "qkv"}
    o, keep = (torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step(x, y, path, wait):
        for m in "qkv":
            hbl.hbl_forward(x, *W[m], hidden, 4, False, y=proj[m], workspace=ws[0], path=path)
            wait()
        q, k, v = (proj[m].view(T, H, D) for m in "qkv")
        hbl.hbl_norm_rope(q, gains[0], pos, table, k=k, k_gain=gains[1], q_out=keep, k_out=k)
        wait()
        hbl.hbl_kv_append_norm(cache, batch, k, v, gains[1], table=table, q=q, q_gain=gains[0], q_out=q)
        wait()
        hbl.hbl_attention_window(cache, batch, q, 700, 4, out=o, workspace=scratch)
        wait()
        hbl.hbl_forward(o.view(T, hidden), *W["o"], hidden, 4, True, y=y, workspace=ws[1], path=path)
        wait()
        d = hbl.hbl_norm_rope_grad(y.view(T, H, D), keep, gains[0], pos, table, grad_k=y.view(T, H, D), k=k, k_gain=gains[1], workspace=sums)
        wait()
        hbl.hbl_forward(d[0].view(T, hidden), *W["q"], hidden, 4, True, y=y, workspace=ws[1], path=path)
        wait()
        return *d, y

    def fresh():
        return torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda")

    want = [[t.clone() for t in step(x, fresh(), hbl.PATH_STREAM, torch.cuda.synchronize)] for x in xs]
    ys = [fresh() for _ in range(24)]
    got = [step(xs[i % 4], y, path, lambda: None) for i, y in enumerate(ys)]
    torch.cuda.synchronize()
    assert hbl.hbl_check_status() == 0
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(out, want[i % 4]))
