"""Cache and attention calls between layers whose contraction lets the next launch begin early, on one stream."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, heads, make_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("T,q_lens,kv_lens", [(3, [1, 1, 1], [900, 20, 300]), (40, [40], [700]), (61, [60, 1], [60, 5000])])
@pytest.mark.parametrize("path", [hbl.PATH_STREAM_OVERLAP, hbl.PATH_AUTO])
def test_each_waits_for_what_the_other_writes(bits, T, q_lens, kv_lens, path):
    """q, k, v of early-releasing layers -> append -> attention -> W_o as another such layer, over and over without a wait in
    between, against the same calls with everything waited for."""
    H, D, hidden = 16, 128, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(T + bits)
    cache = hbl.KvCache.empty(sum(-(-n // 64) for n in kv_lens) + 2, 64, H, D, bits)
    fill(g, cache)
    batch, _ = make_batch(g, cache, q_lens, kv_lens)
    W = {m: hbl.hbl_quantize_weights(torch.randn(hidden, hidden, device="cuda", generator=g) * 0.02) for m in "qkvo"}
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), max(kv_lens))
    xs = [torch.randn(T, hidden, device="cuda", generator=g).bfloat16() for _ in range(4)]
    ws = [hbl.new_workspace(hbl.hbl_workspace_bytes(T, hidden, hidden)) for _ in range(2)]
    scratch = hbl.new_workspace(max(1, hbl.hbl_attention_workspace_bytes(cache, batch, H)))
    proj = {m: torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda") for m in "qkv"}
    o = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")

    def step(x, y, path, wait):
        for m in "qkv":
            hbl.hbl_forward(x, *W[m], hidden, 4, False, y=proj[m], workspace=ws[0], path=path)
            wait()
        q, k, v = (proj[m].view(T, H, D) for m in "qkv")
        hbl.hbl_kv_append(cache, batch, k, v, table=table, q=q, q_out=q)
        wait()
        hbl.hbl_attention(cache, batch, q, out=o, workspace=scratch)
        wait()
        hbl.hbl_forward(o.view(T, hidden), *W["o"], hidden, 4, True, y=y, workspace=ws[1], path=path)
        wait()

    want = []
    for x in xs:
        y = torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda")
        step(x, y, hbl.PATH_STREAM, torch.cuda.synchronize)
        want.append((y, o.clone()))
    ys = [torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda") for _ in range(40)]
    for i, y in enumerate(ys):
        step(xs[i % 4], y, path, lambda: None)
    torch.cuda.synchronize()
    assert hbl.hbl_check_status() == 0
    assert torch.equal(o, want[3][1])
    for i, y in enumerate(ys):
        assert torch.equal(y, want[i % 4][0])
