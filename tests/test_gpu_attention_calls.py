"""Attention over the paged cache, called as the documentation allows and nobody thinks of first: odd scales, many
sequences, wide groups, pieces of both kernels in one call, calls behind calls, graphs, streams."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import check_attention, fill, heads, make_batch

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def setup(seed, q_lens, kv_lens, H, KH, D, bits, page, slots=False, extra=0):
    g = gen(seed)
    n = len(q_lens)
    cache = hbl.KvCache.empty(sum(-(-x // page) for x in kv_lens) + 2, page, KH, D, bits, n if slots else 0)
    fill(g, cache)
    batch, tables = make_batch(g, cache, q_lens, kv_lens, extra_rows=extra, slots=list(range(n)) if slots else None)
    return cache, batch, tables, heads(g, sum(q_lens) + extra, H, D)


@pytest.mark.parametrize("bits", [3, 8, 16])
@pytest.mark.parametrize("q_len", [1, 70])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-6, 3.0])
def test_any_finite_scale(bits, q_len, scale):
    cache, batch, tables, q = setup(1, [q_len], [q_len + 90], 4, 2, 64, bits, 16)
    check_attention(cache, batch, tables, [q_len], [q_len + 90], q, sm_scale=scale)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("n", [33, 75, 1100])
def test_many_sequences_of_every_kind(bits, n):
    q_lens = [(0, 1, 1, 2, 5, 40, 1)[i % 7] if n < 1000 else (1, 6)[i % 2] for i in range(n)]
    kv_lens = [q + (0, 3, 17, 100, 0, 250, 31)[(i * 3) % 7] for i, q in enumerate(q_lens)]
    cache, batch, tables, q = setup(2, q_lens, kv_lens, 4, 1, 64, bits, 16, slots=bits == 4, extra=5)
    check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=list(range(n)) if bits == 4 else None)


@pytest.mark.parametrize("bits", [3, 16])
@pytest.mark.parametrize("group", [3, 16, 17, 32, 300])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [200, 31]), ([3, 1], [40, 500])])
def test_wide_groups(bits, group, q_lens, kv_lens):
    cache, batch, tables, q = setup(3, q_lens, kv_lens, group, 1, 64, bits, 32)
    check_attention(cache, batch, tables, q_lens, kv_lens, q)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_both_kernels_split_in_one_call(bits, D):
    q_lens, kv_lens = [40, 1, 300, 3], [5_000, 30_000, 9_000, 2_000]
    cache, batch, tables, q = setup(4, q_lens, kv_lens, 2, 1, D, bits, 64)
    a = check_attention(cache, batch, tables, q_lens, kv_lens, q)
    b = check_attention(cache, batch, tables, q_lens, kv_lens, q)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_workspace_grows_with_what_is_split_and_not_with_the_prompt():
    """A prompt among decoding steps: only the steps' rows wait in the workspace."""
    cache, batch, tables, q = setup(5, [2000, 1, 1], [2000, 1500, 1800], 32, 32, 128, 4, 64)
    size = hbl.hbl_attention_workspace_bytes(cache, batch, 32)
    assert 0 < size < 16 << 20
    check_attention(cache, batch, tables, [2000, 1, 1], [2000, 1500, 1800], q)


@pytest.mark.parametrize("T", [1, 16, 300])
def test_the_next_projection_reads_what_this_call_wrote(T):
    """W_o's layer behind the attention, its launch chosen by the library: the same as with everything waited for in between."""
    H, D, hidden = 16, 128, 2048
    cache, batch, tables, q = setup(6, [T], [T + 400], H, H, D, 4, 64)
    W, alpha = hbl.hbl_quantize_weights(torch.randn(hidden, hidden, device="cuda", generator=gen(7)) * 0.02)
    qs = [heads(gen(8 + i), T, H, D) for i in range(4)]
    out = torch.empty_like(q)
    ws = hbl.new_workspace(hbl.hbl_workspace_bytes(T, hidden, hidden))
    scratch = hbl.new_workspace(max(1, hbl.hbl_attention_workspace_bytes(cache, batch, H)))
    want = []
    for x in qs:
        hbl.hbl_attention(cache, batch, x, out=out, workspace=scratch)
        torch.cuda.synchronize()
        want.append(hbl.hbl_forward(out.view(T, hidden), W, alpha, hidden, 4, True, workspace=ws))
        torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for x in qs:
            hbl.hbl_attention(cache, batch, x, out=out, workspace=scratch)
            got.append(hbl.hbl_forward(out.view(T, hidden), W, alpha, hidden, 4, True, workspace=ws))
    torch.cuda.synchronize()
    assert hbl.hbl_check_status() == 0
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 4])


def test_a_captured_block_step_is_the_eager_one():
    """q, k, v -> append -> attention -> W_o in one graph, replayed while the sequences grow."""
    H, D, hidden, n = 16, 128, 2048, 3
    g = gen(9)
    W = {m: hbl.hbl_quantize_weights(torch.randn(hidden, hidden, device="cuda", generator=g) * 0.02) for m in "qkvo"}
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), 512)
    caches = [hbl.KvCache.empty(24, 64, H, D, 4, n) for _ in range(2)]
    pages = torch.randperm(24, device="cuda", generator=g).to(torch.int32).reshape(n, 8)
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    lens = torch.tensor([0, 100, 60], dtype=torch.int32, device="cuda")
    batch = hbl.KvBatch(start, lens, pages, tokens=n, max_q_len=1, max_kv_len=512)
    x = torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda")
    ws = hbl.new_workspace(hbl.hbl_workspace_bytes(n, hidden, hidden))
    scratch = hbl.new_workspace(max(1, hbl.hbl_attention_workspace_bytes(caches[0], batch, H)))
    ys = [torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    proj = {m: torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda") for m in "qkv"}
    o = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")

    def step(cache, y):
        for m in "qkv":
            hbl.hbl_forward(x, *W[m], hidden, 4, False, y=proj[m], workspace=ws)
        q, k, v = (proj[m].view(n, H, D) for m in "qkv")
        hbl.hbl_kv_append(cache, batch, k, v, table=table, q=q, q_out=q)
        hbl.hbl_attention(cache, batch, q, out=o, workspace=scratch)
        hbl.hbl_forward(o.view(n, hidden), *W["o"], hidden, 4, True, y=y, workspace=ws)

    x.normal_(generator=g)
    lens.add_(1)
    for i in range(2):
        step(caches[i], ys[i])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], ys[0])
    for _ in range(6):
        x.normal_(generator=g)
        lens.add_(1)
        graph.replay()
        step(caches[1], ys[1])
        torch.cuda.synchronize()
        assert torch.equal(ys[0], ys[1])
    for a in ("k", "v", "k_scale", "v_scale", "bos_k", "bos_v", "bos_k_scale", "bos_v_scale"):
        assert torch.equal(getattr(caches[0], a), getattr(caches[1], a))
    assert hbl.hbl_check_status() == 0


def test_two_streams_at_once():
    cache, batch, tables, q = setup(10, [1, 200], [6000, 900], 8, 4, 128, 4, 64)
    q2 = heads(gen(11), 201, 8, 128)
    want = [hbl.hbl_attention(cache, batch, x) for x in (q, q2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, x in zip(streams, (q, q2)):
            with torch.cuda.stream(s):
                got.append(hbl.hbl_attention(cache, batch, x))                 # (each its own workspace)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_len,group", [(2, 1), (6, 2), (200, 1), (130, 3)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("back", [1, 2, 40])
def test_a_value_that_is_not_finite_reaches_only_rows_that_see_it(D, q_len, group, what, back):
    """bf16 rows: one element of a value among the call's own tokens; the rows before it are as without it."""
    if back > q_len:
        back = q_len
    kv = q_len + 37
    cache, batch, tables, q = setup(12, [q_len], [kv], 2 * group, 2, D, 16, 16)
    clean = hbl.hbl_attention(cache, batch, q)
    n = kv - back
    cache.v[tables[0][n // 16], 1, n % 16, D // 2 + 3] = what
    out = hbl.hbl_attention(cache, batch, q)
    first = q_len - back                                                       # the first token that sees it
    assert torch.equal(out[:first], clean[:first])
    assert torch.equal(out[:, :group], clean[:, :group])                       # the other key head
    assert not torch.isfinite(out[first:, group:, D // 2 + 3]).any()
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("n,q", [(40, 1), (65, 2), (128, 1), (70, 40)])
def test_batches_of_several_rounds_whatever_the_order_of_their_lengths(bits, n, q):
    """More blocks than fit on the GPU at once: long sequences are taken first, and each exactly once."""
    rnd = torch.Generator().manual_seed(n)
    kv_lens = torch.randint(1, 1500, (n,), generator=rnd).tolist()
    kv_lens[3], kv_lens[n - 1], kv_lens[n // 2], kv_lens[7] = 0, 1500, 1500, 1
    q_lens = [q if i % 9 == 2 else 0 if i % 11 == 5 else 1 for i in range(n)]
    q_lens[3] = 0
    kv_lens = [max(a, b) for a, b in zip(q_lens, kv_lens)]
    cache, batch, tables, x = setup(n + bits, q_lens, kv_lens, 32, 16, 64, bits, 64, slots=bits < 8, extra=2)
    check_attention(cache, batch, tables, q_lens, kv_lens, x, slots=list(range(n)) if bits < 8 else None)


def test_a_length_that_makes_no_sense_harms_no_other_sequence():
    n, kv_lens = 64, [(1100, 40, 700, 1300)[i % 4] for i in range(64)]
    cache, batch, tables, q = setup(9, [1] * n, kv_lens, 16, 16, 64, 4, 64)
    good = hbl.hbl_attention(cache, batch, q)
    batch.kv_len[5], batch.kv_len[40] = -3, -2 ** 31
    out = hbl.hbl_attention(cache, batch, q)
    assert hbl.hbl_check_status() == 12
    keep = [i for i in range(n) if i not in (5, 40)]
    assert torch.equal(out[keep], good[keep])
    batch.kv_len[5] = 2 ** 31 - 1                               # beyond its pages: what it has is used, and it is reported
    batch.kv_len[40] = kv_lens[40]
    out = hbl.hbl_attention(cache, batch, q)
    assert hbl.hbl_check_status() == 12
    keep = [i for i in range(n) if i != 5]
    assert torch.equal(out[keep], good[keep])


@pytest.mark.parametrize("q_lens,kv_lens", [([500, 1, 0, 1], [500, 20, 3, 1]), ([600, 1, 1, 2], [9000, 40, 30, 20]), ([1, 2, 600], [60, 50, 600])])
@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("graph", [False, True])
def test_a_call_of_both_kernels_is_complete_for_what_comes_next(q_lens, kv_lens, bits, graph):
    """The short sequences' kernel runs beside the long ones' and is done long before it; the next launch needs both."""
    cache, batch, tables, q = setup(5, q_lens, kv_lens, 8, 8, 128, bits, 64)
    n = sum(q_lens)
    table = hbl.hbl_rope_table([0.0] * 64, 1)                   # angle 0: the next launch of the library copies
    at = torch.zeros(n, dtype=torch.int32, device="cuda")
    want, _ = check_attention(cache, batch, tables, q_lens, kv_lens, q)
    size = hbl.hbl_attention_workspace_bytes(cache, batch, 8)
    ws = hbl.new_workspace(size, q.device) if size else None
    outs = [torch.empty_like(q) for _ in range(8)]
    copies, others = [torch.empty_like(q) for _ in range(8)], [torch.empty_like(q) for _ in range(8)]

    def run():
        for o, c, x in zip(outs, copies, others):
            o.zero_()
            hbl.hbl_attention(cache, batch, q, out=o, workspace=ws)
            hbl.hbl_rope(o, at, table, out=c)
            x.copy_(o)

    run()
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
    for _ in range(5):
        for x in copies + others:
            x.fill_(3.0)
        g.replay() if graph else run()
        for x in copies + others:
            assert torch.equal(x, want)
    assert hbl.hbl_check_status() == 0
