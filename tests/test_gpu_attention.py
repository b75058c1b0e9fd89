"""Attention over the paged cache against a 64-bit evaluation (states_ref.py derives the tolerances)."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, attention64, check_attention, fill, heads, make_batch

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def setup(seed, q_lens, kv_lens, H, KH, D, bits, page, bos=False, extra=2, **kw):
    g = gen(seed)
    n = len(q_lens)
    cache = hbl.KvCache.empty(sum(-(-x // page) for x in kv_lens) + 2, page, KH, D, bits, n + 1 if bos else 0)
    fill(g, cache)
    slots = [(i + 1) % (n + 1) for i in range(n)] if bos else None
    batch, tables = make_batch(g, cache, q_lens, kv_lens, extra_rows=extra, slots=slots, **kw)
    q = heads(g, sum(q_lens) + extra, H, D)
    return cache, batch, tables, q, slots


STEPS = [  # q_lens, kv_lens: decoding steps
    ([1], [1]),
    ([1], [16]),
    ([1], [17]),
    ([1, 1, 1], [63, 64, 65]),
    ([1, 0, 1, 1], [300, 100, 0, 1]),                                         # no query; no token at all
    ([1, 1], [5000, 3]),
    ([2, 1, 3], [2, 129, 1000]),
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("lens", range(len(STEPS)))
@pytest.mark.parametrize("H,KH,D,page", [(4, 4, 128, 64), (8, 2, 64, 16), (7, 1, 128, 32), (2, 2, 256, 16)])
def test_decoding_steps(bits, lens, H, KH, D, page):
    q_lens, kv_lens = STEPS[lens]
    cache, batch, tables, q, slots = setup(1000 + lens, q_lens, kv_lens, H, KH, D, bits, page, bos=bits < 8 and lens % 2 == 0)
    check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=slots)


CHUNKS = [  # q_lens, kv_lens
    ([16], [16]),
    ([17], [17]),
    ([64, 1], [64, 200]),
    ([127, 128, 129], [127, 500, 129]),
    ([257], [1030]),
    ([300, 0, 5, 40], [300, 7, 700, 41]),
    ([40], [30]),                                                             # more queries than tokens: the first rows see nothing
    ([600], [600]),
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("lens", range(len(CHUNKS)))
@pytest.mark.parametrize("H,KH,D,page", [(2, 2, 128, 64), (8, 2, 64, 16), (5, 1, 128, 128), (2, 1, 256, 32)])
def test_chunks(bits, lens, H, KH, D, page):
    q_lens, kv_lens = CHUNKS[lens]
    cache, batch, tables, q, slots = setup(2000 + lens, q_lens, kv_lens, H, KH, D, bits, page, bos=bits < 8 and lens % 2 == 1)
    check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=slots)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [40, 700]), ([130, 3], [130, 64]), ([50], [20])])
def test_without_the_causal_mask(bits, q_lens, kv_lens):
    cache, batch, tables, q, slots = setup(31, q_lens, kv_lens, 4, 2, 128, bits, 32)
    check_attention(cache, batch, tables, q_lens, kv_lens, q, causal=False)


@pytest.mark.parametrize("bits", [3, 16])
def test_long_context_is_split_and_joined(bits):
    q_lens, kv_lens = [1, 1, 20], [40_000, 130, 9_001]
    cache, batch, tables, q, slots = setup(41, q_lens, kv_lens, 4, 2, 128, bits, 64, bos=bits == 3)
    assert hbl.hbl_attention_workspace_bytes(cache, batch, 4) > 0
    a = check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=slots)
    # with a bound far above the lengths, and one below them, the pieces fall differently and the result holds
    for bound in (1 << 20, 256):
        other = hbl.KvBatch(batch.q_start, batch.kv_len, batch.pages, tokens=batch.tokens, max_q_len=20, max_kv_len=bound, bos_slot=batch.bos_slot)
        b = check_attention(cache, other, tables, q_lens, kv_lens, q, slots=slots)
        assert (a[0].float() - b[0].float()).abs().max() < 0.05
    # the same call gives the same bits
    c = check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=slots)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("q_len", [1, 5, 150])
def test_extreme_scores(bits, q_len):
    """Scores that grow along the keys (the running maximum rises all the way), fall, and reach thousands."""
    q_lens, kv_lens = [q_len], [q_len + 500]
    for kind in ("rise", "fall", "huge"):
        cache, batch, tables, q, _ = setup(51, q_lens, kv_lens, 4, 2, 64, bits, 16)
        n = kv_lens[0]
        pos = torch.arange(n, device="cuda")
        ids = torch.tensor(tables[0], device="cuda")[pos // 16]
        ramp = (pos if kind == "rise" else n - pos).float() / n
        if bits == 16:
            x = (q[0, 0].float() * (4 if kind == "huge" else 1) * ramp[:, None]).to(torch.bfloat16)
            cache.k[ids, :, pos % 16] = x[:, None]
        else:
            cache.k_scale[ids, :, pos % 16] = (ramp[:, None] + 0.01) * (20 if kind == "huge" else 2)
        check_attention(cache, batch, tables, q_lens, kv_lens, q, sm_scale=1.0 if kind == "huge" else 0.5)


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("q_len", [1, 140])
def test_what_lies_beyond_a_sequence_does_not_matter(bits, q_len):
    q_lens, kv_lens = [q_len, 1], [q_len + 70, 21]
    cache, batch, tables, q, _ = setup(61, q_lens, kv_lens, 4, 2, 128, bits, 32)
    want = check_attention(cache, batch, tables, q_lens, kv_lens, q)
    live = torch.zeros(cache.n_pages, cache.page_size, dtype=torch.bool, device="cuda")
    for ids, n in zip(tables, kv_lens):
        for p in range(n):
            live[ids[p // 32], p % 32] = True
    dead = (~live)[:, None].expand(-1, 2, -1)
    for x in (cache.k, cache.v):
        x[dead] = float("nan") if bits == 16 else 255
    for x in (cache.k_scale, cache.v_scale):
        if x is not None:
            x[dead] = float("nan")
    got = check_attention(cache, batch, tables, q_lens, kv_lens, q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_len", [6, 200])
def test_a_masked_key_or_scale_that_is_not_finite_reaches_no_row_it_is_masked_for(bits, q_len):
    """The last token's key (bits 16), its key and value (codes: the scale is NaN): only the last row sees them."""
    q_lens, kv_lens = [q_len], [q_len + 10]
    cache, batch, tables, q, _ = setup(62, q_lens, kv_lens, 2, 2, 64, bits, 16, extra=0)
    n = kv_lens[0] - 1
    pg, sl = tables[0][n // 16], n % 16
    out0 = hbl.hbl_attention(cache, batch, q)
    if bits == 16:
        cache.k[pg, :, sl] = float("nan")
    else:
        cache.k_scale[pg, :, sl] = float("nan")
        cache.v_scale[pg, :, sl] = float("inf")
    out = hbl.hbl_attention(cache, batch, q)
    assert torch.isnan(out[-1]).all()
    assert torch.equal(out[:-1], out0[:-1])


def test_strided_queries_and_outputs():
    q_lens, kv_lens = [1, 30], [90, 31]
    cache, batch, tables, q, _ = setup(71, q_lens, kv_lens, 4, 2, 128, 4, 32, extra=0)
    want = hbl.hbl_attention(cache, batch, q)
    fused = torch.zeros(31, 8, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:6] = q
    big = torch.full((31, 9, 136), 5.0, dtype=torch.bfloat16, device="cuda")
    hbl.hbl_attention(cache, batch, fused[:, 2:6], out=big[:, 1:5, :128])
    assert torch.equal(big[:, 1:5, :128], want)
    big[:, 1:5, :128] = 5.0
    assert (big == 5.0).all()


@pytest.mark.parametrize("q_len", [1, 33])
def test_offsets_beyond_32_bits(q_len):
    """A cache of more than 2^31 values, the sequence's pages at its far end."""
    page, KH, D = 128, 8, 128
    n_pages = (1 << 31) // (page * KH * D) + 40
    k = torch.empty(n_pages, KH, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(n_pages, KH, page, D, dtype=torch.bfloat16, device="cuda")
    cache = hbl.KvCache(k, v, bits=16)
    g = gen(81)
    kv = 300
    ids = [n_pages - 1, n_pages - 17, n_pages - 2]
    k[n_pages - 20:], v[n_pages - 20:] = torch.randn(20, KH, page, D, device="cuda", generator=g), torch.randn(20, KH, page, D, device="cuda", generator=g)
    batch = hbl.KvBatch(torch.tensor([0, q_len], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda"),
                        torch.tensor([ids], dtype=torch.int32, device="cuda"), tokens=q_len, max_q_len=q_len, max_kv_len=kv)
    new = heads(g, q_len, KH, D)
    hbl.hbl_kv_append(cache, batch, new, new)
    check_attention(cache, batch, [ids], [q_len], [kv], heads(g, q_len, KH, D))
    ko, vo = hbl.hbl_kv_read(cache, batch)
    assert torch.equal(ko, new) and torch.equal(vo, new)


def test_a_prefix_may_be_shared():
    cache, batch, tables, q, _ = setup(91, [1, 1, 1], [64, 64, 40], 4, 2, 64, 4, 16)
    batch.pages[1, :2] = batch.pages[0, :2]
    batch.pages[2, :3] = batch.pages[0, :3]
    tables[1][:2], tables[2] = tables[0][:2], tables[0][:3]
    check_attention(cache, batch, tables, [1, 1, 1], [64, 64, 40], q)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_len", [1, 100])
@pytest.mark.parametrize("what", ["page", "length", "negative length", "start", "slot"])
def test_bad_indexes_are_reported_and_nothing_behind_them_is_read(bits, q_len, what):
    if what == "slot" and bits == 16:
        pytest.skip("no 8-bit first tokens at 16 bits")
    q_lens, kv_lens = [q_len, 1], [q_len + 60, 33]
    cache, batch, tables, q, slots = setup(95, q_lens, kv_lens, 2, 2, 64, bits, 16, bos=bits == 4)
    good = hbl.hbl_attention(cache, batch, q)
    if what == "page":
        batch.pages[0, 1] = 1 << 30
    elif what == "length":
        batch.kv_len[0] = 2_000_000_000
    elif what == "negative length":
        batch.kv_len[0] = -5
    elif what == "start":
        batch.q_start[2] = 10_000
    else:
        batch.bos_slot[0] = 77
    out = hbl.hbl_attention(cache, batch, q)
    assert hbl.hbl_check_status() == 12
    assert hbl.hbl_check_status() == 0
    other = slice(0, q_len) if what == "start" else slice(q_len, q_len + 1)       # the other sequence is not touched by it
    assert torch.equal(out[other], good[other])


def test_rows_beyond_the_bound_are_left_out():
    cache, batch, tables, q, _ = setup(96, [10], [50], 2, 2, 64, 4, 16, extra=0)
    want = hbl.hbl_attention(cache, batch, q)
    short = hbl.KvBatch(batch.q_start, batch.kv_len, batch.pages, tokens=10, max_q_len=4, max_kv_len=50)
    out = torch.full_like(q, 8.0)
    hbl.hbl_attention(cache, short, q, out=out)
    assert torch.equal(out[:4], want[:4]) and (out[4:] == 8).all()
    assert hbl.hbl_check_status() == 0


def test_a_captured_step_follows_the_cache_and_two_graphs_share_a_workspace():
    q_lens, kv_lens = [1, 1], [100, 2000]
    cache, batch, tables, q, _ = setup(97, q_lens, kv_lens, 4, 2, 128, 4, 64, extra=0, max_pages=40)
    batch.pages[:, :] = torch.arange(80, dtype=torch.int32, device="cuda").reshape(2, 40) % cache.n_pages
    tables = batch.pages.tolist()
    batch.c.max_kv_len = 2500
    ws = hbl.new_workspace(hbl.hbl_attention_workspace_bytes(cache, batch, 4))
    q2 = heads(gen(98), 2, 4, 128)
    outs = [torch.empty_like(q), torch.empty_like(q)]
    for x, o in zip((q, q2), outs):
        hbl.hbl_attention(cache, batch, x, out=o, workspace=ws)
    graphs = []
    for x, o in zip((q, q2), outs):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            hbl.hbl_attention(cache, batch, x, out=o, workspace=ws)
        graphs.append(gr)
    for step in range(3):
        batch.kv_len.add_(150)
        ws.fill_(255)                                                         # whatever the workspace holds
        for gr in graphs:
            gr.replay()
        lens = batch.kv_len.tolist()
        for x, o in zip((q, q2), outs):
            ref, _, tol, _ = attention64(cache, x, q_lens, lens, tables, 128 ** -0.5, True)
            assert ((o.to(F8) - ref).abs() <= tol).all()
    assert hbl.hbl_check_status() == 0


def test_another_stream():
    cache, batch, tables, q, _ = setup(99, [1, 60], [3000, 60], 4, 4, 128, 4, 64, extra=0)
    want = hbl.hbl_attention(cache, batch, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hbl.hbl_attention(cache, batch, q)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("bits,T", [(4, 1), (16, 1), (3, 40), (16, 200)])
def test_from_projections_to_the_input_of_w_o(bits, T):
    """The calls together as a decoder block makes them: the block's q, k, v; append with rotation; attention; W_o."""
    g = gen(7 + T)
    hidden, ffn, H, D = 2048, 8192, 16, 128
    weights, alphas = {}, []
    for n, (o, i) in dict(q=(hidden, hidden), k=(hidden, hidden), v=(hidden, hidden), o=(hidden, hidden), up=(ffn, hidden), gate=(ffn, hidden),
                          down=(hidden, ffn)).items():
        weights[n], a = hbl.hbl_quantize_weights(torch.randn(o, i, device="cuda", generator=g) * 0.02)
        alphas.append(a)
    alpha7 = torch.cat(alphas)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), 1024)
    page, past = 64, 150
    cache = hbl.KvCache.empty(16, page, H, D, bits, 2 if bits < 8 else 0)
    pages = torch.randperm(16, device="cuda", generator=g).to(torch.int32).reshape(2, 8)
    tables = pages.tolist()
    lens = [0, 0]
    for n in (past, T):                                                       # a prompt, then a step or a chunk
        q_lens = [n, n]
        lens = [x + n for x in lens]
        start = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        batch = hbl.KvBatch(start, torch.tensor(lens, dtype=torch.int32, device="cuda"), pages, tokens=2 * n, max_q_len=n, max_kv_len=max(lens))
        x = torch.randn(2 * n, hidden, device="cuda", generator=g).to(torch.bfloat16)
        mid = torch.randn(2 * n, ffn, device="cuda", generator=g).to(torch.bfloat16)
        y = hbl.hbl_block_forward(dict(attn_in=x, o_in=x, ffn_in=x, down_in=mid), weights, alpha7, hidden, ffn, 4)
        q, k, v = (y[c].view(2 * n, H, D) for c in "qkv")
        raw_q = q.clone()
        hbl.hbl_kv_append(cache, batch, k, v, table=table, q=q, q_out=q)
        pos = torch.cat([torch.arange(m - n, m, dtype=torch.int32, device="cuda") for m in lens])
        assert torch.equal(q, hbl.hbl_rope(raw_q, pos, table))
        # the attention of what the cache holds, and the next projection on its output
        out, _ = check_attention(cache, batch, tables, q_lens, lens, q, slots=[0, 1] if bits < 8 else None)
        z = hbl.hbl_forward(out.view(2 * n, hidden), weights["o"], alphas[3], hidden, 4, True)
        assert hbl.hbl_check_status() == 0 and torch.isfinite(z).all()
        if bits == 16:                                                        # and of the projections themselves
            ko, vo = hbl.hbl_kv_read(cache, batch)
            assert torch.equal(vo, v) and torch.equal(ko, hbl.hbl_rope(k.contiguous(), pos, table))
