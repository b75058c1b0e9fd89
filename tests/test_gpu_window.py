"""Attention within a window, with first tokens that stay visible, against a 64-bit evaluation (window_ref.py)."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, check_attention, fill, heads, make_batch
from window_ref import check_window, visible, window64

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


STEPS = [  # q_lens, kv_lens, window, sinks: decoding steps
    ([1], [1], 1, 0),
    ([1, 1, 1], [16, 17, 33], 1, 0),
    ([1, 1, 1], [63, 64, 65], 16, 1),
    ([1, 0, 1, 1], [300, 100, 0, 1], 17, 4),                                  # no query; no token at all
    ([1, 1], [5000, 3], 100, 16),
    ([2, 1, 3], [2, 129, 1000], 64, 17),
    ([2, 1], [40, 700], 30, 5),                                               # the sinks within the window for one sequence
    ([1, 1], [3000, 2049], 2048, 0),
    ([3, 1], [2, 50], 5, 2),                                                  # more queries than tokens: a row sees nothing
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("lens", range(len(STEPS)))
@pytest.mark.parametrize("H,KH,D,page", [(4, 4, 128, 64), (8, 2, 64, 16), (7, 1, 128, 32), (2, 2, 256, 16)])
def test_decoding_steps(bits, lens, H, KH, D, page):
    q_lens, kv_lens, window, sinks = STEPS[lens]
    cache, batch, tables, q, slots = setup(1100 + lens, q_lens, kv_lens, H, KH, D, bits, page, bos=bits < 8 and lens % 2 == 0)
    check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)


CHUNKS = [  # q_lens, kv_lens, window, sinks
    ([17], [17], 1, 0),
    ([64, 1], [64, 200], 16, 3),
    ([127, 128, 129], [127, 500, 129], 33, 1),
    ([257], [1030], 130, 40),
    ([300, 0, 5, 40], [300, 7, 700, 41], 64, 4),
    ([40], [30], 7, 2),                                                       # more queries than tokens: the first rows see nothing
    ([600], [600], 128, 0),
    ([520], [2100], 500, 130),
    ([200, 300], [1400, 340], 250, 200),                                      # more sinks than a tile has keys
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("lens", range(len(CHUNKS)))
@pytest.mark.parametrize("H,KH,D,page", [(2, 2, 128, 64), (8, 2, 64, 16), (5, 1, 128, 128), (2, 1, 256, 32)])
def test_chunks(bits, lens, H, KH, D, page):
    q_lens, kv_lens, window, sinks = CHUNKS[lens]
    cache, batch, tables, q, slots = setup(2100 + lens, q_lens, kv_lens, H, KH, D, bits, page, bos=bits < 8 and lens % 2 == 1)
    check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [900, 70]), ([150, 3], [900, 64])])
def test_every_border_of_window_and_sinks(bits, q_lens, kv_lens):
    """The groups of 16 keys in which a window begins and the sinks end, in all positions to each other."""
    cache, batch, tables, q, slots = setup(3100, q_lens, kv_lens, 4, 2, 64, bits, 16, bos=bits == 4)
    for window in (1, 15, 16, 31, 32, 33, 47, 128, 129, 899, 900):
        for sinks in (0, 1, 15, 16, 17, 64, 127, 128, 129):
            check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)


@pytest.mark.parametrize("bits", [3, 16])
def test_long_windows_are_split_and_joined(bits):
    q_lens, kv_lens = [1, 1, 20], [40_000, 130, 9_001]
    cache, batch, tables, q, slots = setup(41, q_lens, kv_lens, 4, 2, 128, bits, 64, bos=bits == 3)
    assert hbl.hbl_attention_window_workspace_bytes(cache, batch, 4, 8000, 100) > 0
    a = check_window(cache, batch, tables, q_lens, kv_lens, q, 8000, 100, slots=slots)
    # with a bound far above the lengths, and one below them, the pieces fall differently and the result holds
    for bound in (1 << 20, 256):
        other = hbl.KvBatch(batch.q_start, batch.kv_len, batch.pages, tokens=batch.tokens, max_q_len=20, max_kv_len=bound, bos_slot=batch.bos_slot)
        check_window(cache, other, tables, q_lens, kv_lens, q, 8000, 100, slots=slots)
    # the same call gives the same bits
    c = check_window(cache, batch, tables, q_lens, kv_lens, q, 8000, 100, slots=slots)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_len", [1, 90])
def test_a_window_over_everything_is_the_whole_attention(bits, q_len):
    q_lens, kv_lens = [q_len, 1], [q_len + 300, 40]
    cache, batch, tables, q, slots = setup(43, q_lens, kv_lens, 4, 2, 128, bits, 32, bos=bits == 4)
    want = hbl.hbl_attention(cache, batch, q)
    for window, sinks in ((1 << 30, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert torch.equal(hbl.hbl_attention_window(cache, batch, q, window, sinks)[:q_len + 1], want[:q_len + 1])
    for window, sinks in ((q_len + 300, 0), ((1 << 30) - 1, 7), (1, q_len + 300), (1, 2 ** 31 - 1)):
        check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)
    check_attention(cache, batch, tables, q_lens, kv_lens, q, slots=slots)


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("q_len", [1, 140])
@pytest.mark.parametrize("sinks", [0, 4, 40])
def test_what_no_row_sees_does_not_matter(bits, q_len, sinks):
    """Pages that hold nothing that a row sees are nobody's; unseen tokens of the others hold what is not finite."""
    q_lens, kv_lens, window, page = [q_len, 1], [q_len + 470, 321], 70, 32
    cache, batch, tables, q, slots = setup(61, q_lens, kv_lens, 4, 2, 128, bits, page, bos=bits < 8)
    want = check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)
    live = torch.zeros(cache.n_pages, page, dtype=torch.bool, device="cuda")
    given_away = 0
    for b, (ids, nq, nk) in enumerate(zip(tables, q_lens, kv_lens)):
        seen = visible(nq, nk, window, sinks).any(0).tolist()
        for i, x in enumerate(ids):
            mine = seen[i * page:(i + 1) * page]
            if any(mine):
                live[x, :len(mine)] = torch.tensor(mine, device="cuda")
            else:
                batch.pages[b, i] = (-3, 1 << 30)[given_away % 2]
                given_away += 1
    assert given_away > 8
    if bits < 8 and sinks == 0:
        batch.bos_slot.fill_(1 << 20)                                         # nobody sees a first token
    dead = (~live)[:, None].expand(-1, 2, -1)
    for x in (cache.k, cache.v):
        x[dead] = float("nan") if bits == 16 else 255
    for x in (cache.k_scale, cache.v_scale):
        if x is not None:
            x[dead] = float("inf")
    got = check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("q_len", [7, 200])
@pytest.mark.parametrize("which", ["key", "value"])
def test_what_is_not_finite_reaches_the_rows_that_see_it_and_no_others(bits, q_len, which):
    window, sinks = 5, 2
    q_lens, kv_lens = [q_len], [q_len + 40]
    cache, batch, tables, q, _ = setup(62, q_lens, kv_lens, 2, 2, 64, bits, 16, extra=0)
    clean = hbl.hbl_attention_window(cache, batch, q, window, sinks)
    at = kv_lens[0] - 6
    pg, sl = tables[0][at // 16], at % 16
    if bits == 16:
        (cache.k if which == "key" else cache.v)[pg, :, sl] = float("nan")
    else:
        (cache.k_scale if which == "key" else cache.v_scale)[pg, :, sl] = float("nan")
    out = hbl.hbl_attention_window(cache, batch, q, window, sinks)
    sees = visible(q_len, kv_lens[0], window, sinks)[:, at]
    assert 0 < sees.sum() < q_len
    assert torch.isnan(out[sees]).all()
    assert torch.equal(out[~sees], clean[~sees])


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("bits,D", [(16, 64), (16, 128), (16, 256), (8, 128), (4, 256)])
def test_each_key_of_a_tile_with_a_value_that_is_not_finite(bits, D, window):
    """Sequence b's key b has one: the rows that see it become NaN or infinite there, and no others."""
    n, page, sinks = 150, 32, 3
    cache, batch, tables, q, _ = setup(63, [n] * n, [n] * n, 1, 1, D, bits, page, extra=0)

    def run():
        return hbl.hbl_attention_window(cache, batch, q, window, sinks) if window else hbl.hbl_attention(cache, batch, q)
    clean = run()
    for b in range(n):
        at = tables[b][b // page], 0, b % page
        if bits == 16:
            cache.v[(*at, b * 7 % D)] = [float("nan"), float("inf"), -float("inf")][b % 3]
        else:
            cache.v_scale[at] = [float("nan"), float("inf")][b % 2]
    out = run()
    seen = visible(n, n, window, sinks) if window else torch.ones(n, n, device="cuda").tril().bool()
    sees = seen.T.reshape(n * n)                                             # row r of sequence b: does it see key b
    assert (~torch.isfinite(out[sees])).any(-1).all()
    assert torch.equal(out[~sees], clean[~sees])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("q_len", [1, 60])
def test_a_large_scale_outside_the_window_does_not_coarsen_the_weights(bits, q_len):
    """The value scale of a key that no row sees is not what the weights are held against."""
    q_lens, kv_lens, window, sinks = [q_len], [q_len + 100], 21, 3
    cache, batch, tables, q, _ = setup(63, q_lens, kv_lens, 2, 2, 64, bits, 16)
    dead = ~visible(q_len, kv_lens[0], window, sinks).any(0)
    pos = torch.arange(kv_lens[0], device="cuda")[dead]
    cache.v_scale[torch.tensor(tables[0], device="cuda")[pos // 16], :, pos % 16] = 1e30
    check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks)


@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("q_len", [1, 5, 150])
def test_extreme_scores(bits, q_len):
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
        check_window(cache, batch, tables, q_lens, kv_lens, q, 200, 20, sm_scale=1.0 if kind == "huge" else 0.5)


@pytest.mark.parametrize("scale", [0.0, -0.3])
@pytest.mark.parametrize("q_len", [1, 90])
def test_scales_of_zero_and_below(scale, q_len):
    for bits in (4, 16):
        cache, batch, tables, q, _ = setup(52, [q_len], [q_len + 90], 4, 2, 64, bits, 16)
        check_window(cache, batch, tables, [q_len], [q_len + 90], q, 37, 3, sm_scale=scale)


def test_many_sequences():
    g = gen(17)
    kv_lens = torch.randint(1, 700, (150,), device="cuda", generator=g).tolist()
    q_lens = [1 + (i % 3 == 0) * (i % 40) for i in range(150)]
    kv_lens = [max(a, b) for a, b in zip(q_lens, kv_lens)]
    cache, batch, tables, q, _ = setup(18, q_lens, kv_lens, 4, 1, 64, 8, 16)
    check_window(cache, batch, tables, q_lens, kv_lens, q, 90, 4)


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("H,KH,D", [(4, 2, 64), (2, 2, 128), (2, 1, 256)])
def test_chunks_of_a_large_batch(bits, H, KH, D):
    """So many of them, and such a window, that even short chunks are no longer dealt with 16 rows at a time."""
    q_lens = [17 + (7 * i) % 100 for i in range(60)]
    kv_lens = [q + 600 + (97 * i) % 2500 for i, q in enumerate(q_lens)]
    cache, batch, tables, q, slots = setup(19, q_lens, kv_lens, H, KH, D, bits, 32, bos=bits < 8)
    check_window(cache, batch, tables, q_lens, kv_lens, q, 2100, 20, slots=slots)
    check_window(cache, batch, tables, q_lens, kv_lens, q, 130, 3, slots=slots)


def test_strided_queries_and_outputs():
    q_lens, kv_lens = [1, 30], [90, 31]
    cache, batch, tables, q, _ = setup(71, q_lens, kv_lens, 4, 2, 128, 4, 32, extra=0)
    want = hbl.hbl_attention_window(cache, batch, q, 20, 4)
    fused = torch.zeros(31, 8, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:6] = q
    big = torch.full((31, 9, 136), 5.0, dtype=torch.bfloat16, device="cuda")
    hbl.hbl_attention_window(cache, batch, fused[:, 2:6], 20, 4, out=big[:, 1:5, :128])
    assert torch.equal(big[:, 1:5, :128], want)
    big[:, 1:5, :128] = 5.0
    assert (big == 5.0).all()


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("q_len", [1, 100])
@pytest.mark.parametrize("what", ["page", "length", "negative length", "start", "slot"])
def test_bad_indexes_are_reported_and_nothing_behind_them_is_read(bits, q_len, what):
    if what == "slot" and bits == 16:
        pytest.skip("no 8-bit first tokens at 16 bits")
    q_lens, kv_lens = [q_len, 1], [q_len + 60, 33]
    cache, batch, tables, q, slots = setup(95, q_lens, kv_lens, 2, 2, 64, bits, 16, bos=bits == 4)
    good = hbl.hbl_attention_window(cache, batch, q, 20, 4)
    if what == "page":
        batch.pages[0, (q_len + 59) // 16] = 1 << 30
    elif what == "length":
        batch.kv_len[0] = 2_000_000_000
    elif what == "negative length":
        batch.kv_len[0] = -5
    elif what == "start":
        batch.q_start[2] = 10_000
    else:
        batch.bos_slot[0] = 77
    out = hbl.hbl_attention_window(cache, batch, q, 20, 4)
    assert hbl.hbl_check_status() == 12
    assert hbl.hbl_check_status() == 0
    other = slice(0, q_len) if what == "start" else slice(q_len, q_len + 1)       # the other sequence is not touched by it
    assert torch.equal(out[other], good[other])


def test_a_captured_step_follows_the_cache():
    q_lens, kv_lens = [1, 1], [100, 2000]
    cache, batch, tables, q, _ = setup(97, q_lens, kv_lens, 4, 2, 128, 4, 64, extra=0, max_pages=40)
    batch.pages[:, :] = torch.arange(80, dtype=torch.int32, device="cuda").reshape(2, 40) % cache.n_pages
    tables = batch.pages.tolist()
    batch.c.max_kv_len = 2500
    ws = hbl.new_workspace(hbl.hbl_attention_window_workspace_bytes(cache, batch, 4, 900, 4))
    q2 = heads(gen(98), 2, 4, 128)
    outs = [torch.empty_like(q), torch.empty_like(q)]
    graphs = []
    for x, o in zip((q, q2), outs):
        hbl.hbl_attention_window(cache, batch, x, 900, 4, out=o, workspace=ws)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            hbl.hbl_attention_window(cache, batch, x, 900, 4, out=o, workspace=ws)
        graphs.append(gr)
    for _ in range(3):
        batch.kv_len.add_(150)
        ws.fill_(255)                                                         # whatever the workspace holds
        for gr in graphs:
            gr.replay()
        lens = batch.kv_len.tolist()
        for x, o in zip((q, q2), outs):
            ref, _, tol, _ = window64(cache, x, q_lens, lens, tables, 900, 4)
            assert ((o.to(F8) - ref).abs() <= tol).all()
    assert hbl.hbl_check_status() == 0


def test_another_stream():
    cache, batch, tables, q, _ = setup(99, [1, 60], [3000, 60], 4, 4, 128, 4, 64, extra=0)
    want = hbl.hbl_attention_window(cache, batch, q, 700, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hbl.hbl_attention_window(cache, batch, q, 700, 4)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("q_len", [1, 33])
def test_offsets_beyond_32_bits(q_len):
    """A cache of more than 2^31 values, the sequence's pages at its far end."""
    page, KH, D = 128, 8, 128
    n_pages = (1 << 31) // (page * KH * D) + 40
    cache = hbl.KvCache(*(torch.empty(n_pages, KH, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)), bits=16)
    g = gen(81)
    kv, ids = 500, [n_pages - 1, -9, n_pages - 17, n_pages - 2]
    for x in (cache.k, cache.v):
        x[n_pages - 20:] = torch.randn(20, KH, page, D, device="cuda", generator=g)
    batch = hbl.KvBatch(torch.tensor([0, q_len], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda"),
                        torch.tensor([ids], dtype=torch.int32, device="cuda"), tokens=q_len, max_q_len=q_len, max_kv_len=kv)
    check_window(cache, batch, [ids], [q_len], [kv], heads(g, q_len, KH, D), 130, 3)
