"""Attention within a window for sequences whose rows go to the tensor-core tiles: what test_gpu_window.py asks of short ones, and long
windows, whose keys are split.  References and tolerances: window_ref.py."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, heads
from test_gpu_window import gen, setup
from window_ref import check_window, visible, window64

pytestmark = pytest.mark.gpu
ROWS = 160                     # of a key head: more than the 128 that the streaming kernel takes at most


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("q_len", [ROWS, 300])
@pytest.mark.parametrize("H,KH,D", [(2, 2, 64), (2, 1, 128), (2, 2, 256)])
@pytest.mark.parametrize("sinks", [0, 3, 30])
def test_a_large_scale_outside_the_window_does_not_coarsen_the_weights(bits, q_len, H, KH, D, sinks):
    """Unseen keys of the groups of 16 that a window shares with seen ones; their scales are finite, but huge."""
    q_lens, kv_lens, window = [q_len], [q_len + 100], 21
    cache, batch, tables, q, _ = setup(63, q_lens, kv_lens, H, KH, D, bits, 16)
    dead = ~visible(q_len, kv_lens[0], window, sinks).any(0)
    pos = torch.arange(kv_lens[0], device="cuda")[dead]
    assert len(pos) > 40
    cache.v_scale[torch.tensor(tables[0], device="cuda")[pos // 16], :, pos % 16] = 1e30
    check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("what", ["page", "length", "negative length", "start", "slot"])
@pytest.mark.parametrize("n", [1, 2])
def test_bad_indexes_are_reported_and_nothing_behind_them_is_read(bits, what, n):
    if what == "slot" and bits == 16:
        pytest.skip("no 8-bit first tokens at 16 bits")
    if what == "start" and n == 1:
        pytest.skip("no other sequence")
    q_lens, kv_lens = [ROWS, ROWS + 1][:n], [ROWS + 60, ROWS + 33][:n]
    cache, batch, tables, q, slots = setup(95, q_lens, kv_lens, 2, 2, 64, bits, 16, bos=bits == 4, extra=0)
    good = hbl.hbl_attention_window(cache, batch, q, 20, 4)
    if what == "page":
        batch.pages[0, (ROWS + 59) // 16] = 1 << 30
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
    other = slice(0, ROWS) if what == "start" else slice(ROWS, sum(q_lens))       # the other sequence is not touched by it
    assert torch.equal(out[other], good[other])


@pytest.mark.parametrize("bits,group", [(16, 1), (16, 4), (4, 2), (8, 1)])
def test_strided_queries_and_outputs(bits, group):
    q_lens, kv_lens, KH = [ROWS, 3], [ROWS + 59, 31], 2
    H, T = KH * group, ROWS + 3
    cache, batch, tables, q, _ = setup(71, q_lens, kv_lens, H, KH, 128, bits, 32, extra=0)
    want, _ = check_window(cache, batch, tables, q_lens, kv_lens, q, 20, 4)
    fused = torch.zeros(T, H + 4, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:2 + H] = q
    big = torch.full((T, H + 5, 136), 5.0, dtype=torch.bfloat16, device="cuda")
    hbl.hbl_attention_window(cache, batch, fused[:, 2:2 + H], 20, 4, out=big[:, 1:1 + H, :128])
    assert torch.equal(big[:, 1:1 + H, :128], want)
    big[:, 1:1 + H, :128] = 5.0
    assert (big == 5.0).all()


def test_another_stream():
    cache, batch, tables, q, _ = setup(99, [1, ROWS], [3000, 2900], 4, 4, 128, 4, 64, extra=0)
    want = hbl.hbl_attention_window(cache, batch, q, 700, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hbl.hbl_attention_window(cache, batch, q, 700, 4)
    s.synchronize()
    assert torch.equal(got, want)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 values, the sequence's pages at its far end."""
    page, KH, D, q_len = 128, 8, 128, ROWS
    n_pages = (1 << 31) // (page * KH * D) + 40
    cache = hbl.KvCache(*(torch.empty(n_pages, KH, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)), bits=16)
    g = gen(81)
    kv, ids = 640, [n_pages - 1, -9, n_pages - 17, n_pages - 2, n_pages - 20]
    for x in (cache.k, cache.v):
        x[n_pages - 20:] = torch.randn(20, KH, page, D, device="cuda", generator=g)
    batch = hbl.KvBatch(torch.tensor([0, q_len], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda"),
                        torch.tensor([ids], dtype=torch.int32, device="cuda"), tokens=q_len, max_q_len=q_len, max_kv_len=kv)
    check_window(cache, batch, [ids], [q_len], [kv], heads(g, q_len, KH, D), 130, 3)


SPLIT = [  # q_lens, kv_lens, window, sinks: with few items, so that the keys of the tiles are dealt in pieces
    ([300], [9000], 4096, 0),
    ([300], [9000], 4096, 200),                                               # the sinks end within the first piece
    ([300], [9000], 1500, 5),
    ([300], [5000], 2048, 2500),                                              # more sinks than a piece has keys
    ([300], [3000], 8000, 0),                                                 # the window is longer than the sequence
    ([300, 1, 40], [9000, 130, 5000], 4096, 200),                             # one kernel's pieces and the other's
    ([300, 1, 40], [9000, 130, 5000], 1500, 5),
    ([300, 0, 170, 2], [2900, 50, 171, 2], 2100, 17),                         # some with a piece less, or one only
    ([400, 200], [300, 8000], 3000, 40),                                      # more queries than tokens: the first rows see nothing
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("lens", range(len(SPLIT)))
@pytest.mark.parametrize("H,KH,D,page", [(4, 2, 128, 64), (2, 1, 64, 16), (2, 2, 256, 128)])
def test_long_windows_are_split_and_joined(bits, lens, H, KH, D, page):
    q_lens, kv_lens, window, sinks = SPLIT[lens]
    cache, batch, tables, q, slots = setup(4100 + lens, q_lens, kv_lens, H, KH, D, bits, page, bos=bits < 8 and (lens % 2 == 1 or lens == 4))
    longest = max(q_lens)
    for bound in (max(kv_lens), 1 << 20):                                     # exact, and far above the lengths
        b = hbl.KvBatch(batch.q_start, batch.kv_len, batch.pages, tokens=batch.tokens, max_q_len=longest, max_kv_len=bound, bos_slot=batch.bos_slot)
        size = hbl.hbl_attention_window_workspace_bytes(cache, b, H, window, sinks)
        assert size > 0
        ws = hbl.new_workspace(size)
        ws.fill_(255)                                                         # NaN, wherever it is read before it is written
        first = check_window(cache, b, tables, q_lens, kv_lens, q, window, sinks, slots=slots, workspace=ws)
        ws.fill_(255)
        again = check_window(cache, b, tables, q_lens, kv_lens, q, window, sinks, slots=slots, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("sinks", [0, 4])
def test_what_no_row_sees_does_not_matter_to_pieces(bits, sinks):
    q_lens, kv_lens, window, page = [200], [6000], 2500, 32
    cache, batch, tables, q, slots = setup(64, q_lens, kv_lens, 2, 2, 128, bits, page, bos=bits < 8)
    assert hbl.hbl_attention_window_workspace_bytes(cache, batch, 2, window, sinks) > 0
    want = check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, slots=slots)
    seen = visible(q_lens[0], kv_lens[0], window, sinks).any(0).tolist()
    live = torch.zeros(cache.n_pages, page, dtype=torch.bool, device="cuda")
    given_away = 0
    for i, x in enumerate(tables[0]):
        mine = seen[i * page:(i + 1) * page]
        if any(mine):
            live[x, :len(mine)] = torch.tensor(mine, device="cuda")
        else:
            batch.pages[0, i] = (-3, 1 << 30)[given_away % 2]
            given_away += 1
    assert given_away > 90
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
@pytest.mark.parametrize("which", ["key", "value"])
def test_what_is_not_finite_within_a_later_piece(bits, which):
    window, sinks, q_lens, kv_lens = 2000, 2, [250], [4000]
    cache, batch, tables, q, _ = setup(65, q_lens, kv_lens, 2, 2, 64, bits, 16, extra=0)
    assert hbl.hbl_attention_window_workspace_bytes(cache, batch, 2, window, sinks) > 0
    clean = hbl.hbl_attention_window(cache, batch, q, window, sinks)
    for at in (kv_lens[0] - 100, kv_lens[0] - window - 100):                  # some rows do not reach it yet; for some it has gone
        c = hbl.KvCache(cache.k.clone(), cache.v.clone(), None if bits == 16 else cache.k_scale.clone(), None if bits == 16 else cache.v_scale.clone(), bits=bits)
        pg, sl = tables[0][at // 16], at % 16
        if bits == 16:
            (c.k if which == "key" else c.v)[pg, :, sl] = float("nan")
        else:
            (c.k_scale if which == "key" else c.v_scale)[pg, :, sl] = float("nan")
        out = hbl.hbl_attention_window(c, batch, q, window, sinks)
        sees = visible(q_lens[0], kv_lens[0], window, sinks)[:, at]
        assert 0 < sees.sum() < q_lens[0]
        assert torch.isnan(out[sees]).all()
        assert torch.equal(out[~sees], clean[~sees])


def test_a_captured_chunk_follows_the_cache():
    """Two graphs that share a workspace, replayed one after the other while the lengths grow."""
    q_lens, kv_lens = [ROWS, 1], [1900, 400]
    cache, batch, tables, q, _ = setup(97, q_lens, kv_lens, 4, 2, 128, 4, 64, extra=0, max_pages=60)
    batch.pages[:, :] = torch.arange(120, dtype=torch.int32, device="cuda").reshape(2, 60) % cache.n_pages
    tables = batch.pages.tolist()
    batch.c.max_kv_len = 3000
    size = hbl.hbl_attention_window_workspace_bytes(cache, batch, 4, 1300, 4)
    assert size > 0
    ws = hbl.new_workspace(size)
    q2 = heads(gen(98), ROWS + 1, 4, 128)
    outs = [torch.empty_like(q), torch.empty_like(q)]
    graphs = []
    for x, o in zip((q, q2), outs):
        hbl.hbl_attention_window(cache, batch, x, 1300, 4, out=o, workspace=ws)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            hbl.hbl_attention_window(cache, batch, x, 1300, 4, out=o, workspace=ws)
        graphs.append(gr)
    for _ in range(3):
        batch.kv_len.add_(310)
        ws.fill_(255)
        for gr in graphs:
            gr.replay()
        lens = batch.kv_len.tolist()
        for x, o in zip((q, q2), outs):
            ref, _, tol, _ = window64(cache, x, q_lens, lens, tables, 1300, 4)
            assert ((o.to(F8) - ref).abs() <= tol).all()
    assert hbl.hbl_check_status() == 0


def test_calls_at_the_same_time():
    """Two streams, a workspace each: split chunks beside a batch of chunks and steps, over one cache, again and again."""
    cache, batch, tables, q, _ = setup(98, [300], [6000], 4, 2, 128, 4, 64, extra=0)
    lens = [200, 1, 40], [2900, 3100, 50]
    g = gen(97)
    starts = torch.tensor([0, 200, 201, 241], dtype=torch.int32, device="cuda")
    other = hbl.KvBatch(starts, torch.tensor(lens[1], dtype=torch.int32, device="cuda"), batch.pages[:, :64].expand(3, -1).contiguous(), tokens=241,
                        max_q_len=200, max_kv_len=3100)                       # (three sequences with the first one's tokens)
    q2 = heads(g, 241, 4, 128)
    calls = [(batch, q, 4096, 17, [300], [6000], tables), (other, q2, 1500, 5, *lens, [tables[0][:64]] * 3)]
    spaces = [hbl.new_workspace(max(1, hbl.hbl_attention_window_workspace_bytes(cache, b, 4, w, s))) for b, _, w, s, *_ in calls]
    assert spaces[0].numel() > 1
    want = [check_window(cache, b, t, ql, kl, x, w, s)[0] for b, x, w, s, ql, kl, t in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i, (b, x, w, s, *_) in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                got[i].append(hbl.hbl_attention_window(cache, b, x, w, s, workspace=spaces[i]))
    torch.cuda.synchronize()
    for a, outs in zip(want, got):
        assert all(torch.equal(a, o) for o in outs)
    assert hbl.hbl_check_status() == 0
