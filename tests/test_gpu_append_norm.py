"""Normalised keys and queries on the way into the cache: the codes, scales and values of the fp32 formula, bit for bit."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import decode, heads
from window_ref import check_window

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
EPS = 2.0 ** -20


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def gain_of(g, D, dtype):
    return (1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(dtype)


def plain(x, gain, rows, interleaved):
    """fp32, products and sums in the documented order; the statistic in 64 bits, rounded once."""
    r = (1 / (x.double().square().mean(-1, keepdim=True) + EPS).sqrt()).float()
    z = x.float() if gain is None else x.float() * gain.float()
    if rows is not None:
        half = rows.shape[1]
        c, s = rows[:, None].unbind(-1)
        a, b = (z[..., 0:2 * half:2], z[..., 1:2 * half:2]) if interleaved else (z[..., :half], z[..., half:2 * half])
        a, b = a * c - b * s, b * c + a * s
        z = torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), z[..., 2 * half:]], -1)
    return z * r


def codes(x, bits):
    c = torch.full((), float(2 ** (bits - 1) - 1), device="cuda")
    top = x.abs().amax(-1)
    return torch.round(x * (c / (top + 1e-5))[..., None]).long() + 2 ** (bits - 1), top / c


def batch_of(g, cache, q_lens, kv_lens, extra=0):
    page = cache.page_size
    ids = torch.randperm(cache.n_pages, device="cuda", generator=g).to(torch.int32)
    width = max(-(-n // page) for n in kv_lens)
    pages = torch.full((len(kv_lens), width), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(kv_lens):
        w = -(-n // page)
        pages[b, :w] = ids[at:at + w]
        at += w
    start = [sum(q_lens[:i]) for i in range(len(q_lens) + 1)]
    batch = hbl.KvBatch(torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor(kv_lens, dtype=torch.int32, device="cuda"), pages,
                        tokens=start[-1] + extra, max_q_len=max(q_lens), max_kv_len=max(kv_lens))
    pos = torch.cat([torch.arange(n - q, n, device="cuda") for q, n in zip(q_lens, kv_lens)])
    seq = torch.repeat_interleave(torch.arange(len(q_lens), device="cuda"), torch.tensor(q_lens, device="cuda"))
    return batch, pos, pages[seq, pos // page].long(), pos % page


def check_cache(bits, interleaved, q_lens, kv_lens, H, KH, D, rot, gain):
    g = gen(sum(kv_lens) + D + bits)
    cache = hbl.KvCache.empty(sum(-(-n // 32) for n in kv_lens) + 2, 32, KH, D, bits, len(kv_lens) if bits < 8 else 0)
    batch, pos, page, slot = batch_of(g, cache, q_lens, kv_lens)
    T = len(pos)
    q, k, v = heads(g, T, H, D), heads(g, T, KH, D), heads(g, T, KH, D)
    gq, gk = (None if gain is None else gain_of(g, D, gain) for _ in range(2))
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(rot), max(kv_lens) + 1) if rot else None
    q_out = hbl.hbl_kv_append_norm(cache, batch, k, v, gk, table=table, interleaved=interleaved, q=q, q_gain=gq, norm_eps=EPS)
    assert hbl.hbl_check_status() == 0
    rows = table[pos] if rot else None
    assert torch.equal(q_out, plain(q, gq, rows, interleaved).to(BF16))
    assert torch.equal(q_out, hbl.hbl_norm_rope(q, gq, pos.int() if rot else None, table, norm_eps=EPS, interleaved=interleaved)[0])
    for x, buf, scale, first, first_scale in ((plain(k, gk, rows, interleaved), cache.k, cache.k_scale, cache.bos_k, cache.bos_k_scale),
                                              (v.float(), cache.v, cache.v_scale, cache.bos_v, cache.bos_v_scale)):
        if bits == 16:
            assert torch.equal(buf[page, :, slot], x.to(BF16))
            continue
        u, sc = codes(x, bits)
        assert torch.equal(decode(buf[page, :, slot], bits, D), u) and torch.equal(scale[page, :, slot], sc)
        if first is not None:
            u, sc = codes(x, 8)
            starts = (pos == 0).nonzero().flatten()
            seq = [b for b, (a, n) in enumerate(zip(q_lens, kv_lens)) if a == n]
            assert torch.equal(first[seq].long(), u[starts]) and torch.equal(first_scale[seq], sc[starts])


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [1]), ([1, 1, 1], [700, 17, 1]), ([100, 3, 41], [100, 60, 500]), ([700, 900], [700, 900])])
@pytest.mark.parametrize("H,KH,D,rot,gain", [(4, 4, 128, 128, BF16), (7, 1, 128, 64, torch.float32), (8, 2, 64, 32, None), (3, 3, 256, 256, BF16), (4, 2, 128, 0, BF16)])
def test_the_cache_holds_the_formula(bits, interleaved, q_lens, kv_lens, H, KH, D, rot, gain):
    check_cache(bits, interleaved, q_lens, kv_lens, H, KH, D, rot, gain)


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,KH,D,rot,gain", [(9001, 4, 4, 128, 128, BF16), (9001, 7, 1, 128, 64, torch.float32), (13000, 8, 2, 64, 64, BF16), (14000, 7, 3, 64, 32, None),
                                               (5000, 5, 2, 256, 128, BF16), (4001, 32, 8, 128, 128, BF16)])
def test_prompts_of_several_heads_to_a_thread(bits, interleaved, T, H, KH, D, rot, gain):
    check_cache(bits, interleaved, [T - 5, 5], [T - 5, 64], H, KH, D, rot, gain)


@pytest.mark.parametrize("bits", [4, 16])
def test_strides_positions_and_rows_behind_the_last_sequence(bits):
    g = gen(3)
    D, H, KH, T, extra = 128, 4, 2, 70, 5
    cache, other = (hbl.KvCache.empty(8, 16, KH, D, bits) for _ in range(2))
    batch, pos, page, slot = batch_of(g, cache, [T], [T + 20], extra)
    fused = heads(g, T + extra, H + 2 * KH, D)
    keep = fused.clone()
    gq, gk = gain_of(g, D, BF16), gain_of(g, D, BF16)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), 4096)
    turns = torch.randint(0, 4096, (T + extra,), device="cuda", generator=g, dtype=torch.int32)
    q, k, v = fused[:, :H], fused[:, H:H + KH], fused[:, H + KH:]
    want = hbl.hbl_kv_append_norm(other, batch, k.contiguous(), v.contiguous(), gk, table=table, positions=turns, q=q.contiguous(), q_gain=gq, norm_eps=EPS)
    hbl.hbl_kv_append_norm(cache, batch, k, v, gk, table=table, positions=turns, q=q, q_gain=gq, q_out=q, norm_eps=EPS)
    assert hbl.hbl_check_status() == 0
    assert torch.equal(q[:T], want[:T]) and torch.equal(fused[:, H:], keep[:, H:]) and torch.equal(fused[T:], keep[T:])
    assert torch.equal(q[:T], hbl.hbl_norm_rope(keep[:T, :H], gq, turns[:T], table, norm_eps=EPS)[0])
    assert torch.equal(cache.k, other.k) and torch.equal(cache.v, other.v)


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
def test_heads_of_zeros_and_what_is_not_finite(bits):
    g = gen(4)
    D, KH, T = 64, 2, 5
    cache = hbl.KvCache.empty(2, 16, KH, D, bits)
    batch, pos, page, slot = batch_of(g, cache, [T], [T])
    k, v = heads(g, T, KH, D), heads(g, T, KH, D)
    k[0] = 0
    k[1, 0, 3] = float("nan")
    k[2, 1, 9] = float("inf")
    gk = gain_of(g, D, BF16)
    hbl.hbl_kv_append_norm(cache, batch, k, v, gk, norm_eps=EPS)
    ko, vo = hbl.hbl_kv_read(cache, batch)
    assert hbl.hbl_check_status() == 0
    assert (ko[0] == 0).all() and torch.isnan(ko[1, 0]).all() and torch.isfinite(ko[1, 1]).all() and torch.isfinite(ko[2, 0]).all()
    assert torch.isnan(ko[2, 1]).all() if bits < 16 else torch.isnan(ko[2, 1, 9])
    assert torch.isfinite(vo).all() and torch.isfinite(ko[3:]).all()


def test_places_out_of_range_are_reported_and_left_out():
    g = gen(5)
    cache = hbl.KvCache.empty(4, 16, 2, 64, 8)
    batch, pos, page, slot = batch_of(g, cache, [20, 20], [20, 20])
    batch.pages[0, 1] = 99
    k, v = heads(g, 40, 2, 64), heads(g, 40, 2, 64)
    hbl.hbl_kv_append_norm(cache, batch, k, v, None)
    assert hbl.hbl_check_status() == 12 and hbl.hbl_check_status() == 0
    batch.pages[0, 1] = batch.pages[1, 1]
    assert (cache.k_scale != 0).sum() == 36 * 2


@pytest.mark.parametrize("bits,T", [(4, 1), (16, 1), (3, 40), (8, 130), (16, 200)])
def test_from_projections_to_the_input_of_w_o(bits, T):
    """The calls together as a decoder block with normalised heads and a window makes them, in a captured graph too."""
    g = gen(7 + T)
    hidden, ffn, H, D, window, sinks = 2048, 8192, 16, 128, 100, 4
    weights, alphas = {}, []
    for n, (o, i) in dict(q=(hidden, hidden), k=(hidden, hidden), v=(hidden, hidden), o=(hidden, hidden), up=(ffn, hidden), gate=(ffn, hidden),
                          down=(hidden, ffn)).items():
        weights[n], a = hbl.hbl_quantize_weights(torch.randn(o, i, device="cuda", generator=g) * 0.02)
        alphas.append(a)
    alpha7 = torch.cat(alphas)
    gq, gk = gain_of(g, D, BF16), gain_of(g, D, BF16)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), 1024)
    page, past = 64, 350
    cache = hbl.KvCache.empty(20, page, H, D, bits, 2 if bits < 8 else 0)
    pages = torch.randperm(20, device="cuda", generator=g).to(torch.int32).reshape(2, 10)
    lens = [0, 0]

    def layer(x, mid, batch, out):
        y = hbl.hbl_block_forward(dict(attn_in=x, o_in=x, ffn_in=x, down_in=mid), weights, alpha7, hidden, ffn, 4)
        n = x.shape[0]
        q, k, v = (y[c].view(n, H, D) for c in "qkv")
        raw = q.clone()
        hbl.hbl_kv_append_norm(cache, batch, k, v, gk, table=table, q=q, q_gain=gq, q_out=q, norm_eps=EPS)
        hbl.hbl_attention_window(cache, batch, q, window, sinks, out=out)
        return raw, q, hbl.hbl_forward(out.view(n, hidden), weights["o"], alphas[3], hidden, 4, True)

    for n in (past, T):                                                       # a prompt, then a step or a chunk
        q_lens = [n, n]
        lens = [x + n for x in lens]
        batch = hbl.KvBatch(torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"), pages,
                            tokens=2 * n, max_q_len=n, max_kv_len=max(lens))
        x = torch.randn(2 * n, hidden, device="cuda", generator=g).to(BF16)
        mid = torch.randn(2 * n, ffn, device="cuda", generator=g).to(BF16)
        out = torch.empty(2 * n, H, D, dtype=BF16, device="cuda")
        raw, q, z = layer(x, mid, batch, out)
        assert hbl.hbl_check_status() == 0 and torch.isfinite(z).all()
        pos = torch.cat([torch.arange(m - n, m, dtype=torch.int32, device="cuda") for m in lens])
        assert torch.equal(q, hbl.hbl_norm_rope(raw, gq, pos, table, norm_eps=EPS)[0])
        want, _ = check_window(cache, batch, pages.tolist(), q_lens, lens, q, window, sinks, slots=[0, 1] if bits < 8 else None)
        assert torch.equal(out, want)
    side = torch.cuda.Stream()                                                # the step once more, captured
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, mid, batch, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, _, zg = layer(x, mid, batch, out)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want) and torch.equal(zg, z)
    assert hbl.hbl_check_status() == 0
