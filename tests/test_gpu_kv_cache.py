"""Tokens into a paged cache and out of it: codes, scales and places against the quantizer's definition."""
import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import F8, decode, heads, make_batch

pytestmark = pytest.mark.gpu
EPS = 1e-5
POISON = 0xA5


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def new_cache(n_pages, page, heads_, D, bits, slots=0):
    c = hbl.KvCache.empty(n_pages, page, heads_, D, bits, slots)
    for t in (c.k, c.v, c.bos_k, c.bos_v):
        if t is not None:
            t.fill_(POISON if t.dtype == torch.uint8 else 9.0)
    for t in (c.k_scale, c.v_scale, c.bos_k_scale, c.bos_v_scale):
        if t is not None:
            t.fill_(-3.0)
    return c


def quant32(x, bits):
    """The definition, in fp32 with every operation rounded once (a scalar divided by a tensor is a true division)."""
    c = torch.full((), float(2 ** (bits - 1) - 1), device="cuda")
    gamma = x.abs().amax(-1)
    u = torch.round(x * (c / (gamma + EPS))[..., None]) + 2 ** (bits - 1)
    return u.long(), gamma / c


def expected_places(tables, q_lens, kv_lens, page):
    """(page, slot, position, sequence) of every token."""
    out = []
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        out += [(tables[b][p // page], p % page, p, b) for p in range(kv - n, kv)]
    return out


CASES = [  # q_lens, kv_lens, heads, kv heads, D, page
    ([1], [1], 2, 1, 128, 16),
    ([1, 1, 1], [17, 16, 64], 4, 4, 64, 16),
    ([5, 0, 33, 1], [5, 40, 47, 129], 8, 2, 128, 32),
    ([3, 70], [1000, 70], 5, 5, 256, 64),
    ([1] * 40, list(range(1, 41)), 4, 2, 64, 16),
    ([2] * 1100, [2 + i % 7 for i in range(1100)], 2, 1, 64, 16),
    ([700], [900], 32, 32, 128, 128),
]


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_puts_the_quantized_heads_where_they_belong(bits, case, interleaved):
    q_lens, kv_lens, H, KH, D, page = CASES[case]
    g = gen(100 * case + bits)
    slots = len(q_lens) if bits in (3, 4) and case % 2 == 0 else 0
    cache = new_cache(sum(-(-n // page) for n in kv_lens) + 2, page, KH, D, bits, slots)
    perm = torch.randperm(len(q_lens), generator=torch.Generator().manual_seed(case)).tolist() if slots else None
    extra = 3
    batch, tables = make_batch(g, cache, q_lens, kv_lens, max_pages=max(-(-n // page) for n in kv_lens) + 1, extra_rows=extra, slots=perm)
    n = sum(q_lens)
    k, v, q = heads(g, n + extra, KH, D), heads(g, n + extra, KH, D), heads(g, n + extra, H, D)
    if n > 1:
        k[n // 2, 0] = 0                                                    # a head of zeros
    rot = D // 2 if case % 3 == 1 else D
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(rot), max(kv_lens))
    before = {a: getattr(cache, a).clone() for a in ("k", "v", "k_scale", "v_scale", "bos_k", "bos_v", "bos_k_scale", "bos_v_scale")
              if getattr(cache, a) is not None}
    q_out = torch.full_like(q, 3.0)
    hbl.hbl_kv_append(cache, batch, k, v, table=table, interleaved=interleaved, q=q, q_out=q_out, eps=EPS)
    assert hbl.hbl_check_status() == 0
    places = expected_places(tables, q_lens, kv_lens, page)
    pg, sl, pos, sq = (torch.tensor(x, device="cuda") for x in zip(*places))
    pos32 = pos.to(torch.int32)
    assert torch.equal(q_out[:n], hbl.hbl_rope(q[:n].contiguous(), pos32, table, interleaved=interleaved)) and (q_out[n:] == 3).all()
    turned = hbl.hbl_rope(k[:n].float().contiguous(), pos32, table, interleaved=interleaved)     # fp32, itself tested bit for bit
    for name, x in (("k", turned), ("v", v[:n].float())):
        buf, want = getattr(cache, name), before[name].clone()
        if bits == 16:
            want[pg, :, sl] = x.to(torch.bfloat16)
            assert torch.equal(buf, want)
            continue
        u, s = quant32(x, bits)
        assert torch.equal(decode(buf[pg, :, sl], bits, D), u)
        want[pg, :, sl] = buf[pg, :, sl]
        assert torch.equal(buf, want), "rows of other tokens"
        scale = before[name + "_scale"].clone()
        scale[pg, :, sl] = s
        assert torch.equal(getattr(cache, name + "_scale"), scale)
        if slots:
            first = pos == 0
            u8, s8 = quant32(x[first], 8)
            rows = torch.tensor(perm, device="cuda")[sq[first]]
            codes, scales = before["bos_" + name].clone(), before["bos_" + name + "_scale"].clone()
            codes[rows], scales[rows] = u8.to(torch.uint8), s8
            assert torch.equal(getattr(cache, "bos_" + name), codes) and torch.equal(getattr(cache, "bos_" + name + "_scale"), scales)
    # and out again
    ko, vo = hbl.hbl_kv_read(cache, batch)
    assert hbl.hbl_check_status() == 0
    for name, got in (("k", ko), ("v", vo)):
        if bits == 16:
            value = getattr(cache, name)[pg, :, sl]
        else:
            value = (decode(getattr(cache, name)[pg, :, sl], bits, D) - 2 ** (bits - 1)).float() * getattr(cache, name + "_scale")[pg, :, sl][..., None]
            if slots:
                rows = torch.tensor(perm, device="cuda")[sq]
                v8 = (getattr(cache, "bos_" + name)[rows].float() - 128) * getattr(cache, "bos_" + name + "_scale")[rows][..., None]
                value = torch.where((pos == 0)[:, None, None], v8, value)
            value = value.to(torch.bfloat16)
        assert torch.equal(got[:n], value)


@pytest.mark.parametrize("bits", [3, 4, 8])
def test_values_and_unrotated_keys_are_those_of_the_row_quantizer(bits):
    """hbl_quantize_kv and the append share their definition: the same codes and scales, bit for bit."""
    g = gen(bits)
    T, KH, D, page = 50, 3, 128, 16
    cache = new_cache(6, page, KH, D, bits)
    batch, tables = make_batch(g, cache, [T], [T])
    k, v = heads(g, T, KH, D), heads(g, T, KH, D)
    hbl.hbl_kv_append(cache, batch, k, v)
    pg = torch.tensor([tables[0][p // page] for p in range(T)], device="cuda")
    sl = torch.arange(T, device="cuda") % page
    for x, buf, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        codes, s, _, _ = hbl.hbl_quantize_kv(x, bits, 0, EPS)
        assert torch.equal(buf[pg, :, sl].reshape(T * KH, -1), codes) and torch.equal(scale[pg, :, sl].reshape(-1), s)
    assert hbl.hbl_check_status() == 0


def test_positions_of_the_callers_and_strided_in_place_queries():
    g = gen(9)
    T, H, KH, D, page = 30, 4, 2, 128, 32
    fused = heads(g, T, H + 2 * KH, D)
    q, k, v = fused[:, :H], fused[:, H:H + KH], fused[:, H + KH:]
    keep = fused.clone()
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), 1000)
    pos = torch.randint(0, 1000, (T,), device="cuda", generator=g, dtype=torch.int32)
    cache = new_cache(4, page, KH, D, 16)
    batch, tables = make_batch(g, cache, [10, 20], [50, 20])
    got = hbl.hbl_kv_append(cache, batch, k, v, table=table, positions=pos, q=q, q_out=q)
    assert hbl.hbl_check_status() == 0 and got is q
    assert torch.equal(q, hbl.hbl_rope(keep[:, :H].contiguous(), pos, table))
    assert torch.equal(fused[:, H:], keep[:, H:])
    pg, sl, _, _ = (torch.tensor(x, device="cuda") for x in zip(*expected_places(tables, [10, 20], [50, 20], page)))
    assert torch.equal(cache.k[pg, :, sl], hbl.hbl_rope(keep[:, H:H + KH].contiguous(), pos, table))
    assert torch.equal(cache.v[pg, :, sl], keep[:, H + KH:])


@pytest.mark.parametrize("bits", [3, 4, 8])
def test_heads_that_are_not_finite_read_as_nan(bits):
    g = gen(11)
    cache = new_cache(2, 16, 3, 64, bits, 1 if bits < 8 else 0)
    batch, tables = make_batch(g, cache, [4], [4])
    k, v = heads(g, 4, 3, 64), heads(g, 4, 3, 64)
    k[0, 1, 5], k[2, 0, 63], v[1, 2, 0] = float("nan"), float("inf"), -float("inf")
    hbl.hbl_kv_append(cache, batch, k, v)
    ko, vo = hbl.hbl_kv_read(cache, batch)
    bad_k, bad_v = torch.zeros(4, 3, dtype=torch.bool, device="cuda"), torch.zeros(4, 3, dtype=torch.bool, device="cuda")
    bad_k[0, 1] = bad_k[2, 0] = bad_v[1, 2] = True
    assert torch.equal(torch.isnan(ko).all(-1), bad_k) and torch.equal(torch.isnan(vo).all(-1), bad_v)
    assert torch.equal(torch.isnan(ko).any(-1), bad_k) and torch.equal(torch.isnan(vo).any(-1), bad_v)
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("what", ["page high", "page negative", "position", "length beyond the table", "negative length", "slot", "start"])
def test_bad_indexes_are_reported_and_their_tokens_left_out(what):
    g = gen(12)
    cache = new_cache(6, 16, 2, 64, 4, 2)
    batch, tables = make_batch(g, cache, [4, 4], [20, 4], slots=[0, 1])
    k, v = heads(g, 8, 2, 64), heads(g, 8, 2, 64)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(64), 20)
    kw = {}
    good = [True] * 8
    if what.startswith("page"):
        batch.pages[0, 1] = 6 if what == "page high" else -1
        good[:4] = [False] * 4                                              # positions 16 .. 19 lie in that page
    elif what == "position":
        kw["positions"] = torch.tensor([0, 20, -1, 19, 0, 1, 2, 3], dtype=torch.int32, device="cuda")
        good[1] = good[2] = False
    elif what == "length beyond the table":
        batch.kv_len[0] = 34                                                # two pages hold 32: positions 30, 31 fit
        table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(64), 64)
        good[2] = good[3] = False
    elif what == "negative length":
        batch.kv_len[0] = -1
        good[:4] = [False] * 4
    elif what == "slot":
        batch.bos_slot[1] = 2
        good[4] = False                                                     # the second sequence's first token
    else:
        batch.q_start[2] = 9                                                # more rows than there are
        good[4:] = [False] * 4
    before = cache.k.clone()
    hbl.hbl_kv_append(cache, batch, k, v, table=table, **kw)
    assert hbl.hbl_check_status() == 12
    assert hbl.hbl_check_status() == 0
    written = (cache.k != before).any(-1).sum().item()
    assert written == 2 * sum(good)
    hbl.hbl_kv_read(cache, batch)
    assert hbl.hbl_check_status() == (0 if what == "position" else 12)


def test_append_in_a_graph_follows_the_lengths():
    g = gen(13)
    cache = new_cache(8, 16, 2, 128, 4)
    batch, tables = make_batch(g, cache, [1, 1], [5, 40], max_pages=4)
    batch.pages[:, :] = torch.tensor([[0, 1, 2, 3], [4, 5, 6, 7]], dtype=torch.int32)
    k, v = heads(g, 2, 2, 128), heads(g, 2, 2, 128)
    hbl.hbl_kv_append(cache, batch, k, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hbl.hbl_kv_append(cache, batch, k, v)
    for step in range(20):
        batch.kv_len.add_(1)
        k.copy_(heads(g, 2, 2, 128))
        graph.replay()
        u, s = quant32(k.float(), 4)
        for b, n in enumerate((6 + step, 41 + step)):
            pg, sl = 4 * b + (n - 1) // 16, (n - 1) % 16
            assert torch.equal(decode(cache.k[pg, :, sl], 4, 128), u[b]) and torch.equal(cache.k_scale[pg, :, sl], s[b])
    assert hbl.hbl_check_status() == 0


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("H,KH,D", [(32, 32, 128), (32, 8, 128), (32, 32, 256), (16, 16, 64), (7, 1, 128)])
def test_calls_that_fill_the_gpu(bits, H, KH, D):
    """Many tokens: several heads to a thread, in every number that the launch chooses between."""
    g = gen(bits + H + D)
    page, T = 64, 2_500_000 // ((H + 2 * KH) * D // 8)
    cache = new_cache(-(-T // page) + 1, page, KH, D, bits, 1 if bits < 8 else 0)
    batch, tables = make_batch(g, cache, [T], [T], slots=[0] if bits < 8 else None)
    k, v, q = heads(g, T, KH, D), heads(g, T, KH, D), heads(g, T, H, D)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), T)
    for interleaved in (False, True):
        q_out = hbl.hbl_kv_append(cache, batch, k, v, table=table, interleaved=interleaved, q=q)
        ko, vo = hbl.hbl_kv_read(cache, batch)
        assert hbl.hbl_check_status() == 0
        pos = torch.arange(T, device="cuda", dtype=torch.int32)
        assert torch.equal(q_out, hbl.hbl_rope(q, pos, table, interleaved=interleaved))
        turned = hbl.hbl_rope(k.float(), pos, table, interleaved=interleaved)
        pg, sl = torch.tensor(tables[0], device="cuda")[pos.long() // page], pos.long() % page
        for x, buf, scale, out in ((turned, cache.k, cache.k_scale, ko), (v.float(), cache.v, cache.v_scale, vo)):
            if bits == 16:
                assert torch.equal(out, x.to(torch.bfloat16)) and torch.equal(buf[pg, :, sl], out)
                continue
            u, s = quant32(x, bits)
            assert torch.equal(decode(buf[pg, :, sl], bits, D), u) and torch.equal(scale[pg, :, sl], s)
            value = ((u - 2 ** (bits - 1)).float() * s[..., None]).to(torch.bfloat16)
            if bits < 8:
                u8, s8 = quant32(x[:1], 8)
                value[0] = ((u8 - 128).float() * s8[..., None]).to(torch.bfloat16)[0]
            assert torch.equal(out, value)
