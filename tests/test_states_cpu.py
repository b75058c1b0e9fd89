"""Rotary frequencies, argument checks of the cache and attention calls: no GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2504_18415_b200 import build, hbl


@pytest.fixture(scope="module")
def L():
    build.build()
    return hbl.lib()


P, N = C.c_void_p(1024), C.c_void_p(0)          # P is never dereferenced on the host: validation must stop first


def fields(*groups):
    return [(n, t) for t, names in groups for n in names.split()]


def strides(names):
    return " ".join(f"{n}_{s}_stride" for n in names.split() for s in ("token", "head"))


class Rope(C.Structure):                        # the argument structures as include/hbl.h declares them
    _fields_ = fields((C.c_void_p, "x out positions table"), (C.c_longlong, strides("x out")),
                      (C.c_int, "dtype tokens n_heads head_dim n_pos rot_dim layout backward"))


class Append(C.Structure):
    _fields_ = fields((C.c_void_p, "k v q q_out"), (C.c_longlong, strides("k v q q_out")), (C.c_void_p, "table positions"),
                      (C.c_int, "n_heads n_pos rot_dim layout"), (C.c_float, "eps"))


class Attention(C.Structure):
    _fields_ = fields((C.c_void_p, "q out lse"), (C.c_longlong, strides("q out")), (C.c_int, "n_heads causal"), (C.c_float, "sm_scale"))


def test_frequencies_follow_their_formulas(L):
    for rot in (2, 64, 128, 256):
        f = hbl.hbl_rope_frequencies(rot, 10000.0)
        assert f == pytest.approx([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], rel=1e-15)
        assert hbl.hbl_rope_frequencies(rot, 10000.0, hbl.ROPE_LINEAR, factor=4.0) == pytest.approx([x / 4 for x in f], rel=1e-15)
    f = hbl.hbl_rope_frequencies(128)
    g = hbl.hbl_rope_frequencies(128, scaling=hbl.ROPE_BASE, factor=8.0)
    assert g[0] == 1.0 and f[-1] / g[-1] == pytest.approx(8.0, rel=1e-12)       # fastest pair kept, slowest stretched by the factor
    h = hbl.hbl_rope_frequencies(128, scaling=hbl.ROPE_PARTS, factor=8.0, trained_len=2048, slow=1.0, fast=4.0)
    for x, y in zip(f, h):
        turns = 2048 * x / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / 3.0))
        assert y == pytest.approx(keep * x + (1 - keep) * x / 8, rel=1e-14)
    assert h[0] == f[0] and h[-1] == f[-1] / 8
    assert hbl.hbl_rope_frequencies(128, scaling=hbl.ROPE_PARTS, factor=1.0, trained_len=2048) == pytest.approx(f, rel=1e-15)


def test_frequencies_refuse_what_has_no_meaning(L):
    out = (C.c_double * 128)()
    f = lambda base=1e4, rot=64, kind=0, factor=2.0, length=100.0, slow=1.0, fast=4.0, o=out: \
        L.hbl_rope_frequencies(base, rot, kind, factor, length, slow, fast, o)
    assert f() == 0
    assert f(o=None) == 1
    assert f(rot=0) == 2 and f(rot=63) == 2 and f(rot=258) == 2
    assert f(kind=4) == 10 and f(kind=-1) == 10
    assert f(base=1.0) == 2 and f(base=math.nan) == 2 and f(base=math.inf) == 2
    assert f(kind=1, factor=0.5) == 2 and f(kind=2, factor=math.nan) == 2 and f(kind=2, rot=2) == 2
    assert f(kind=3, length=0.0) == 2 and f(kind=3, slow=4.0) == 2 and f(kind=3, slow=0.0) == 2
    assert f(kind=0, factor=0.0, length=0.0, slow=0.0, fast=0.0) == 0            # not looked at


def test_table_and_rope_refusals(L):
    host = (C.c_double * 64)(*([1.0] * 64))
    t = lambda freq=host, n=64, amp=1.0, first=0, pos=16, table=P: L.hbl_rope_table(freq, n, amp, first, pos, table, N)
    assert t(pos=0) == 0
    assert t(n=0) == 2 and t(n=129) == 2 and t(pos=-1) == 2 and t(first=-1) == 2
    assert t(first=0x7fffffff, pos=1) == 11
    assert t(amp=math.inf) == 2
    assert t(freq=None) == 1 and t(table=N) == 1 and t(table=C.c_void_p(1032)) == 5
    def r(**k):
        a = Rope(1024, 1 << 20, 1024, 1024, 1024, 128, 1024, 128, 1, 4, 8, 128, 16, 128, 0, 0)
        for n, v in k.items():
            setattr(a, dict(dt="dtype", T="tokens", H="n_heads", D="head_dim", ts="x_token_stride", hs="x_head_stride", ots="out_token_stride",
                            ohs="out_head_stride", pos="positions", rot="rot_dim").get(n, n), v.value or 0 if isinstance(v, C.c_void_p) else v)
        return L.hbl_rope(bytes(a), N)
    assert L.hbl_rope(None, N) == 1
    assert r(T=0) == 0
    assert r(dt=2) == 10 and r(layout=2) == 10
    assert r(T=-1) == 2 and r(H=0) == 2 and r(D=12) == 2 and r(D=264) == 2
    assert r(rot=24) == 2 and r(rot=0) == 2 and r(rot=144) == 2 and r(n_pos=0) == 2
    assert r(x=N) == 1 and r(pos=N) == 1 and r(table=N) == 1 and r(out=N) == 1
    assert r(x=C.c_void_p(1028)) == 5 and r(ts=1028) == 5 and r(ohs=4) == 5 and r(table=C.c_void_p(1028)) == 5 and r(pos=C.c_void_p(1026)) == 5
    assert r(ts=-1024) == 2
    assert r(out=P, ots=2048) == 2                                              # in place, other strides


def cache_t(**k):
    c = hbl.hbl_kv_cache_t()
    c.k = c.v = c.k_scale = c.v_scale = 1 << 20
    c.n_pages, c.page_size, c.n_kv_heads, c.head_dim, c.bits, c.n_slots = 8, 16, 4, 128, 4, 0
    for n, v in k.items():
        setattr(c, n, v)
    return c


def batch_t(**k):
    b = hbl.hbl_kv_batch_t()
    b.q_start = b.kv_len = b.pages = 1 << 20
    b.n_seqs, b.tokens, b.max_pages, b.max_q_len, b.max_kv_len = 2, 4, 8, 2, 100
    for n, v in k.items():
        setattr(b, n, v)
    return b


@pytest.mark.parametrize("kind,packed", [(Rope, hbl._ROPE_T), (Append, hbl._APPEND_T), (Attention, hbl._ATTENTION_T)])
def test_packed_arguments_are_the_structures_of_the_header(kind, packed):
    assert packed.size == C.sizeof(kind)
    values = [0.5 + i if t is C.c_float else 1 + i for i, (_, t) in enumerate(kind._fields_)]
    got = kind.from_buffer_copy(packed.pack(*values))
    assert [getattr(got, n) for n, _ in kind._fields_] == values


def append_t(**k):
    a = Append()
    a.k = a.v = 1 << 20
    for n in ("k", "v", "q", "q_out"):
        setattr(a, n + "_token_stride", 512)
        setattr(a, n + "_head_stride", 128)
    a.n_heads, a.n_pos, a.rot_dim, a.layout, a.eps = 4, 128, 128, 0, 1e-5
    for n, v in k.items():
        setattr(a, n, v)
    return bytes(a)


def attention_t(**k):
    a = Attention()
    a.q = a.out = 1 << 20
    for n in ("q", "out"):
        setattr(a, n + "_token_stride", 512)
        setattr(a, n + "_head_stride", 128)
    a.n_heads, a.causal, a.sm_scale = 4, 1, 0.1
    for n, v in k.items():
        setattr(a, n, v)
    return bytes(a)


BAD_CACHES = [(dict(bits=5), 4), (dict(head_dim=96), 2), (dict(n_kv_heads=0), 2), (dict(n_pages=0), 2), (dict(page_size=8), 2),
              (dict(page_size=24), 2), (dict(page_size=8192), 2), (dict(k=0), 1), (dict(v=0), 1), (dict(k=1 << 20 | 8), 5),
              (dict(k_scale=0), 1), (dict(v_scale=(1 << 20) + 2), 5), (dict(bits=16), 10), (dict(bos_k=1 << 20), 1),
              (dict(bos_k=1 << 20, bos_v=1 << 20, bos_k_scale=1 << 20, bos_v_scale=1 << 20), 2),
              (dict(bits=8, bos_k=1 << 20), 4)]
BAD_BATCHES = [(dict(n_seqs=-1), 2), (dict(tokens=-1), 2), (dict(max_pages=-1), 2), (dict(max_q_len=-1), 2), (dict(max_kv_len=-1), 2),
               (dict(max_kv_len=(1 << 30) + 1), 11), (dict(q_start=0), 1), (dict(kv_len=0), 1), (dict(pages=0), 1), (dict(pages=(1 << 20) + 2), 5)]


def test_cache_and_batch_refusals(L):
    app, att, ref = append_t(), attention_t(), C.byref
    calls = [lambda c, b: L.hbl_kv_append(c, b, app, N), lambda c, b: L.hbl_kv_read(c, b, P, P, N),
             lambda c, b: L.hbl_attention(c, b, att, P, 1 << 40, N)]
    for call in calls:
        assert call(None, ref(batch_t())) == 1 and call(ref(cache_t()), None) == 1
        for k, want in BAD_CACHES:
            assert call(ref(cache_t(**k)), ref(batch_t())) == want, k
        for k, want in BAD_BATCHES:
            assert call(ref(cache_t()), ref(batch_t(**k))) == want, k
        assert call(ref(cache_t()), ref(batch_t(n_seqs=0))) == 0                 # nothing to do
        assert call(ref(cache_t()), ref(batch_t(tokens=0, q_start=0))) == 0
    for k, want in BAD_CACHES:
        assert L.hbl_attention_workspace_bytes(ref(cache_t(**k)), ref(batch_t()), 4) == 0
    assert L.hbl_attention_workspace_bytes(ref(cache_t()), ref(batch_t()), 6) == 0


def test_append_read_and_attention_refusals(L):
    ref = C.byref
    ap = lambda **k: L.hbl_kv_append(ref(cache_t()), ref(batch_t()), append_t(**k), N)
    assert L.hbl_kv_append(ref(cache_t()), ref(batch_t()), None, N) == 1
    assert ap(eps=0.0) == 7 and ap(eps=math.nan) == 7
    assert ap(k=0) == 1 and ap(v=0) == 1
    assert ap(k=(1 << 20) + 8) == 5 and ap(k_token_stride=511) == 5 and ap(v_head_stride=-128) == 2
    assert ap(q=1 << 20) == 1                                                   # nowhere to put them
    assert ap(q=1 << 20, q_out=1 << 20) == 1                                    # nothing to rotate them by
    rot = dict(table=1 << 20)
    assert ap(**rot, rot_dim=8) == 2 and ap(**rot, rot_dim=144) == 2 and ap(**rot, n_pos=0) == 2 and ap(**rot, layout=3) == 10
    assert ap(table=(1 << 20) + 8) == 5
    assert ap(**rot, q=1 << 20, q_out=1 << 20, n_heads=0) == 2
    assert ap(**rot, q=1 << 20, q_out=1 << 20, q_token_stride=1024) == 2        # in place, other strides
    assert ap(**rot, q=1 << 20, q_out=(1 << 20) + 4) == 5
    assert ap(positions=(1 << 20) + 1) == 5
    assert L.hbl_kv_read(ref(cache_t()), ref(batch_t()), N, P, N) == 1 and L.hbl_kv_read(ref(cache_t()), ref(batch_t()), P, C.c_void_p(1032), N) == 5
    at = lambda ws=P, n=1 << 40, **k: L.hbl_attention(ref(cache_t()), ref(batch_t()), attention_t(**k), ws, n, N)
    assert L.hbl_attention(ref(cache_t()), ref(batch_t()), None, P, 1 << 40, N) == 1
    assert at(n_heads=6) == 2 and at(n_heads=0) == 2 and at(sm_scale=math.inf) == 2 and at(sm_scale=math.nan) == 2
    assert at(q=0) == 1 and at(out=0) == 1 and at(q=(1 << 20) + 8) == 5 and at(out_token_stride=4) == 5 and at(lse=(1 << 20) + 2) == 5
    assert at(ws=C.c_void_p(1536)) == 5
    # a batch whose keys are split needs its workspace
    long = batch_t(max_kv_len=65536, max_pages=4096)
    need = L.hbl_attention_workspace_bytes(ref(cache_t()), ref(long), 4)
    assert need > 0
    assert L.hbl_attention(ref(cache_t()), ref(long), attention_t(), N, 0, N) == 1
    assert L.hbl_attention(ref(cache_t()), ref(long), attention_t(), P, need - 1, N) == 6
    assert L.hbl_attention(ref(cache_t()), ref(batch_t(max_q_len=0)), attention_t(), P, 1 << 40, N) == 0


def test_binding_refuses_what_is_not_on_the_gpu():
    z = torch.zeros
    with pytest.raises(ValueError):
        hbl.KvCache(z(2, 1, 16, 64, dtype=torch.uint8), z(2, 1, 16, 64, dtype=torch.uint8), z(2, 1, 16), z(2, 1, 16), bits=4)
    with pytest.raises(hbl.HblError):
        hbl.KvCache(z(2, 1, 16, 64, dtype=torch.uint8), z(2, 1, 16, 64, dtype=torch.uint8), bits=5)
    with pytest.raises(ValueError):
        hbl.KvBatch(z(2, dtype=torch.int32), z(1, dtype=torch.int32), z(1, 1, dtype=torch.int32), tokens=1, max_q_len=1, max_kv_len=1)
    with pytest.raises(ValueError):
        hbl.hbl_rope(z(1, 1, 16, dtype=torch.bfloat16), z(1, dtype=torch.int32), z(1, 8, 2))


def test_outputs_whose_heads_lie_on_each_other_are_refused(L):
    rope = lambda ts, hs, tokens=8, heads=4: L.hbl_rope(bytes(Rope(1024, 1 << 30, 1024, 1024, 0, 0, ts, hs, 1, tokens, heads, 128, 16, 128, 0, 0)), N)
    assert rope(0, 128) == 2 and rope(512, 0) == 2 and rope(512, 120) == 2 and rope(120, 1024) == 2 and rope(128, 128) == 2
    assert rope(0, 0, heads=1) == 2 and rope(0, 0, tokens=1) == 2
    ref = C.byref
    rot = dict(table=1 << 20, q=1 << 20, q_out=1 << 24)
    ap = lambda **k: L.hbl_kv_append(ref(cache_t()), ref(batch_t()), append_t(**rot, **k), N)
    assert ap(q_out_token_stride=0) == 2 and ap(q_out_head_stride=0) == 2 and ap(q_out_head_stride=120) == 2
    assert ap(q_out_token_stride=512, q_out_head_stride=512) == 2
    at = lambda **k: L.hbl_attention(ref(cache_t()), ref(batch_t()), attention_t(**k), P, 1 << 40, N)
    assert at(out_token_stride=0) == 2 and at(out_head_stride=0) == 2 and at(out_head_stride=64) == 2
    assert at(out_token_stride=512, out_head_stride=512) == 2


def test_very_long_sequences_are_split(L):
    # a piece stays far below what the kernel's bounded waits allow for
    ref = C.byref
    cache = cache_t(n_pages=262144, page_size=4096, n_kv_heads=1)
    need = lambda n: L.hbl_attention_workspace_bytes(ref(cache), ref(batch_t(tokens=65536, max_q_len=65536, n_seqs=1, max_pages=262144, max_kv_len=n)), 4)
    assert need(1 << 24) == 0
    for pieces in (2, 64):
        rows = pieces * 65536 * 4
        assert need(pieces << 24) == rows * 128 * 4 + rows * 4
