"""Argument checks of the norm, its gradients, the normalising append and the attention within a window: no GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2504_18415_b200 import build, hbl
from test_states_cpu import BAD_BATCHES, BAD_CACHES, append_t, attention_t, batch_t, cache_t, fields, strides


@pytest.fixture(scope="module")
def L():
    build.build()
    return hbl.lib()


P, N = C.c_void_p(1024), C.c_void_p(0)          # P is never dereferenced on the host: validation must stop first


class Part(C.Structure):                        # the argument structures as include/hbl.h declares them
    _fields_ = fields((C.c_void_p, "x gain out"), (C.c_longlong, "x_token_stride x_head_stride out_token_stride out_head_stride"))


class Norm(C.Structure):
    _fields_ = [("q", Part), ("k", Part)] + fields((C.c_void_p, "positions table"),
                                                   (C.c_int, "n_q_heads n_k_heads dtype gain_dtype tokens head_dim n_pos rot_dim layout"), (C.c_float, "norm_eps"))


class Grad(C.Structure):
    _fields_ = [("forward", Norm)] + fields((C.c_void_p, "q_grad k_grad q_grad_gain k_grad_gain"), (C.c_longlong, strides("q_grad k_grad")))


class HeadNorm(C.Structure):
    _fields_ = fields((C.c_void_p, "q_gain k_gain"), (C.c_int, "gain_dtype"), (C.c_float, "norm_eps"))


def norm_t(kind=Norm, **k):
    a = kind()
    f = a.forward if kind is Grad else a
    for i, p in enumerate((f.q, f.k)):
        p.x, p.gain, p.out = (2 + i) << 20, 1 << 10, (4 + i) << 20
        p.x_token_stride = p.out_token_stride = 1024
        p.x_head_stride = p.out_head_stride = 128
    f.positions = f.table = 1 << 10
    f.n_q_heads, f.n_k_heads, f.dtype, f.gain_dtype, f.tokens, f.head_dim, f.n_pos, f.rot_dim, f.layout, f.norm_eps = 8, 2, 1, 1, 4, 128, 16, 128, 0, 1e-6
    if kind is Grad:
        a.q_grad, a.k_grad, a.q_grad_gain, a.k_grad_gain = 6 << 20, 7 << 20, 1 << 11, 1 << 12
        a.q_grad_token_stride = a.k_grad_token_stride = 1024
        a.q_grad_head_stride = a.k_grad_head_stride = 128
    for n, v in k.items():
        at, _, field = n.partition("__")
        if at in ("q", "k") and field:
            setattr(getattr(f, at), field, v)
        else:
            setattr(a if n in dict(getattr(kind, "_fields_")) else f, n, v)
    return bytes(a)


BAD_NORMS = [(dict(dtype=2), 10), (dict(gain_dtype=2), 10), (dict(layout=2), 10), (dict(tokens=-1), 2), (dict(n_q_heads=0), 2), (dict(n_k_heads=-1), 2),
             (dict(n_q_heads=(1 << 20) + 1), 11), (dict(n_k_heads=(1 << 20) + 1), 11), (dict(head_dim=12), 2), (dict(head_dim=264), 2), (dict(head_dim=0), 2),
             (dict(rot_dim=24), 2), (dict(rot_dim=0), 2), (dict(rot_dim=144), 2), (dict(n_pos=0), 2), (dict(norm_eps=-1e-9), 7), (dict(norm_eps=math.nan), 7),
             (dict(norm_eps=math.inf), 7), (dict(positions=0), 1), (dict(positions=(1 << 10) + 2), 5), (dict(table=(1 << 10) + 8), 5),
             (dict(q__x=0), 1), (dict(q__out=0), 1), (dict(k__x=0), 1), (dict(k__out=0), 1), (dict(q__x=(2 << 20) + 8), 5), (dict(k__out=(5 << 20) + 8), 5),
             (dict(q__gain=(1 << 10) + 8), 5), (dict(k__gain=(1 << 10) + 4), 5), (dict(q__x_token_stride=1028), 5), (dict(k__x_head_stride=-128), 2),
             (dict(q__out_token_stride=0), 2), (dict(q__out_head_stride=0), 2), (dict(k__out_head_stride=120), 2), (dict(q__out_token_stride=512), 2),
             (dict(q__out=2 << 20, q__out_token_stride=2048), 2),                # in place, other strides
             (dict(k__out=4 << 20), 2)]                                          # one output for both


def test_norm_refusals(L):
    call = lambda **k: L.hbl_norm_rope(norm_t(**k), N)
    assert L.hbl_norm_rope(None, N) == 1
    for k, want in BAD_NORMS:
        assert call(**k) == want, k
    assert call(tokens=0, q__x=0, q__out=0, positions=0) == 0                    # nothing to do
    assert call(tokens=0, dtype=3) == 10


def test_gradient_refusals(L):
    call = lambda ws=P, n=1 << 30, **k: L.hbl_norm_rope_grad(norm_t(Grad, **k), ws, n, N)
    assert L.hbl_norm_rope_grad(None, P, 1 << 30, N) == 1
    for k, want in BAD_NORMS:
        assert call(**k) == want, k
    assert call(q_grad=0) == 1 and call(k_grad=0) == 1 and call(q_grad=(6 << 20) + 8) == 5 and call(k_grad_token_stride=4) == 5
    assert call(q_grad_head_stride=-8) == 2 and call(q_grad_gain=(1 << 11) + 2) == 5
    assert call(q_grad=4 << 20, q_grad_token_stride=2048) == 2                   # over the gradient, other strides
    assert call(k_grad_gain=1 << 11) == 2                                        # one sum for both gains
    need = L.hbl_norm_rope_grad_workspace_bytes(4, 8, 2, 128)
    assert need > 0 and need % 1024 == 0
    assert call(ws=N) == 1 and call(ws=C.c_void_p(1536)) == 5 and call(n=need - 1) == 6
    for bad in ((0, 8, 2, 128), (4, 0, 2, 128), (4, 8, -1, 128), (4, 8, 2, 100), (4, 8, 2, 512), (-1, 8, 2, 128)):
        assert L.hbl_norm_rope_grad_workspace_bytes(*bad) == 0


def test_normalising_append_refusals(L):
    ref = C.byref
    norm = lambda **k: bytes(HeadNorm(*[dict(dict(q_gain=1 << 10, k_gain=1 << 10, gain_dtype=1, norm_eps=1e-6), **k)[n] for n, _ in HeadNorm._fields_]))
    call = lambda c=cache_t(), b=batch_t(), a=append_t(), n=norm(): L.hbl_kv_append_norm(ref(c), ref(b), a, n, N)
    assert call(n=None) == 1 and call(a=None) == 1
    assert L.hbl_kv_append_norm(None, ref(batch_t()), append_t(), norm(), N) == 1 and L.hbl_kv_append_norm(ref(cache_t()), None, append_t(), norm(), N) == 1
    for k, want in BAD_CACHES:
        assert call(c=cache_t(**k)) == want, k
    for k, want in BAD_BATCHES:
        assert call(b=batch_t(**k)) == want, k
    assert call(b=batch_t(n_seqs=0)) == 0
    assert call(n=norm(gain_dtype=5)) == 10 and call(n=norm(norm_eps=-1.0)) == 7 and call(n=norm(norm_eps=math.nan)) == 7 and call(n=norm(norm_eps=math.inf)) == 7
    assert call(n=norm(q_gain=(1 << 10) + 8)) == 5 and call(n=norm(k_gain=(1 << 10) + 2)) == 5
    for k, want in [(dict(eps=0.0), 7), (dict(k=0), 1), (dict(v=0), 1), (dict(k=(1 << 20) + 8), 5), (dict(q=1 << 20), 1),
                    (dict(q=1 << 20, q_out=1 << 24, q_out_token_stride=0), 2), (dict(q=1 << 20, q_out=1 << 20, q_token_stride=1024), 2),
                    (dict(table=1 << 20, rot_dim=8), 2), (dict(positions=(1 << 20) + 1), 5)]:
        assert call(a=append_t(**k)) == want, k


def test_window_refusals(L):
    ref = C.byref
    call = lambda c=cache_t(), b=batch_t(), w=64, s=4, ws=P, n=1 << 40, **k: L.hbl_attention_window(ref(c), ref(b), attention_t(**k), w, s, ws, n, N)
    assert call(w=0) == 2 and call(w=-5) == 2 and call(s=-1) == 2 and call(causal=0) == 2
    assert L.hbl_attention_window(None, ref(batch_t()), attention_t(), 64, 4, P, 1 << 40, N) == 1
    assert L.hbl_attention_window(ref(cache_t()), ref(batch_t()), None, 64, 4, P, 1 << 40, N) == 1
    for k, want in BAD_CACHES:
        assert call(c=cache_t(**k)) == want, k
    for k, want in BAD_BATCHES:
        assert call(b=batch_t(**k)) == want, k
    assert call(b=batch_t(n_seqs=0)) == 0 and call(b=batch_t(max_q_len=0)) == 0
    assert call(n_heads=6) == 2 and call(sm_scale=math.nan) == 2 and call(q=0) == 1 and call(out=0) == 1 and call(out_head_stride=64) == 2
    size = L.hbl_attention_window_workspace_bytes
    long = batch_t(max_kv_len=65536, max_pages=4096)
    assert size(ref(cache_t()), ref(long), 4, 0, 4) == 0 and size(ref(cache_t()), ref(long), 4, 64, -1) == 0 and size(ref(cache_t()), ref(long), 6, 64, 4) == 0
    assert size(ref(cache_t()), ref(long), 4, 64, 4) == 0                        # a short window is not split
    need = size(ref(cache_t()), ref(long), 4, 30000, 4)
    assert 0 < need <= L.hbl_attention_workspace_bytes(ref(cache_t()), ref(long), 4)
    assert size(ref(cache_t()), ref(long), 4, 2 ** 31 - 1, 2 ** 31 - 1) == L.hbl_attention_workspace_bytes(ref(cache_t()), ref(long), 4)
    assert call(b=long, w=30000, ws=N, n=0) == 1 and call(b=long, w=30000, n=need - 1) == 6 and call(b=long, w=30000, ws=C.c_void_p(1536)) == 5


@pytest.mark.parametrize("kind,packed", [(Norm, hbl._NORM_ROPE_T), (HeadNorm, hbl._HEAD_NORM_T)])
def test_packed_arguments_are_the_structures_of_the_header(kind, packed):
    assert packed.size == C.sizeof(kind)
    plain = []

    def walk(s):
        for n, t in s._fields_:
            if issubclass(t, C.Structure):
                yield from walk(t)
            else:
                yield t

    types = list(walk(kind))
    values = [0.5 + i if t is C.c_float else 1 + i for i, t in enumerate(types)]
    got = kind.from_buffer_copy(packed.pack(*values))

    def read(s):
        for n, t in s._fields_:
            if issubclass(t, C.Structure):
                read(getattr(s, n))
            else:
                plain.append(getattr(s, n))

    read(got)
    assert plain == values
    assert hbl._NORM_ROPE_T.size + hbl._NORM_GRAD_T.size == C.sizeof(Grad)


def test_binding_refuses_what_is_not_on_the_gpu():
    z = torch.zeros(1, 1, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        hbl.hbl_norm_rope(z, None, None, None)
    with pytest.raises(ValueError):
        hbl.hbl_norm_rope_grad(z, z, None, None, None)
    with pytest.raises(ValueError):
        hbl.hbl_norm_rope_grad(z, z, None, None, None, k=z)
