"""Strides of outputs: heads that lie on each other are refused, whatever pair of tokens they belong to.  No GPU: every call
has a second fault, an address that is not aligned, which is found after the strides (5), so nothing is ever launched."""
import ctypes as C
import random

import pytest

from paper_2504_18415_b200 import build, hbl
from test_states_cpu import Rope, append_t, attention_t, batch_t, cache_t


@pytest.fixture(scope="module")
def L():
    build.build()
    return hbl.lib()


def rope(L, ts, hs, tokens, heads, D=16):
    """Status of hbl_rope with an output of these strides: 2 where it is refused, 5 where it is not."""
    return L.hbl_rope(bytes(Rope(1024, 1 << 30, 1026, 1024, 0, 0, ts, hs, 1, tokens, heads, D, 16, 16, 0, 0)), C.c_void_p(0))


def overlap(ts, hs, tokens, heads, D):
    at = sorted(t * ts + h * hs for t in range(tokens) for h in range(heads))
    return any(b - a < D for a, b in zip(at, at[1:]))


def test_a_head_of_the_next_token(L):
    assert rope(L, 32, 16, 8, 3) == 2                          # head 2 of a token is head 0 of the next one
    assert rope(L, 32, 16, 8, 2) == 5 and rope(L, 48, 16, 8, 3) == 5
    assert rope(L, 16, 32, 3, 8) == 2 and rope(L, 16, 48, 3, 8) == 5
    assert rope(L, 40, 16, 8, 3) == 2                          # half of it
    assert rope(L, 48, 32, 2, 2) == 5                          # 0, 48 and 32, 80: apart, though neither lies between the other's
    assert rope(L, 48, 32, 3, 4) == 2
    assert rope(L, 1 << 60, 1 << 59, 1 << 20, 3) == 2 and rope(L, 1 << 60, 1 << 40, 1 << 30, 1 << 10) == 5


def test_every_small_layout(L):
    rnd = random.Random(1)
    seen = set()
    for _ in range(4000):
        D = rnd.choice([16, 32])
        ts, hs, tokens, heads = 8 * rnd.randint(0, 40), 8 * rnd.randint(0, 40), rnd.randint(1, 9), rnd.randint(1, 9)
        want = overlap(ts, hs, tokens, heads, D)
        seen.add(want)
        assert rope(L, ts, hs, tokens, heads, D) == (2 if want else 5), (ts, hs, tokens, heads, D)
    assert seen == {True, False}


def test_the_other_outputs(L):
    ref, N = C.byref, C.c_void_p(0)
    batch = ref(batch_t())
    out = lambda ts: L.hbl_attention(ref(cache_t()), batch, attention_t(out_token_stride=ts, out_head_stride=128, lse=(1 << 20) + 2), C.c_void_p(1024), 1 << 40, N)
    assert out(256) == 2 and out(512) == 5
    q = dict(table=1 << 20, q=1 << 20, q_out=1 << 24, q_out_head_stride=128, positions=(1 << 20) + 1)
    app = lambda ts: L.hbl_kv_append(ref(cache_t()), batch, append_t(**q, q_out_token_stride=ts), N)
    assert app(256) == 2 and app(512) == 5
