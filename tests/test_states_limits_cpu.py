"""Sizes beyond what the attention call takes: refused on the host.  No GPU."""
import ctypes as C

from paper_2504_18415_b200 import build, hbl
from test_states_cpu import attention_t, batch_t, cache_t


def test_more_heads_than_there_can_be():
    build.build()
    L, ref, N = hbl.lib(), C.byref, C.c_void_p(0)
    cache, batch = ref(cache_t(n_kv_heads=1)), ref(batch_t(tokens=1, n_seqs=1))
    for n in ((1 << 20) + 1, 1 << 30, (1 << 30) + 1, 0x7fffffff):
        assert L.hbl_attention(cache, batch, attention_t(n_heads=n), C.c_void_p(1024), 1 << 62, N) == 11
        assert L.hbl_attention_workspace_bytes(cache, batch, n) == 0
