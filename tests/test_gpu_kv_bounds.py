"""hbl_kv_append with `tokens` as an upper bound: rows behind the last sequence are not used."""
import ctypes as C

import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import heads, make_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [3, 4, 8, 16])
@pytest.mark.parametrize("q_lens,kv_lens,bound", [([1, 1, 3], [1, 30, 3], 64), ([2, 0], [20, 5], 3), ([0, 0], [4, 5], 40), ([300, 40], [300, 90], 4000)])
def test_tokens_beyond_the_sequences_rows(bits, q_lens, kv_lens, bound):
    """The call as a C caller makes it whose `tokens` is the most that a captured step may bring."""
    H, KH, D, page, n = 4, 2, 128, 16, sum(q_lens)
    g = torch.Generator(device="cuda")
    g.manual_seed(bits + n)
    cache, want = (hbl.KvCache.empty(sum(-(-x // page) for x in kv_lens) + 1, page, KH, D, bits) for _ in range(2))
    batch, _ = make_batch(g, cache, q_lens, kv_lens)
    k, v, q = heads(g, n, KH, D), heads(g, n, KH, D), heads(g, n, H, D)
    table = hbl.hbl_rope_table(hbl.hbl_rope_frequencies(D), max(kv_lens))
    q_want = hbl.hbl_kv_append(want, batch, k, v, table=table, q=q)
    big = torch.full((n + 8, H, D), 3.0, dtype=torch.bfloat16, device="cuda")     # the first n rows are the call's
    wide = hbl.KvBatch(batch.q_start, batch.kv_len, batch.pages, tokens=bound, max_q_len=max(q_lens), max_kv_len=max(kv_lens))
    rows = [torch.full((bound, *t.shape[1:]), float("nan"), dtype=t.dtype, device="cuda") for t in (k, v, q)]
    for x, t in zip(rows, (k, v, q)):                                         # (what lies behind is of no account, and may not be there)
        x[:n] = t
    at = [x.data_ptr() for x in rows]
    args = hbl._APPEND_T.pack(*at, big.data_ptr(), *(KH * D, D) * 2, *(H * D, D) * 2, table.data_ptr(), 0, H, table.shape[0], D, 0, 1e-5)
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert hbl.lib().hbl_kv_append(cache.ref, wide.ref, args, stream) == 0
    assert hbl.hbl_check_status() == 0
    assert torch.equal(big[:n], q_want) and (big[n:] == 3).all()
    for a in ("k", "v", "k_scale", "v_scale"):
        if getattr(cache, a) is not None:
            assert torch.equal(getattr(cache, a), getattr(want, a))
