"""The attention over a cache of codes against 64 bits, with the bound that its own roundings give.

states_ref.py bounds both kinds of cache by what the coarser one needs: weights rounded to bf16, 2^-8 of their value.  Over codes
a weight p_j vs_j is rounded to fp16, whose half step is 2^-11 of the value (eps / 2 = 2^-10 / 2), and a code is exact, so

    |out - ref| <= 2^-8 |ref| + (2^-11 + e) A + n 2^-30 max |v|,      A = sum_j p_j |v_j| / sum_j p_j,

with the output's own rounding to bf16, e for what fp32 adds, and the fixed step of fp16 below 2^-14, each as derived there.
That step is at most 2^-31 max vs in a weight; n 2^-30 max |v| counts codes of at most 2^(b-1).  A first token kept at 8 bits
has codes of up to 2^7, so it adds 2^-24 max vs.
"""
import math

import torch

from states_ref import F8, sequence_values

FP16_HALF_STEP = torch.finfo(torch.float16).eps / 2
BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def bound(ref, A, e, n, v_max, first_scale=0.0):
    return BF16_HALF_STEP * ref.abs() + (FP16_HALF_STEP + e) * A + n * 2.0 ** -30 * v_max + 2.0 ** -24 * first_scale + 1e-30


def attention_codes64(cache, q, q_lens, kv_lens, tables, sm_scale, causal=True, slots=None):
    """(out, tolerance) of every row in fp64; every row sees a key."""
    T, H, D = q.shape
    group, dev = H // cache.n_kv_heads, q.device
    out, tol = torch.zeros(T, H, D, dtype=F8, device=dev), torch.zeros(T, H, D, dtype=F8, device=dev)
    at = 0
    for b, (nq, nk) in enumerate(zip(q_lens, kv_lens)):
        slot8 = None if cache.bos_k is None else (slots[b] if slots is not None else b)
        seen = torch.arange(nq, device=dev) + (nk - nq) if causal else torch.full((nq,), nk - 1, device=dev)
        mask = torch.arange(nk, device=dev)[None] <= seen[:, None]
        for h in range(H):
            k = sequence_values(cache, "k", tables[b], nk, h // group, slot8)
            v = sequence_values(cache, "v", tables[b], nk, h // group, slot8)
            x = q[at:at + nq, h].to(F8)
            s = (x @ k.T * sm_scale).masked_fill(~mask, -math.inf)
            size = ((x.abs() @ k.abs().T) * abs(sm_scale)).masked_fill(~mask, 0).amax(-1)
            p = torch.softmax(s, -1)
            e = 2 * (D + 4) * 2.0 ** -23 * size + (nk / 16 + 64) * 2.0 ** -23 + 2.0 ** -20
            r = slice(at, at + nq)
            out[r, h] = p @ v
            vs = cache.v_scale[torch.as_tensor(tables[b], device=dev).long(), h // group].max()
            tol[r, h] = bound(out[r, h], p @ v.abs(), e[:, None], nk, v.abs().max(), vs if slot8 is not None else 0.0)
        at += nq
    return out, tol
