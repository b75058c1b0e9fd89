"""64-bit reference of the attention within a window, with the tolerances that states_ref.py (bf16) and codes_bound.py (codes)
derive: the sums are no longer than those of the whole sequence, so their bounds hold.  What the weights are held against, max vs and
max |v|, is that of the keys that some row of the sequence sees."""
import math

import torch

from codes_bound import bound
from paper_2504_18415_b200 import hbl
from states_ref import F8, sequence_values


def visible(nq, nk, window, sinks, device="cuda"):
    """[nq, nk]: which tokens the last nq of nk see."""
    i = torch.arange(nk - nq, nk, device=device)[:, None]
    j = torch.arange(nk, device=device)[None]
    return (j <= i) & ((j > i - window) | (j < sinks))


def window64(cache, q, q_lens, kv_lens, tables, window, sinks, sm_scale=None, slots=None):
    """(out, lse, tolerance of out, tolerance of lse), row for row, in fp64."""
    T, H, D = q.shape
    sm_scale = D ** -0.5 if sm_scale is None else sm_scale
    group, dev = H // cache.n_kv_heads, q.device
    out, tol = torch.zeros(T, H, D, dtype=F8, device=dev), torch.zeros(T, H, D, dtype=F8, device=dev)
    lse, tol_lse = torch.full((T, H), -math.inf, dtype=F8, device=dev), torch.zeros(T, H, dtype=F8, device=dev)
    at = 0
    for b, (nq, nk) in enumerate(zip(q_lens, kv_lens)):
        slot8 = None if cache.bos_k is None else (slots[b] if slots is not None else b)
        r = slice(at, at + nq)
        at += nq
        if not nq or not nk:
            continue
        mask = visible(nq, nk, window, sinks)
        pages = torch.as_tensor(tables[b], device=dev).clamp(0, cache.n_pages - 1)            # (what no row sees may lie anywhere)
        for h in range(cache.n_kv_heads):
            k, v = (sequence_values(cache, n, pages, nk, h, slot8) for n in "kv")
            k, v = (torch.where(mask.any(0)[:, None], x, torch.zeros_like(x)) for x in (k, v))
            x = q[r, h * group:(h + 1) * group].to(F8).transpose(0, 1)                        # [group, nq, D]
            s = (x @ k.T * sm_scale).masked_fill(~mask, -math.inf)
            size = ((x.abs() @ k.abs().T) * abs(sm_scale)).masked_fill(~mask, 0).amax(-1)     # largest sum of magnitudes
            z = torch.logsumexp(s, -1)
            p = torch.where(mask, torch.exp(s - z[..., None]), torch.zeros_like(s))           # rows that see nothing: 0
            o = p @ v
            e_s = (D + 4) * 2.0 ** -23 * size
            steps = (nk / 16 + 64) * 2.0 ** -23
            e = 2 * e_s + steps + 2.0 ** -20
            if cache.bits == 16:
                t = 2.0 ** -8 * o.abs() + (2.0 ** -8 + e)[..., None] * (p @ v.abs()) * 1.01 + 1e-30
            else:
                at_key = torch.arange(nk, device=dev)
                scales = torch.where(mask.any(0), cache.v_scale[pages[at_key // cache.page_size].long(), h, at_key % cache.page_size], 0.0)
                t = bound(o, p @ v.abs(), e[..., None], nk, v.abs().max(), 0.0 if slot8 is None else scales.max()) * 1.01
            hh = slice(h * group, (h + 1) * group)
            out[r, hh], tol[r, hh], lse[r, hh] = o.transpose(0, 1), t.transpose(0, 1), z.T
            tol_lse[r, hh] = (e_s + steps + 2.0 ** -20 * (1 + z.abs())).T
    return out, lse, tol, tol_lse


def check_window(cache, batch, tables, q_lens, kv_lens, q, window, sinks, sm_scale=None, slots=None, **kw):
    T, H, D = q.shape
    out = torch.full((T, H, D), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 77.0, device="cuda")
    hbl.hbl_attention_window(cache, batch, q, window, sinks, sm_scale=sm_scale, out=out, lse=lse, **kw)
    assert hbl.hbl_check_status() == 0
    n = sum(q_lens)
    ref, z, tol, tol_z = window64(cache, q[:n], q_lens, kv_lens, tables, window, sinks, sm_scale, slots)
    err = (out[:n].to(F8) - ref).abs()
    assert not torch.isnan(out[:n]).any()
    assert (err <= tol).all(), f"out: {(err / tol).max().item():.3f} of the tolerance"
    empty = torch.isinf(z)
    assert torch.equal(empty, torch.isinf(lse[:n]) & (lse[:n] < 0)), "rows that see nothing"
    assert (out[:n][empty] == 0).all()
    dz = (lse[:n].to(F8) - z).abs()[~empty]
    assert (dz <= tol_z[~empty]).all(), f"lse: {(dz / tol_z[~empty]).max().item():.3f} of the tolerance"
    assert (out[n:] == 77).all() and (lse[n:] == 77).all(), "rows behind the last sequence"
    return out, lse
