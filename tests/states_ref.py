"""64-bit references and builders for the tests of rotary positions, the paged cache and the attention over it.

Tolerances are derived, not tuned.  A rounding to bf16 is off by at most 2^-8 of the value (half a step).  An output of
the attention is rounded once to bf16, and each p_j (times the value row's scale) once before it is multiplied, so

    |out - ref| <= 2^-8 |ref| + (2^-8 + e) A,      A = sum_j p_j |v_j| / sum_j p_j,

where e collects what fp32 adds: the scores, sums of head_dim products, are off by at most (head_dim + 4) 2^-23 times the
sum of the products' magnitudes, which moves p by that factor and p's sum with it (twice); N additions to an
accumulator by at most N 2^-23 of A; 2^-20 covers exp2, the scales' products and the division.

Codes: where p_j vs_j goes through fp16 instead (2^-12 of the value), it is held as p_j vs_j / vr * 2^7 with vr the power
of two above the largest value scale, vr <= 2 max vs, and below 2^-14 fp16 has a fixed step of 2^-24: a weight is then off by
at most 2^-25 2^-7 vr <= 2^-31 max vs.  p's sum is at least 1 (the maximum is one of the scores), a code is at most
2^(b-1) <= 4/3 of what makes max |v| out of max vs, so n keys add at most n 2^-30 max |v|.
"""
import math

import torch

from paper_2504_18415_b200 import hbl

F8 = torch.float64


def rotate64(x, table, positions, interleaved=False, backward=False):
    """x [T, H, D] fp64, table fp32 [n_pos, half, 2]."""
    half = table.shape[1]
    rows = table.to(F8)[positions.long()]
    c, s = rows[:, None, :, 0], rows[:, None, :, 1]
    if backward:
        s = -s
    x = x.to(F8).clone()
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    x1, x2 = x[..., a].clone(), x[..., b].clone()
    x[..., a] = c * x1 - s * x2
    x[..., b] = c * x2 + s * x1
    return x


def decode(packed, bits, D):
    """uint8 [..., D * bits / 8] -> int64 codes [..., D]."""
    bit = (packed.long()[..., None] >> torch.arange(8, device=packed.device)) & 1
    return (bit.flatten(-2).unflatten(-1, (D, bits)) << torch.arange(bits, device=packed.device)).sum(-1)


def row_values(cache, which, page, head, slot):
    """The fp64 value of one or more rows of a cache, as its layout says."""
    x = (cache.k if which == "k" else cache.v)[page, head, slot]
    if cache.bits == 16:
        return x.to(F8)
    scale = (cache.k_scale if which == "k" else cache.v_scale)[page, head, slot]
    return (decode(x, cache.bits, cache.head_dim) - 2 ** (cache.bits - 1)).to(F8) * scale.to(F8)[..., None]


def sequence_values(cache, which, pages, length, head, slot8=None):
    """fp64 [length, D]: a sequence's rows of one head, page by page."""
    pos = torch.arange(length, device=cache.k.device)
    ids = torch.as_tensor(pages, device=cache.k.device)[pos // cache.page_size].long()
    x = row_values(cache, which, ids, head, pos % cache.page_size)
    if slot8 is not None and length > 0:
        codes = (cache.bos_k if which == "k" else cache.bos_v)[slot8, head]
        scale = (cache.bos_k_scale if which == "k" else cache.bos_v_scale)[slot8, head]
        x[0] = (codes.to(F8) - 128) * scale.to(F8)
    return x


def attention64(cache, q, q_lens, kv_lens, tables, sm_scale, causal, slots=None):
    """(out, lse, tolerance of out, tolerance of lse), row for row, in fp64."""
    T, H, D = q.shape
    group = H // cache.n_kv_heads
    dev = q.device
    out, tol = torch.zeros(T, H, D, dtype=F8, device=dev), torch.zeros(T, H, D, dtype=F8, device=dev)
    lse, tol_lse = torch.full((T, H), -math.inf, dtype=F8, device=dev), torch.zeros(T, H, dtype=F8, device=dev)
    at = 0
    for b, (nq, nk) in enumerate(zip(q_lens, kv_lens)):
        slot8 = None if cache.bos_k is None else (slots[b] if slots is not None else b)
        for h in range(cache.n_kv_heads if nq and nk else 0):
            k = sequence_values(cache, "k", tables[b], nk, h, slot8)
            v = sequence_values(cache, "v", tables[b], nk, h, slot8)
            seen = torch.arange(nq, device=dev) + (nk - nq) if causal else torch.full((nq,), nk - 1, device=dev)
            mask = torch.arange(nk, device=dev)[None] <= seen[:, None]
            for g in range(group):
                x = q[at:at + nq, h * group + g].to(F8)
                s = (x @ k.T * sm_scale).masked_fill(~mask, -math.inf)
                size = ((x.abs() @ k.abs().T) * abs(sm_scale)).masked_fill(~mask, 0).amax(-1)     # largest sum of magnitudes
                z = torch.logsumexp(s, -1)
                p = torch.exp(s - z[:, None])
                p = torch.where(mask.any(-1)[:, None] & mask, p, torch.zeros_like(p))             # rows that see nothing: 0
                r = slice(at, at + nq)
                hh = h * group + g
                clean = torch.where(mask.any(0)[:, None], v, torch.zeros_like(v))                 # (a row nobody sees may hold anything)
                out[r, hh] = p @ clean
                lse[r, hh] = z
                e_s = (D + 4) * 2.0 ** -23 * size
                steps = (nk / 16 + 64) * 2.0 ** -23
                e = 2 * e_s + steps + 2.0 ** -20
                tol[r, hh] = 2.0 ** -8 * out[r, hh].abs() + (2.0 ** -8 + e)[:, None] * (p @ clean.abs()) * 1.01 + 1e-30
                if cache.bits < 16:
                    tol[r, hh] += nk * 2.0 ** -30 * clean.abs().max()
                tol_lse[r, hh] = e_s + steps + 2.0 ** -20 * (1 + z.abs())
        at += nq
    return out, lse, tol, tol_lse


def heads(gen, rows, n, D, outliers=True):
    """Heads as projections give them: near Gaussian with a few large channels."""
    x = torch.randn(rows, n, D, device="cuda", generator=gen)
    if outliers:
        x = x * (1 + 9 * (torch.rand(n, D, device="cuda", generator=gen) < 0.01))
    return x.to(torch.bfloat16)


def make_batch(gen, cache, q_lens, kv_lens, max_pages=None, extra_rows=0, slots=None):
    """Pages dealt at random; returns (batch, page lists)."""
    need = [-(-n // cache.page_size) for n in kv_lens]
    assert sum(need) <= cache.n_pages
    ids = torch.randperm(cache.n_pages, device="cuda", generator=gen).tolist()
    width = max(max(need), 1) if max_pages is None else max_pages
    tables, at = [], 0
    rows = torch.full((len(need), width), -7, dtype=torch.int32)            # entries beyond a sequence's length: nonsense
    for b, n in enumerate(need):
        tables.append(ids[at:at + n])
        rows[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
        at += n
    start = [0]
    for n in q_lens:
        start.append(start[-1] + n)
    slot_t = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    batch = hbl.KvBatch(torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor(kv_lens, dtype=torch.int32, device="cuda"),
                        rows.cuda(), tokens=start[-1] + extra_rows, max_q_len=max(q_lens, default=0), max_kv_len=max(kv_lens, default=0),
                        bos_slot=slot_t)
    return batch, tables


def fill(gen, cache):
    """Random contents, put in by hand (not by the library's append)."""
    shape = cache.k.shape[:3]
    for x, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        if cache.bits == 16:
            x.copy_(heads(gen, shape[0] * shape[2], shape[1], cache.head_dim).reshape(shape[0], shape[2], shape[1], -1).transpose(1, 2))
        else:
            u = torch.randint(1, 2 ** cache.bits, (*shape, cache.head_dim), device="cuda", generator=gen)
            bit = (u[..., None] >> torch.arange(cache.bits, device="cuda")) & 1
            x.copy_((bit.flatten(-2).unflatten(-1, (-1, 8)) << torch.arange(8, device="cuda")).sum(-1).to(torch.uint8))
            scale.copy_((0.5 + torch.rand(shape, device="cuda", generator=gen)) * 2.5 / 2 ** (cache.bits - 1))
    if cache.bos_k is not None:
        for x, scale in ((cache.bos_k, cache.bos_k_scale), (cache.bos_v, cache.bos_v_scale)):
            x.copy_(torch.randint(1, 256, x.shape, device="cuda", generator=gen).to(torch.uint8))
            scale.copy_((0.5 + torch.rand(scale.shape, device="cuda", generator=gen)) * 0.03)


def check_attention(cache, batch, tables, q_lens, kv_lens, q, causal=True, sm_scale=None, slots=None, **kw):
    T, H, D = q.shape
    out = torch.full((T, H, D), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 77.0, device="cuda")
    hbl.hbl_attention(cache, batch, q, sm_scale=sm_scale, causal=causal, out=out, lse=lse, **kw)
    assert hbl.hbl_check_status() == 0
    n = sum(q_lens)
    ref, z, tol, tol_z = attention64(cache, q[:n], q_lens, kv_lens, tables, D ** -0.5 if sm_scale is None else sm_scale, causal, slots)
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
