"""Operators of the paged low-bit cache of attention states: what is measured, and their plain forms.

Three operators take the projections of a decoder block (W_q, W_k, W_v) to the input of W_o:

  rope       rotary positions on the heads of a tensor, and their backward pass;
  append     the new tokens' keys (rotated on the way) and values go into the pages of a cache, quantized per head
             to 3, 4 or 8 bits or kept in bf16; the queries are rotated by the same call;
  attention  the queries of the new tokens, one or many per sequence, over all tokens the cache holds.

Cache: pages of `page` tokens, [page][kv head][slot][row].  A row is a head's codes as a little-endian bit string
(u = q + 2^(bits-1)) with one fp32 scale per row, or bf16 values.  The first token of a sequence may be kept at 8 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # one decoding step of 16 sequences of a 7B-shaped model (32 heads of 128): latency counts
        dict(name="rope_step", op="rope", tokens=16, heads=32, dim=128, rot=128, dtype="bf16", interleaved=False, backward=False, context=4096),
        # queries of a large prefill batch of the same model
        dict(name="rope_prefill", op="rope", tokens=16384, heads=32, dim=128, rot=128, dtype="bf16", interleaved=False, backward=False, context=16384),
        # the backward pass on an fp32 gradient: odd token count, neighbouring pairs, half of the head, far positions
        dict(name="rope_backward", op="rope", tokens=3333, heads=20, dim=128, rot=64, dtype="f32", interleaved=True, backward=True, context=131072),
        # one decoding step of 64 sequences, 4-bit cache
        dict(name="append_step", op="append", seqs=64, q_len=1, kv_len=4096, heads=32, kv_heads=32, dim=128, bits=4, page=64, ragged=True, bos=False,
             interleaved=False, rot=128, context=4096),
        # four prompts of the training length, 3-bit cache with the first token at 8 bits
        dict(name="append_prompts", op="append", seqs=4, q_len=2048, kv_len=2048, heads=32, kv_heads=32, dim=128, bits=3, page=64, ragged=False, bos=True,
             interleaved=False, rot=128, context=2048),
        # chunks of uneven lengths onto half-filled sequences, shared key heads, bf16 cache, small pages
        dict(name="append_chunks", op="append", seqs=9, q_len=511, kv_len=3001, heads=16, kv_heads=4, dim=64, bits=16, page=16, ragged=True, bos=False,
             interleaved=True, rot=32, context=4096),
        # one decoding step of a few short sequences: latency counts
        dict(name="step_short", op="attention", seqs=4, q_len=1, kv_len=509, heads=32, kv_heads=32, dim=128, bits=4, page=64, ragged=True, bos=True, causal=True),
        # one decoding step of a full batch, 4-bit cache: bound by the cache's bytes
        dict(name="step_batch", op="attention", seqs=64, q_len=1, kv_len=4096, heads=32, kv_heads=32, dim=128, bits=4, page=64, ragged=True, bos=True, causal=True),
        # one sequence with a very long context, shared key heads, bf16 cache
        dict(name="step_long", op="attention", seqs=1, q_len=1, kv_len=131072, heads=32, kv_heads=8, dim=128, bits=16, page=128, ragged=False, bos=False, causal=True),
        # a chunk of a prompt over what came before it, 8-bit cache
        dict(name="chunk_over_cache", op="attention", seqs=1, q_len=512, kv_len=16384, heads=32, kv_heads=32, dim=128, bits=8, page=64, ragged=False, bos=False, causal=True),
        # uneven chunks, decoding steps among them, small heads, 3-bit cache, small pages
        dict(name="mixed_ragged", op="attention", seqs=13, q_len=333, kv_len=2047, heads=16, kv_heads=4, dim=64, bits=3, page=16, ragged=True, bos=True, causal=True),
        # a whole prompt, bf16 cache: bound by the tensor cores
        dict(name="prompt_8k", op="attention", seqs=1, q_len=8192, kv_len=8192, heads=32, kv_heads=32, dim=128, bits=16, page=128, ragged=False, bos=False, causal=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (16, 16), (16, 4), (16, 2), (8, 8), (20, 4), (7, 1), (64, 8)])
    dim = rng.choice([64, 128, 128, 256])
    if op == "rope":
        return dict(op=op, tokens=_log(rng, 1, 16384 * 32 * 128 // (heads * dim) // 2), heads=heads, dim=dim, rot=rng.choice([dim, dim // 2]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), interleaved=rng.random() < 0.5, backward=rng.random() < 0.5, context=_log(rng, 2048, 131072))
    kind = dict(heads=heads, kv_heads=kv_heads, dim=dim, bits=rng.choice([3, 4, 8, 16]), page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6)
    kind["bos"] = kind["bits"] in (3, 4) and rng.random() < 0.5
    if op == "append":
        seqs = _log(rng, 1, 64)
        q_len = _log(rng, 1, max(1, 8192 * 32 * 128 // (heads * dim * seqs) // 4))
        kv_len = min(131072, q_len + _log(rng, 1, 8192))
        return dict(op=op, seqs=seqs, q_len=q_len, kv_len=kv_len, interleaved=rng.random() < 0.5, rot=rng.choice([dim, dim // 2]), context=kv_len, **kind)
    while True:
        seqs = _log(rng, 1, 96)
        q_len = 1 if rng.random() < 0.4 else _log(rng, 1, 4096)
        kv_len = q_len + _log(rng, 1, 65536)
        # no more bytes and pairs than the largest listed cases, and a plain form that fits the card
        if seqs * kv_len * kv_heads * dim <= 64 * 4096 * 32 * 128 // 2 and seqs * heads * q_len * kv_len * dim <= 32 * 8192 * 8192 * 128 // 4:
            return dict(op=op, seqs=seqs, q_len=q_len, kv_len=kv_len, causal=rng.random() < 0.8, **kind)


# ---- what a case holds -----------------------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, all tokens) of each sequence.  Ragged: the first sequence is the longest, some add one token only."""
    n, q, kv = case["seqs"], case["q_len"], case["kv_len"]
    if not case["ragged"]:
        return [q] * n, [kv] * n
    r = random.Random("%d %d %d" % (n, q, kv))
    qs, kvs = [q], [kv]
    for _ in range(n - 1):
        a = 1 if r.random() < 0.3 else r.randint(1, q)
        qs.append(a)
        kvs.append(a + int((kv - q) * r.random()))
    return qs, kvs


def _pairs(case):
    """Scores that the mask leaves, per head."""
    return sum(q * kv - (q * (q - 1) // 2 if case["causal"] else 0) for q, kv in zip(*_lengths(case)))


def work(case):
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * case["dim"] * size + case["tokens"] * (4 + 4 * case["rot"]), "flops": 3 * n * case["rot"]}
    qs, kvs = _lengths(case)
    row = case["dim"] * case["bits"] // 8 + (0 if case["bits"] == 16 else 4)
    if case["op"] == "append":
        t = sum(qs)
        kv = 2 * t * case["kv_heads"]
        out = kv * row + (0 if case["bits"] == 16 else kv * case["dim"] * 2)   # quantized heads are handed out as values too
        flops = 3 * t * (case["heads"] + case["kv_heads"]) * case["rot"] + (0 if case["bits"] == 16 else 4 * kv * case["dim"])
        return {"bytes": 2 * t * case["heads"] * case["dim"] * 2 + kv * case["dim"] * 2 + out + t * 4 * case["rot"], "flops": flops}
    cache = 2 * case["kv_heads"] * sum(kvs) * row
    rows = sum(qs) * case["heads"]
    return {"bytes": cache + rows * (2 * case["dim"] * 2 + 4), "flops": 4 * case["heads"] * case["dim"] * _pairs(case)}


# ---- inputs ----------------------------------------------------------------------------------------------------

class State:
    pass


def _pack(u, bits):
    """Codes [..., dim] (uint8) -> bytes [..., dim * bits / 8]: a little-endian bit string."""
    if bits == 8:
        return u
    if bits == 4:
        return u[..., 0::2] | (u[..., 1::2] << 4)
    g = u.to(torch.int32).reshape(*u.shape[:-1], -1, 8)
    word = (g << (3 * torch.arange(8, device=u.device, dtype=torch.int32))).sum(-1, dtype=torch.int32)
    return torch.stack([word & 255, (word >> 8) & 255, word >> 16], -1).to(torch.uint8).flatten(-2)


def _codes(x, bits):
    """The absmax quantizer of each row: codes (uint8) and fp32 scale."""
    c = torch.full((), float(2 ** (bits - 1) - 1), device=x.device, dtype=x.dtype)
    gamma = x.abs().amax(-1)
    u = torch.round(x * (c / (gamma + EPS))[..., None]) + 2 ** (bits - 1)
    return u.to(torch.uint8), gamma / c


def _table(case, device):
    """[context, rot / 2, 2] cosines and sines, angles in 64 bits."""
    half = case["rot"] // 2
    freq = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=device), -torch.arange(half, dtype=torch.float64, device=device) / half)
    angle = torch.arange(case["context"], dtype=torch.float64, device=device)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def prepare(case, seed):
    dev = "cuda"
    s = State()
    s.case = case
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dim, heads = case["dim"], case["heads"]

    def heads_of(rows, n, dtype=torch.bfloat16):
        # projections are near Gaussian, with a few channels that are much larger
        x = torch.randn(rows, n, dim, device=dev, generator=g)
        return (x * (1 + 9 * (torch.rand(n, dim, device=dev, generator=g) < 0.01))).to(dtype)

    if case["op"] == "rope":
        s.x = heads_of(case["tokens"], heads, torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        s.table = _table(case, dev)
        s.positions = torch.randint(0, case["context"], (case["tokens"],), device=dev, generator=g, dtype=torch.int32)
        s.out = torch.empty_like(s.x)
        return s

    kv_heads, bits, page = case["kv_heads"], case["bits"], case["page"]
    qs, kvs = _lengths(case)
    n, t = len(qs), sum(qs)
    wide = [-(-kv // page) for kv in kvs]
    n_pages, most = sum(wide) + 3, max(wide)
    ids = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32)      # a sequence's pages lie anywhere
    s.pages = torch.zeros(n, most, dtype=torch.int32, device=dev)
    at = 0
    for b, w in enumerate(wide):
        s.pages[b, :w] = ids[at:at + w]
        at += w
    s.q_start = torch.tensor([sum(qs[:b]) for b in range(n + 1)], dtype=torch.int32, device=dev)
    s.kv_len = torch.tensor(kvs, dtype=torch.int32, device=dev)
    s.tokens, s.max_q, s.max_kv = t, max(qs), max(kvs)
    # where each new token goes
    seq = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(qs, device=dev))
    s.seq = seq
    s.position = (s.kv_len - s.q_start[1:] + s.q_start[:-1])[seq] + torch.arange(t, device=dev, dtype=torch.int32) - s.q_start[seq]
    # the cache, filled
    shape = (n_pages, kv_heads, page)
    s.k_scale = s.v_scale = s.bos = None
    if bits == 16:
        s.k = torch.empty(*shape, dim, dtype=torch.bfloat16, device=dev)
        s.v = torch.empty(*shape, dim, dtype=torch.bfloat16, device=dev)
    else:
        s.k = torch.empty(*shape, dim * bits // 8, dtype=torch.uint8, device=dev)
        s.v = torch.empty(*shape, dim * bits // 8, dtype=torch.uint8, device=dev)
        s.k_scale = torch.empty(*shape, device=dev)
        s.v_scale = torch.empty(*shape, device=dev)
    step = max(1, (1 << 26) // (kv_heads * page * dim))
    for x, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
        for p in range(0, n_pages, step):
            h = heads_of(min(step, n_pages - p) * page, kv_heads).reshape(-1, page, kv_heads, dim).transpose(1, 2)
            if bits == 16:
                x[p:p + step] = h
            else:
                u, scale[p:p + step] = _codes(h.float(), bits)
                x[p:p + step] = _pack(u, bits)
    if case["bos"]:
        s.bos = []
        for _ in range(2):
            s.bos += list(_codes(heads_of(n, kv_heads).float(), 8))           # keys, their scales, values, their scales
    s.q = heads_of(t, heads)
    s.out = torch.zeros_like(s.q)
    s.sm_scale = 1.0 / math.sqrt(dim)
    if case["op"] == "append":
        s.new_k, s.new_v = heads_of(t, kv_heads), heads_of(t, kv_heads)
        s.table = _table(case, dev)
    else:
        s.lse = torch.zeros(t, heads, device=dev)
    s.plan = None
    return s


# ---- the framework's calls ---------------------------------------------------------------------------------------

def _plan(s):
    """The handles that a serving program keeps beside its cache: made once."""
    from paper_2504_18415_b200 import hbl
    if s.plan is None:
        c = s.case
        bos = dict(zip(("bos_k", "bos_k_scale", "bos_v", "bos_v_scale"), s.bos)) if s.bos else {}
        cache = hbl.KvCache(s.k, s.v, s.k_scale, s.v_scale, bits=c["bits"], **bos)
        batch = hbl.KvBatch(s.q_start, s.kv_len, s.pages, tokens=s.tokens, max_q_len=s.max_q, max_kv_len=s.max_kv)
        ws = None
        if c["op"] == "attention":
            ws = hbl.new_workspace(hbl.hbl_attention_workspace_bytes(cache, batch, c["heads"]))
        s.plan = (cache, batch, ws)
    return s.plan


def _run_own(s):
    from paper_2504_18415_b200 import hbl
    c = s.case
    if c["op"] == "rope":
        return hbl.hbl_rope(s.x, s.positions, s.table, interleaved=c["interleaved"], backward=c["backward"], out=s.out)
    cache, batch, ws = _plan(s)
    if c["op"] == "append":
        hbl.hbl_kv_append(cache, batch, s.new_k, s.new_v, table=s.table, interleaved=c["interleaved"], q=s.q, q_out=s.out, eps=EPS)
        if c["bits"] == 16:
            return [s.out, s.k, s.v]
        return [s.out, *hbl.hbl_kv_read(cache, batch), s.k_scale, s.v_scale]
    hbl.hbl_attention(cache, batch, s.q, sm_scale=s.sm_scale, causal=c["causal"], out=s.out, lse=s.lse, workspace=ws)
    return [s.out, s.lse]


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _rotate(x, cos_sin, interleaved, backward):
    """x [T, heads, dim] in 32 bits; cos_sin [T, rot / 2, 2]."""
    half = cos_sin.shape[1]
    c, sn = cos_sin[:, None, :, 0], cos_sin[:, None, :, 1]
    if backward:
        sn = -sn
    r = x[..., :2 * half]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    ra, rb = a * c - b * sn, b * c + a * sn
    r = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([r, x[..., 2 * half:]], -1)


def _unpack(x, bits):
    if bits == 8:
        return x
    if bits == 4:
        return torch.stack([x & 15, x >> 4], -1).flatten(-2)
    b = x.to(torch.int32).reshape(*x.shape[:-1], -1, 3)
    word = b[..., 0] | (b[..., 1] << 8) | (b[..., 2] << 16)
    return ((word[..., None] >> (3 * torch.arange(8, device=x.device, dtype=torch.int32))) & 7).flatten(-2)


def _store(x, scale, pages, s, bits, bos):
    """Quantizes x [T, kv heads, dim] (32 bits), stores codes and scales in the pages; returns the stored values in bf16."""
    u, sc = _codes(x, bits)
    page, slot = pages
    s.cur[page, :, slot] = _pack(u, bits)
    scale[page, :, slot] = sc
    value = (u.float() - 2 ** (bits - 1)) * sc[..., None]
    if bos is not None:
        first = (s.position == 0)[:, None, None]
        u8, sc8 = _codes(x, 8)
        value = torch.where(first, (u8.float() - 128) * sc8[..., None], value)
    return value.to(torch.bfloat16)


def _cached(s, x, scale, bos, dtype):
    """The cache's values by sequence: [n, kv heads, length, dim]."""
    c = s.case
    got = x[s.pages.long()].transpose(1, 2).flatten(2, 3)
    if c["bits"] == 16:
        return got.to(dtype)
    value = (_unpack(got, c["bits"]).to(dtype) - 2 ** (c["bits"] - 1)) * scale[s.pages.long()].transpose(1, 2).flatten(2, 3)[..., None].to(dtype)
    if bos is not None:
        value[:, :, 0] = (bos[0].to(dtype) - 128) * bos[1][..., None].to(dtype)
    return value


def run(state):
    s, c = state, state.case
    if own:
        return _run_own(s)
    if c["op"] == "rope":
        return _rotate(s.x.float(), s.table[s.positions.long()], c["interleaved"], c["backward"]).to(s.x.dtype)
    if c["op"] == "append":
        rows = s.table[s.position.long()]
        q = _rotate(s.q.float(), rows, c["interleaved"], False).to(torch.bfloat16)
        k = _rotate(s.new_k.float(), rows, c["interleaved"], False)
        page = s.pages[s.seq, (s.position // c["page"]).long()].long()
        slot = (s.position % c["page"]).long()
        if c["bits"] == 16:
            s.k[page, :, slot] = k.to(torch.bfloat16)
            s.v[page, :, slot] = s.new_v
            return [q, s.k, s.v]
        s.cur = s.k
        kq = _store(k, s.k_scale, (page, slot), s, c["bits"], s.bos)
        s.cur = s.v
        vq = _store(s.new_v.float(), s.v_scale, (page, slot), s, c["bits"], s.bos)
        return [q, kq, vq, s.k_scale, s.v_scale]
    n, group = len(s.kv_len), c["heads"] // c["kv_heads"]
    k = _cached(s, s.k, s.k_scale, s.bos[0:2] if s.bos else None, torch.float32)
    v = _cached(s, s.v, s.v_scale, s.bos[2:4] if s.bos else None, torch.float32)
    # queries by sequence, padded: [n, kv heads, group * max_q, dim]
    q_len = s.q_start[1:] - s.q_start[:-1]
    i = torch.arange(s.max_q, device=k.device)
    row = (s.q_start[:-1, None] + i).clamp(max=s.tokens - 1).long()
    q = s.q[row].float().reshape(n, s.max_q, c["kv_heads"], group, c["dim"]).permute(0, 2, 3, 1, 4)
    score = (q.flatten(2, 3) @ k.transpose(-1, -2)).mul_(s.sm_scale).unflatten(2, (group, s.max_q))
    j = torch.arange(k.shape[2], device=k.device)
    last = (s.kv_len - q_len)[:, None] + i if c["causal"] else (s.kv_len - 1)[:, None].expand(n, s.max_q)
    hidden = (j > last[..., None]) | (j >= s.kv_len[:, None, None])
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = v.masked_fill((j >= s.kv_len[:, None])[:, None, :, None], 0)
    o = (p.flatten(2, 3) @ v).unflatten(2, (group, s.max_q)) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    at = (s.seq, (torch.arange(s.tokens, device=k.device) - s.q_start[s.seq]).long())
    s.out.copy_(o.permute(0, 3, 1, 2, 4)[at].flatten(1, 2))
    s.lse.copy_(lse.permute(0, 3, 1, 2)[at].flatten(1, 2))
    return [s.out, s.lse]


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    half = case["rot"] // 2 if "rot" in case else 0

    def turned(x, pos, sign=1.0):
        z = x.to(f8)
        w = torch.view_as_complex(s.table[pos.long()].to(f8))[:, None]
        w = w.conj() if sign < 0 else w
        r = z[..., :2 * half].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        r = r if case["interleaved"] else r.transpose(-1, -2)
        r = torch.view_as_real(torch.view_as_complex(r.contiguous()) * w)
        r = r if case["interleaved"] else r.transpose(-1, -2)
        return torch.cat([r.flatten(-2), z[..., 2 * half:]], -1)

    if case["op"] == "rope":
        return turned(s.x, s.positions, -1.0 if case["backward"] else 1.0)

    bits = case["bits"]
    if case["op"] == "append":
        k, v = turned(s.new_k, s.position), s.new_v.to(f8)
        where = [(int(p), int(o)) for p, o in zip(s.pages[s.seq, (s.position // case["page"]).long()].tolist(), (s.position % case["page"]).tolist())]
        page, slot = (torch.tensor(w, device=k.device) for w in zip(*where))
        outs, scales = [turned(s.q, s.position)], []
        for x, buf, scale in ((k, s.k, s.k_scale), (v, s.v, s.v_scale)):
            if bits == 16:
                whole = buf.to(f8)
                whole[page, :, slot] = x
                outs.append(whole)
                continue
            width = torch.where((s.position == 0) & bool(case["bos"]), 8, bits).to(f8)[:, None]
            top = x.abs().max(dim=-1).values
            level = 2 ** (width - 1) - 1
            value = torch.round(x * (level / (top + EPS))[..., None]) * (top / level)[..., None]
            outs.append(value)
            whole = scale.to(f8)
            whole[page, :, slot] = top / (2 ** (bits - 1) - 1)
            scales.append(whole)
        return outs + scales

    qs, kvs = _lengths(case)
    group, kv_heads = case["heads"] // case["kv_heads"], case["kv_heads"]
    out = torch.zeros(s.tokens, case["heads"], case["dim"], dtype=f8, device=s.q.device)
    lse = torch.zeros(s.tokens, case["heads"], dtype=f8, device=s.q.device)

    def head(x, scale, bos, b, h):
        ids = s.pages[b, :-(-kvs[b] // case["page"])].long()
        row = x[ids, h].flatten(0, 1)[:kvs[b]]
        if bits == 16:
            return row.to(f8)
        string = row.to(torch.int64)                                # the codes out of the bytes' bits, one after another
        bit = (string[..., None] >> torch.arange(8, device=row.device)) & 1
        code = (bit.flatten(-2).unflatten(-1, (case["dim"], bits)) << torch.arange(bits, device=row.device)).sum(-1)
        value = (code - 2 ** (bits - 1)).to(f8) * scale[ids, h].flatten()[:kvs[b], None].to(f8)
        if bos is not None:
            value[0] = (bos[0][b, h].to(f8) - 128) * bos[1][b, h].to(f8)
        return value

    at = 0
    for b, (nq, nk) in enumerate(zip(qs, kvs)):
        seen = torch.arange(nq, device=s.q.device) + (nk - nq) if case["causal"] else torch.full((nq,), nk - 1, device=s.q.device)
        mask = torch.arange(nk, device=s.q.device)[None] <= seen[:, None]
        for h in range(kv_heads):
            kk = head(s.k, s.k_scale, s.bos[0:2] if s.bos else None, b, h)
            vv = head(s.v, s.v_scale, s.bos[2:4] if s.bos else None, b, h)
            for g in range(group):
                x = s.q[at:at + nq, h * group + g].to(f8) @ kk.T * s.sm_scale
                x = torch.where(mask, x, torch.full_like(x, -math.inf))
                z = torch.logsumexp(x, -1)
                lse[at:at + nq, h * group + g] = z
                out[at:at + nq, h * group + g] = torch.exp(x - z[:, None]) @ vv
        at += nq
    return [out, lse]
