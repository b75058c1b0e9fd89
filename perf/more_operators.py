"""Normalised queries and keys, and attention within a window: what is measured, and the operators' plain forms.

  norm     each query and key head divided by its root mean square, times a gain, and rotated, in one pass:
             o = r R(gain * x),  r = 1 / sqrt(mean_d x^2 + eps)
  grad     the backward pass of that: gradients of the heads and of the two gains
  append   the same on the way into the pages of a low-bit cache: normalised, rotated, quantized, written; queries as well
  window   attention over the cache in which a token sees itself, the window - 1 tokens before it, and the sequence's first
           `sinks` tokens, for decoding steps, chunks and prompts

Cache: pages of `page` tokens, [page][kv head][slot][row].  A row is a head's codes as a little-endian bit string
(u = q + 2^(bits-1)) with one fp32 scale per row, or bf16 values.  The first token of a sequence may be kept at 8 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-5              # of the quantizer
NORM_EPS = 2.0 ** -20   # of the norm: the same number in every type


def listed():
    return [
        # one decoding step of 16 sequences, shared key heads: latency counts
        dict(name="norm_step", op="norm", tokens=16, heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16", gain="bf16", interleaved=False, context=4096),
        # queries and keys of a large batch of prompts
        dict(name="norm_prompts", op="norm", tokens=16384, heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16", gain="bf16", interleaved=False, context=16384),
        # the training step's backward pass over the same number of tokens
        dict(name="grad_batch", op="grad", tokens=16384, heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16", gain="bf16", interleaved=False, context=2048),
        # fp32 gradients: odd token count, neighbouring pairs, half of the head, fp32 gains
        dict(name="grad_f32", op="grad", tokens=3333, heads=20, kv_heads=4, dim=128, rot=64, dtype="f32", gain="f32", interleaved=True, context=131072),
        # one decoding step of 64 sequences, 4-bit cache
        dict(name="append_step", op="append", seqs=64, q_len=1, kv_len=4096, heads=32, kv_heads=8, dim=128, bits=4, page=64, ragged=True, bos=False,
             interleaved=False, rot=128, gain="bf16", context=4096),
        # four prompts of the training length, 3-bit cache with the first token at 8 bits
        dict(name="append_prompts", op="append", seqs=4, q_len=2048, kv_len=2048, heads=32, kv_heads=32, dim=128, bits=3, page=64, ragged=False, bos=True,
             interleaved=False, rot=128, gain="bf16", context=2048),
        # one decoding step of a few short sequences, 8-bit cache: latency counts
        dict(name="window_step_short", op="window", seqs=4, q_len=1, kv_len=509, heads=32, kv_heads=8, dim=128, bits=8, page=64, ragged=True, bos=False,
             window=128, sinks=4),
        # one decoding step of a full batch, 4-bit cache, the first token at 8 bits
        dict(name="window_step_batch", op="window", seqs=64, q_len=1, kv_len=4096, heads=32, kv_heads=32, dim=128, bits=4, page=64, ragged=True, bos=True,
             window=1024, sinks=4),
        # one sequence with a very long context, bf16 cache: only the window is read
        dict(name="window_step_long", op="window", seqs=1, q_len=1, kv_len=131072, heads=32, kv_heads=8, dim=128, bits=16, page=128, ragged=False, bos=False,
             window=4096, sinks=16),
        # uneven chunks, decoding steps among them, small heads, 3-bit cache, small pages, an odd window
        dict(name="window_chunks", op="window", seqs=13, q_len=333, kv_len=2047, heads=16, kv_heads=4, dim=64, bits=3, page=16, ragged=True, bos=True,
             window=301, sinks=5),
        # a chunk of a prompt over what came before it, 8-bit cache
        dict(name="window_chunk_8bit", op="window", seqs=1, q_len=2048, kv_len=16384, heads=32, kv_heads=32, dim=128, bits=8, page=64, ragged=False, bos=False,
             window=2048, sinks=64),
        # a whole prompt, bf16 cache
        dict(name="window_prompt", op="window", seqs=1, q_len=8192, kv_len=8192, heads=32, kv_heads=32, dim=128, bits=16, page=128, ragged=False, bos=False,
             window=1024, sinks=4),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "grad", "append", "window", "window", "window"])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (16, 16), (16, 4), (16, 2), (8, 8), (20, 4), (7, 1), (64, 8)])
    gain = rng.choice(["bf16", "f32"])
    if op in ("norm", "grad"):
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(op=op, tokens=_log(rng, 1, 16384 * 40 * 128 // ((heads + kv_heads) * dim) // (1 if dtype == "bf16" else 2)), heads=heads, kv_heads=kv_heads,
                    dim=dim, rot=rng.choice([dim, dim // 32 * 16]), dtype=dtype, gain=gain, interleaved=rng.random() < 0.5, context=_log(rng, 2048, 131072))
    dim = rng.choice([64, 128, 128, 256])
    kind = dict(heads=heads, kv_heads=kv_heads, dim=dim, bits=rng.choice([3, 4, 8, 16]), page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6)
    kind["bos"] = kind["bits"] in (3, 4) and rng.random() < 0.5
    if op == "append":
        seqs = _log(rng, 1, 64)
        q_len = _log(rng, 1, max(1, 8192 * 32 * 128 // (heads * dim * seqs) // 4))
        kv_len = min(131072, q_len + _log(rng, 1, 8192))
        return dict(op=op, seqs=seqs, q_len=q_len, kv_len=kv_len, interleaved=rng.random() < 0.5, rot=rng.choice([dim, dim // 2]), gain=gain, context=kv_len,
                    **kind)
    while True:
        seqs = _log(rng, 1, 96)
        q_len = 1 if rng.random() < 0.4 else _log(rng, 1, 4096)
        kv_len = q_len + _log(rng, 1, 65536)
        case = dict(op=op, seqs=seqs, q_len=q_len, kv_len=kv_len, window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 5, 16, 64]), **kind)
        # no more bytes and pairs than the largest listed cases, and a plain form that fits the card
        if seqs * kv_len * kv_heads * dim <= 64 * 4096 * 32 * 128 // 2 and seqs * heads * q_len * _span(case, q_len) * dim <= 32 * 8192 * 8192 * 128 // 8:
            return case


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


def _span(case, q_len):
    """Keys that a sequence's new tokens see at most."""
    return min(case["kv_len"], case["sinks"] + case["window"] + q_len - 1)


def _seen(case):
    """(keys that some row sees, pairs of a row and a key that it sees), over all sequences."""
    keys = pairs = 0
    w, s = case["window"], case["sinks"]
    for q, kv in zip(*_lengths(case)):
        low = max(0, kv - q + 1 - w)
        keys += kv - low + min(s, low)
        for i in range(kv - q, kv):
            at = max(0, i + 1 - w)
            pairs += i + 1 - at + min(s, at)
    return keys, pairs


def work(case):
    if case["op"] in ("norm", "grad"):
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        size = 2 if case["dtype"] == "bf16" else 4
        tensors, flops = (2, 4 * case["dim"] + 3 * case["rot"]) if case["op"] == "norm" else (3, 11 * case["dim"] + 3 * case["rot"])
        return {"bytes": tensors * n * case["dim"] * size + case["tokens"] * (4 + 4 * case["rot"]), "flops": n * flops}
    qs, kvs = _lengths(case)
    row = case["dim"] * case["bits"] // 8 + (0 if case["bits"] == 16 else 4)
    if case["op"] == "append":
        t = sum(qs)
        kv = 2 * t * case["kv_heads"]
        out = kv * row + (0 if case["bits"] == 16 else kv * case["dim"] * 2)   # quantized heads are handed out as values too
        flops = t * (case["heads"] + case["kv_heads"]) * (4 * case["dim"] + 3 * case["rot"]) + (0 if case["bits"] == 16 else 4 * kv * case["dim"])
        return {"bytes": 2 * t * case["heads"] * case["dim"] * 2 + kv * case["dim"] * 2 + out + t * 4 * case["rot"], "flops": flops}
    keys, pairs = _seen(case)
    rows = sum(qs) * case["heads"]
    return {"bytes": 2 * case["kv_heads"] * keys * row + rows * (2 * case["dim"] * 2 + 4), "flops": 4 * case["heads"] * case["dim"] * pairs}


# ---- inputs ----------------------------------------------------------------------------------------------------

class State:
    pass


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


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
    dim, heads, kv_heads = case["dim"], case["heads"], case["kv_heads"]

    def heads_of(rows, n, dtype=torch.bfloat16):
        # projections are near Gaussian, with a few channels that are much larger
        x = torch.randn(rows, n, dim, device=dev, generator=g)
        return (x * (1 + 9 * (torch.rand(n, dim, device=dev, generator=g) < 0.01))).to(dtype)

    if "gain" in case:      # learned, around one
        s.q_gain, s.k_gain = ((1 + 0.2 * torch.randn(dim, device=dev, generator=g)).to(_type(case["gain"])) for _ in range(2))
    if case["op"] in ("norm", "grad"):
        t, dtype = case["tokens"], _type(case["dtype"])
        s.q, s.k = heads_of(t, heads, dtype), heads_of(t, kv_heads, dtype)
        s.table = _table(case, dev)
        s.positions = torch.randint(0, case["context"], (t,), device=dev, generator=g, dtype=torch.int32)
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
        s.ws = None
        if case["op"] == "grad":
            s.grad_q, s.grad_k = (torch.randn(t, n, dim, device=dev, generator=g).to(dtype) for n in (heads, kv_heads))
        return s

    bits, page = case["bits"], case["page"]
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
        if c["op"] == "window":
            ws = hbl.new_workspace(hbl.hbl_attention_window_workspace_bytes(cache, batch, c["heads"], c["window"], c["sinks"]))
        s.plan = (cache, batch, ws)
    return s.plan


def _run_own(s):
    from paper_2504_18415_b200 import hbl
    c = s.case
    if c["op"] == "norm":
        return hbl.hbl_norm_rope(s.q, s.q_gain, s.positions, s.table, k=s.k, k_gain=s.k_gain, norm_eps=NORM_EPS, interleaved=c["interleaved"],
                                 q_out=s.q_out, k_out=s.k_out)
    if c["op"] == "grad":
        if s.ws is None:
            s.ws = hbl.new_workspace(hbl.hbl_norm_rope_grad_workspace_bytes(c["tokens"], c["heads"], c["kv_heads"], c["dim"]))
        return hbl.hbl_norm_rope_grad(s.grad_q, s.q, s.q_gain, s.positions, s.table, grad_k=s.grad_k, k=s.k, k_gain=s.k_gain, norm_eps=NORM_EPS,
                                      interleaved=c["interleaved"], dq=s.q_out, dk=s.k_out, workspace=s.ws)
    cache, batch, ws = _plan(s)
    if c["op"] == "append":
        hbl.hbl_kv_append_norm(cache, batch, s.new_k, s.new_v, s.k_gain, table=s.table, interleaved=c["interleaved"], q=s.q, q_gain=s.q_gain, q_out=s.out,
                               norm_eps=NORM_EPS, eps=EPS)
        if c["bits"] == 16:
            return [s.out, s.k, s.v]
        return [s.out, *hbl.hbl_kv_read(cache, batch), s.k_scale, s.v_scale]
    hbl.hbl_attention_window(cache, batch, s.q, c["window"], sinks=c["sinks"], sm_scale=s.sm_scale, out=s.out, lse=s.lse, workspace=ws)
    return [s.out, s.lse]


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _rotate(x, cos_sin, interleaved, backward=False):
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


def _inverse_rms(x):
    """Of each head, summed in 64 bits (values that are quantized afterwards lie next to borders), rounded once."""
    return (1.0 / (x.double().square().mean(-1, keepdim=True) + NORM_EPS).sqrt()).float()


def _norm_rotate(x, gain, rows, interleaved):
    return _rotate(x.float() * gain.float(), rows, interleaved) * _inverse_rms(x)


def _norm_grad(grad, x, gain, rows, interleaved):
    t, r, xf = _rotate(grad.float(), rows, interleaved, True), _inverse_rms(x), x.float()
    u = t * gain.float()
    dx = r * (u - xf * (r * r * (xf * u).mean(-1, keepdim=True)))
    return dx.to(x.dtype), (t * xf * r).sum((0, 1), dtype=torch.float64).float()


def _unpack(x, bits):
    if bits == 8:
        return x
    if bits == 4:
        return torch.stack([x & 15, x >> 4], -1).flatten(-2)
    b = x.to(torch.int32).reshape(*x.shape[:-1], -1, 3)
    word = b[..., 0] | (b[..., 1] << 8) | (b[..., 2] << 16)
    return ((word[..., None] >> (3 * torch.arange(8, device=x.device, dtype=torch.int32))) & 7).flatten(-2)


def _store(x, codes, scale, page, slot, s):
    """Quantizes x [T, kv heads, dim] (32 bits), stores codes and scales in the pages; returns the stored values in bf16."""
    bits = s.case["bits"]
    u, sc = _codes(x, bits)
    codes[page, :, slot] = _pack(u, bits)
    scale[page, :, slot] = sc
    value = (u.float() - 2 ** (bits - 1)) * sc[..., None]
    if s.bos is not None:
        u8, sc8 = _codes(x, 8)
        value = torch.where((s.position == 0)[:, None, None], (u8.float() - 128) * sc8[..., None], value)
    return value.to(torch.bfloat16)


def _gather(s, x, scale, bos, at):
    """Values of the keys at[n, j] of each sequence: [n, kv heads, j, dim]."""
    c, seq = s.case, torch.arange(at.shape[0], device=at.device)[:, None]
    page, slot = s.pages[seq, at // c["page"]].long(), at % c["page"]
    got = x[page, :, slot]
    if c["bits"] == 16:
        return got.float().transpose(1, 2)
    value = (_unpack(got, c["bits"]).float() - 2 ** (c["bits"] - 1)) * scale[page, :, slot][..., None]
    if bos is not None:
        first = ((bos[0].float() - 128) * bos[1][..., None])[:, None]
        value = torch.where((at == 0)[..., None, None], first, value)
    return value.transpose(1, 2)


def _window(s):
    c, n, group = s.case, len(s.kv_len), s.case["heads"] // s.case["kv_heads"]
    dev = s.q.device
    q_len = (s.q_start[1:] - s.q_start[:-1]).long()
    kv = s.kv_len.long()
    # the keys that a sequence's rows see: its sinks, and what the windows reach, from the first row's on
    low = (kv - q_len + 1 - c["window"]).clamp(min=0)
    sinks = torch.arange(min(c["sinks"], s.max_kv), device=dev)
    reach = torch.arange(min(s.max_kv, c["window"] + s.max_q - 1), device=dev)
    at = torch.cat([sinks.expand(n, -1), low[:, None] + reach], 1)
    there = torch.cat([sinks < low[:, None], low[:, None] + reach < kv[:, None]], 1)       # a sink within reach is counted there
    at = torch.minimum(at, kv[:, None] - 1).clamp(min=0)
    k = _gather(s, s.k, s.k_scale, s.bos[0:2] if s.bos else None, at)
    v = _gather(s, s.v, s.v_scale, s.bos[2:4] if s.bos else None, at)
    # queries by sequence, padded: [n, kv heads, group * max_q, dim]
    i = torch.arange(s.max_q, device=dev)
    row = (s.q_start[:-1, None] + i).clamp(max=s.tokens - 1).long()
    q = s.q[row].float().reshape(n, s.max_q, c["kv_heads"], group, c["dim"]).permute(0, 2, 3, 1, 4)
    score = (q.flatten(2, 3) @ k.transpose(-1, -2)).mul_(s.sm_scale).unflatten(2, (group, s.max_q))
    last = ((kv - q_len)[:, None] + i)[..., None]
    key = at[:, None]
    hidden = ~there[:, None] | (key > last) | ((key <= last - c["window"]) & (key >= c["sinks"]))
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = v.masked_fill(~there[:, None, :, None], 0)
    o = (p.flatten(2, 3) @ v).unflatten(2, (group, s.max_q)) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    where = (s.seq, (torch.arange(s.tokens, device=dev) - s.q_start[s.seq]).long())
    s.out.copy_(o.permute(0, 3, 1, 2, 4)[where].flatten(1, 2))
    s.lse.copy_(lse.permute(0, 3, 1, 2)[where].flatten(1, 2))
    return [s.out, s.lse]


def run(state):
    s, c = state, state.case
    if own:
        return _run_own(s)
    if c["op"] == "norm":
        rows = s.table[s.positions.long()]
        return tuple(_norm_rotate(x, g, rows, c["interleaved"]).to(x.dtype) for x, g in ((s.q, s.q_gain), (s.k, s.k_gain)))
    if c["op"] == "grad":
        rows = s.table[s.positions.long()]
        return _norm_grad(s.grad_q, s.q, s.q_gain, rows, c["interleaved"]) + _norm_grad(s.grad_k, s.k, s.k_gain, rows, c["interleaved"])
    if c["op"] == "append":
        rows = s.table[s.position.long()]
        q = _norm_rotate(s.q, s.q_gain, rows, c["interleaved"]).to(torch.bfloat16)
        k = _norm_rotate(s.new_k, s.k_gain, rows, c["interleaved"])
        page, slot = s.pages[s.seq, (s.position // c["page"]).long()].long(), (s.position % c["page"]).long()
        if c["bits"] == 16:
            s.k[page, :, slot] = k.to(torch.bfloat16)
            s.v[page, :, slot] = s.new_v
            return [q, s.k, s.v]
        return [q, _store(k, s.k, s.k_scale, page, slot, s), _store(s.new_v.float(), s.v, s.v_scale, page, slot, s), s.k_scale, s.v_scale]
    return _window(s)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    half = case["rot"] // 2 if "rot" in case else 0

    def turned(z, pos, sign=1.0):
        w = torch.view_as_complex(s.table[pos.long()].to(f8))[:, None]
        w = w.conj() if sign < 0 else w
        r = z[..., :2 * half].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        r = r if case["interleaved"] else r.transpose(-1, -2)
        r = torch.view_as_real(torch.view_as_complex(r.contiguous()) * w)
        r = r if case["interleaved"] else r.transpose(-1, -2)
        return torch.cat([r.flatten(-2), z[..., 2 * half:]], -1)

    def unit(x):
        """Heads of root mean square one, and what they were divided by."""
        z = x.to(f8)
        size = torch.linalg.vector_norm(z, dim=-1, keepdim=True)
        size = torch.sqrt(size * size / case["dim"] + NORM_EPS)
        return z / size, size

    if case["op"] == "norm":
        return tuple(turned(unit(x)[0] * g.to(f8), s.positions) for x, g in ((s.q, s.q_gain), (s.k, s.k_gain)))
    if case["op"] == "grad":
        got = []
        for x, g, grad in ((s.q, s.q_gain, s.grad_q), (s.k, s.k_gain, s.grad_k)):
            z, size = unit(x)
            back = turned(grad.to(f8), s.positions, -1.0)
            inner = back * g.to(f8)
            got += [(inner - z * torch.einsum("thd,thd->th", z, inner)[..., None] / case["dim"]) / size, torch.einsum("thd,thd->d", back, z)]
        return tuple(got)

    bits = case["bits"]
    if case["op"] == "append":
        k, v = turned(unit(s.new_k)[0] * s.k_gain.to(f8), s.position), s.new_v.to(f8)
        where = [(int(p), int(o)) for p, o in zip(s.pages[s.seq, (s.position // case["page"]).long()].tolist(), (s.position % case["page"]).tolist())]
        page, slot = (torch.tensor(w, device=k.device) for w in zip(*where))
        outs, scales = [turned(unit(s.q)[0] * s.q_gain.to(f8), s.position)], []
        for x, buf, scale in ((k, s.k, s.k_scale), (v, s.v, s.v_scale)):
            if bits == 16:
                whole = buf.to(f8)
                whole[page, :, slot] = x
                outs.append(whole)
                continue
            width = torch.where((s.position == 0) & bool(case["bos"]), 8, bits).to(f8)[:, None]
            top = x.abs().max(dim=-1).values
            level = 2 ** (width - 1) - 1
            outs.append(torch.round(x * (level / (top + EPS))[..., None]) * (top / level)[..., None])
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
        i = torch.arange(nk - nq, nk, device=s.q.device)[:, None]
        j = torch.arange(nk, device=s.q.device)[None]
        mask = (j <= i) & ((i - j < case["window"]) | (j < case["sinks"]))
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
