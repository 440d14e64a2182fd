"""The operators of decoding in four bits, as measurable cases.

Elements are e2m1 (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) in blocks of 32 with a common scale
2^(b - 127) held as one byte b.  Kinds:

    append   keys and values of new tokens into a paged cache, keys and queries rotated by their positions on the way, then
             the tokens read back as what the cache now stands for
    attend   attention over the paged cache: one token a sequence, a few, or a chunk of a prompt
    matvec   one to sixteen tokens against a weight in four bits; `out` says whether fp32 logits, bf16 outputs or bf16 outputs
             added to a residual come of it
    gateup   the gate and up projections of a SwiGLU layer in four bits, silu(gate) * up

Layer shapes are those of the library's benchmark workloads:

    llama   H = 4096, I = 14336, V = 128256, 32 query heads, 8 key heads of 128
    qwen    H = 3584, I = 18944, V = 152064, 28 query heads, 4 key heads of 128
    odd     H = 1056, I = 2080,  V = 32001   (multiples of 32 but not of 64, a ragged vocabulary)

A cache is a tensor [pages, key heads, block bytes] of uint8.  A block of P tokens of D dimensions holds, one after the other:
the key codes [P][D / 2] (low nibble first), the key scales [P][D / 32], the value codes [P / 4][16][D / 32][4] whose byte
(q, l, g, t) has dimension 32 g + l of token 4 q + t in its low nibble and dimension 32 g + 16 + l in its high one, and the value
scales [P / 4][D / 32][4].
"""
import math

import torch

own = False

DEV = "cuda"
LAYERS = {"llama": (4096, 14336, 128256), "qwen": (3584, 18944, 152064), "odd": (1056, 2080, 32001)}
HEADS = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 8, 64), "shared": (16, 1, 64), "wide": (16, 4, 256)}
ROPE_BASE = 500000.0


def _append(name, heads, seqs, tokens, page, far, rot=1.0, interleaved=False):
    return {"name": name, "kind": "append", "heads": heads, "seqs": seqs, "tokens": tokens, "page": page, "far": far,
            "rot": rot, "interleaved": interleaved}


def _attend(name, heads, seqs, tokens, kv, page, ragged=False, window=0):
    return {"name": name, "kind": "attend", "heads": heads, "seqs": seqs, "tokens": tokens, "kv": kv, "page": page,
            "ragged": ragged, "window": window}


def _matvec(name, n, k, m, out):
    return {"name": name, "kind": "matvec", "N": n, "K": k, "M": m, "out": out}


def listed():
    return [
        # one decoded token of one sequence: all latency
        _append("append_1", "llama", 1, 1, 64, 32767),
        # one step of a batch of long contexts, 48 sequences at their own positions
        _append("append_batch_48", "qwen", 48, 1, 16, 262143),
        # a chunk of a prompt, K and V of 8192 tokens
        _append("append_chunk_8192", "llama", 1, 8192, 64, 131071),
        # one token after a short prompt: all latency
        _attend("attend_317", "llama", 1, 1, 317, 16),
        # a serving batch, every sequence of its own length up to 8192
        _attend("attend_batch_32", "llama", 32, 1, 8192, 64, ragged=True),
        # one token after a long context
        _attend("attend_131072", "llama", 1, 1, 131072, 64),
        # the last chunk of a long prompt against all of it
        _attend("attend_chunk_2048", "llama", 1, 2048, 16384, 64),
        # several tokens a sequence (drafts to be verified), seven query heads to a key head, odd lengths, a sliding window
        _attend("attend_window_5", "qwen", 7, 5, 6001, 16, ragged=True, window=4096),
        # the head of one token
        _matvec("head_llama", 128256, 4096, 1, "fp32"),
        # the down projection of one token, with its residual
        _matvec("down_llama", 4096, 14336, 1, "residual"),
        # sixteen tokens against a small ragged weight
        _matvec("odd_16", 2083, 1056, 16, "bf16"),
        # the gate and up projections of a small batch
        {"name": "gateup_5", "kind": "gateup", "N": 18944, "K": 3584, "M": 5},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "matvec", "matvec", "gateup"])
    if kind in ("append", "attend"):
        case = {"kind": kind, "heads": rng.choice(["llama", "llama", "qwen", "qwen", "small", "shared", "wide"]),
                "page": rng.choice([16, 16, 32, 64, 64, 128, 256])}
    if kind == "append":
        seqs = rng.choice([1, 1, _log_int(rng, 2, 64)])
        return dict(case, seqs=seqs, tokens=_log_int(rng, 1, max(1, 8192 // seqs)), far=_log_int(rng, 8192, 458751),
                    rot=rng.choice([1.0, 1.0, 0.5, 0.0]), interleaved=rng.random() < 0.3)
    if kind == "attend":
        form = rng.choice(["decode", "decode", "few", "chunk"])
        if form == "decode":
            seqs, tokens = rng.choice([1, 1, _log_int(rng, 2, 64)]), 1
        elif form == "few":
            seqs, tokens = _log_int(rng, 1, 16), rng.randint(2, 16)
        else:
            seqs, tokens = rng.choice([1, 1, 2, 3]), _log_int(rng, 17, 1500)
        # no more keys than the largest listed cases have, in all and times the tokens that ask for them
        most = min(131072 // seqs, (1 << 24) // (seqs * tokens))
        return dict(case, seqs=seqs, tokens=tokens, kv=max(tokens, _log_int(rng, 1, most)), ragged=rng.random() < 0.6,
                    window=rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]))
    _, layer = rng.choice(list(LAYERS.items()))
    h, i, v = layer
    if kind == "gateup":
        return {"kind": kind, "N": rng.choice([i, i, 32 * _log_int(rng, 1, 400) + 7]), "K": h, "M": rng.choice([1, 1, rng.randint(2, 16)])}
    n, k = rng.choice([(v, h), (h, i), (h, h), (_log_int(rng, 1, v), h), (h, 32 * _log_int(rng, 1, 512))])
    return {"kind": kind, "N": n, "K": k, "M": rng.choice([1, 1, rng.randint(2, 16)]), "out": rng.choice(["fp32", "bf16", "residual"])}


# Four bits

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _encode(x):
    """Codes 0 to 15 (uint8) and scale bytes of x [..., 32 n], from its own type on (64 bits: nothing is rounded on the way).

    The scale is the power of two that brings the largest magnitude of a block to at most 7, which 6 is half a step away from;
    elements go to the nearest value, ties to the even code.  A block with an infinity or a NaN gets byte 255, which stands for NaN."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(torch.where(torch.isfinite(top), top, 0.0))
    s = torch.where(top > 0, e - 3 + (m > 0.875).to(e.dtype), -125).clamp(-125, 125)
    a = torch.ldexp(b.abs(), -s)
    c = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * (b < 0).byte())
    fine = torch.isfinite(b).all(-1, keepdim=True)
    return (torch.where(fine, c, 0).to(torch.uint8).flatten(-2), torch.where(fine, s + 127, 255).squeeze(-1).to(torch.uint8))


def _decode(codes, scales, dtype=torch.float32):
    """The values of codes [..., 32 n] and scale bytes [..., n]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=dtype, device=codes.device)
    s = torch.where(scales < 255, torch.exp2(scales.to(dtype) - 127.0), float("nan"))
    return (table[codes.long()].unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _pack(codes):
    """Two codes a byte, the low nibble first."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _block_bytes(page, d):
    return page * (d // 2 + d // 32) * 2


def _places(page, d, at, dev):
    """Offsets within a block of what token `at` [T] has there: key codes [T, d/2], key scales [T, d/32], value codes and scales."""
    g, l = torch.arange(d // 32, device=dev), torch.arange(16, device=dev)
    at = at.unsqueeze(-1)
    q, t = at // 4, at % 4
    kc = at * (d // 2) + torch.arange(d // 2, device=dev)
    ks = page * (d // 2) + at * (d // 32) + g
    vc = page * (d // 2 + d // 32) + q * (2 * d) + (l * (d // 8) + g.unsqueeze(-1) * 4).flatten() + t      # (g, l) in the order of the bytes
    vs = page * (d + d // 32) + q * (d // 8) + g * 4 + t
    return kc, ks, vc, vs


def _value_bytes(codes):
    """Value codes [..., d] as bytes [..., d / 2] in the order (g, l) of _places."""
    c = codes.unflatten(-1, (-1, 2, 16))
    return (c[..., 0, :] | (c[..., 1, :] << 4)).flatten(-2)


def _value_codes(b):
    b = b.unflatten(-1, (-1, 16))
    return torch.stack((b & 15, b >> 4), -2).flatten(-3)


def _store(cache, page, d, slots, k, v):
    """k, v [T, heads, d] into the cache."""
    for_page, at = slots // page, slots % page
    heads = torch.arange(cache.shape[1], device=cache.device)
    where = (for_page[:, None, None], heads[None, :, None])
    kc, ks, vc, vs = (p[:, None, :] for p in _places(page, d, at, cache.device))
    codes, scales = _encode(k)
    cache[where + (kc,)] = _pack(codes)
    cache[where + (ks,)] = scales
    codes, scales = _encode(v)
    cache[where + (vc,)] = _value_bytes(codes)
    cache[where + (vs,)] = scales


def _load(cache, page, d, slots):
    """k, v [T, heads, d] in 32 bits as the cache holds them."""
    for_page, at = slots // page, slots % page
    heads = torch.arange(cache.shape[1], device=cache.device)
    where = (for_page[:, None, None], heads[None, :, None])
    kc, ks, vc, vs = (p[:, None, :] for p in _places(page, d, at, cache.device))
    return (_decode(_unpack(cache[where + (kc,)]), cache[where + (ks,)]), _decode(_value_codes(cache[where + (vc,)]), cache[where + (vs,)]))


# Inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(gen, shape, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(torch.bfloat16)


def _weight(gen, n, k):
    """Codes [n, k / 2] and scale bytes [n, k / 32] of a weight of the usual spread."""
    rows = max(1, (1 << 26) // k)
    parts = [_encode(torch.randn((min(rows, n - r), k), generator=gen, device=DEV) * 0.02) for r in range(0, n, rows)]
    return torch.cat([_pack(c) for c, _ in parts]), torch.cat([s for _, s in parts])


def _pages_of(gen, seqs, kv, page):
    """A table [seqs, pages of a sequence] over a pool in any order, with a few pages that nobody has."""
    each = -(-kv // page)
    pool = torch.randperm(seqs * each + 3, generator=gen, device=DEV).to(torch.int32)
    return pool[:seqs * each].view(seqs, each).contiguous(), seqs * each + 3


def prepare(case, seed):
    gen = _generator(seed)
    st = {"case": case}
    kind = case["kind"]
    if kind == "append":
        hq, hkv, d = HEADS[case["heads"]]
        seqs, tokens, page = case["seqs"], case["tokens"], case["page"]
        n = seqs * tokens
        # queries, keys and values as one projection leaves them
        qkv = _normal(gen, (n, hq + 2 * hkv, d))
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        first = torch.randint(0, max(1, case["far"] - tokens + 2), (seqs, 1), generator=gen, device=DEV)
        st["positions"] = (first + torch.arange(tokens, device=DEV)).flatten().to(torch.int32)
        table, pages = _pages_of(gen, seqs, tokens + page, page)
        at = torch.randint(0, page, (seqs, 1), generator=gen, device=DEV) + torch.arange(tokens, device=DEV)
        st["slots"] = (table.long().gather(1, at // page) * page + at % page).flatten()
        rot = int(case["rot"] * d) // 2 * 2
        st["inv_freq"] = (ROPE_BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / max(1, rot))).float()
        st["cache"] = torch.randint(0, 256, (pages, hkv, _block_bytes(page, d)), generator=gen, device=DEV, dtype=torch.uint8)
        st["q_out"] = torch.empty((n, hq, d), dtype=torch.bfloat16, device=DEV)
        st["k_out"], st["v_out"] = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    elif kind == "attend":
        hq, hkv, d = HEADS[case["heads"]]
        seqs, tokens, kv, page = case["seqs"], case["tokens"], case["kv"], case["page"]
        table, pages = _pages_of(gen, seqs, kv, page)
        # what is left of earlier sequences lies behind the last token of a page and in the pages that nobody has
        cache = torch.randint(0, 256, (pages, hkv, _block_bytes(page, d)), generator=gen, device=DEV, dtype=torch.uint8)
        lens, asked = torch.full((seqs,), kv, device=DEV), torch.full((seqs,), tokens, device=DEV)
        if case["ragged"]:
            lens = torch.randint(min(kv, max(tokens, kv // 8)), kv + 1, (seqs,), generator=gen, device=DEV)
            lens[0] = kv
            asked -= torch.arange(seqs, device=DEV) % (tokens - tokens // 2)
        for b in range(seqs):
            for r in range(0, int(lens[b]), 16384):
                at = torch.arange(r, min(r + 16384, int(lens[b])), device=DEV)
                k, v = (torch.randn((at.numel(), hkv, d), generator=gen, device=DEV) for _ in range(2))
                _store(cache, page, d, table[b].long()[at // page] * page + at % page, k, v)
        st["cache"], st["table"], st["lens"] = cache, table, lens.to(torch.int32)
        st["starts"] = torch.cat([torch.zeros(1, device=DEV, dtype=torch.long), asked.cumsum(0)]).to(torch.int32)
        n = int(asked.sum())
        st["max_q"] = int(asked.max())
        st["q"] = _normal(gen, (n, hq, d))
        st["out"] = torch.empty((n, hq, d), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((n, hq), dtype=torch.float32, device=DEV)
    else:
        n, k, m = case["N"], case["K"], case["M"]
        st["x"] = _normal(gen, (m, k))
        st["w"] = _weight(gen, n, k)
        if kind == "gateup":
            st["w_up"] = _weight(gen, n, k)
        elif case["out"] == "residual":
            st["residual"] = _normal(gen, (m, n))
        st["out"] = torch.empty((m, n), dtype=torch.float32 if case.get("out") == "fp32" else torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    return st


# The plain forms

def _rotated(x, cos, sin, rot, interleaved):
    """x [T, heads, d] in 64 bits with its first `rot` dimensions rotated by the angles of cos, sin [T, 1, rot / 2]."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    head = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((head, x[..., rot:]), -1)


def _plain_append(st):
    case = st["case"]
    d, page = st["k"].shape[-1], case["page"]
    rot = 2 * st["inv_freq"].numel()
    # in 64 bits: the angles of far positions, and values next to a border between two codes
    angle = (st["positions"].double()[:, None] * st["inv_freq"].double())[:, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    q = _rotated(st["q"].double(), cos, sin, rot, case["interleaved"]).to(torch.bfloat16)
    k = _rotated(st["k"].double(), cos, sin, rot, case["interleaved"])
    _store(st["cache"], page, d, st["slots"], k, st["v"].double())
    k, v = _load(st["cache"], page, d, st["slots"])
    return {"q": q, "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attend(st):
    case, q = st["case"], st["q"]
    page, window = case["page"], case["window"]
    (n, hq, d), (seqs, each), hkv = q.shape, st["table"].shape, st["cache"].shape[1]
    kv, group, most = case["kv"], hq // hkv, st["max_q"]
    at = torch.arange(kv, device=q.device)
    slots = st["table"].long()[:, at // page] * page + at % page
    k, v = _load(st["cache"], page, d, slots.flatten())
    lens, starts = st["lens"].long(), st["starts"].long()
    k, v = (t.view(seqs, kv, hkv, d).transpose(1, 2) for t in (k, v))
    live = at < lens[:, None]                                                     # [seqs, kv]
    v = torch.where(live[:, None, :, None], v, 0.0)
    # queries padded to the longest of their kind: [seqs, most]
    i = torch.arange(most, device=q.device)
    asked = starts[1:] - starts[:-1]
    row = (starts[:-1, None] + i).clamp(max=n - 1)
    place = lens[:, None] - asked[:, None] + i
    seen = live[:, None, :] & (at <= place[..., None])                            # [seqs, most, kv]
    if window:
        seen &= at > place[..., None] - window
    x = q.float()[row].view(seqs, most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, hkv, most * group, d)
    s = torch.matmul(x, k.transpose(-1, -2).contiguous()).view(seqs, hkv, most, group, kv) / math.sqrt(d)
    s = s.masked_fill(~seen[:, None, :, None, :], float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    del s
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(seqs, hkv, most * group, kv), v.contiguous()).view(seqs, hkv, most, group, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (top + torch.log(total)).squeeze(-1)
    # back to the rows that were asked for
    b = torch.searchsorted(starts, torch.arange(n, device=q.device), right=True) - 1
    j = torch.arange(n, device=q.device) - starts[b]
    return {"out": o.permute(0, 2, 1, 3, 4)[b, j].reshape(n, hq, d).to(torch.bfloat16), "lse": lse.permute(0, 2, 1, 3)[b, j].reshape(n, hq)}


def _plain_product(x, w):
    return x.float() @ _decode(_unpack(w[0]), w[1]).t()


def _plain(st):
    kind = st["case"]["kind"]
    if kind == "append":
        return _plain_append(st)
    if kind == "attend":
        return _plain_attend(st)
    y = _plain_product(st["x"], st["w"])
    if kind == "gateup":
        y = y / (1.0 + torch.exp(-y)) * _plain_product(st["x"], st["w_up"])
    if "residual" in st:
        y = y + st["residual"].float()
    return {"out": y.to(st["out"].dtype)}


def run(st):
    if not own:
        return _plain(st)
    from paper_2504_12526_amd import binding
    case = st["case"]
    if case["kind"] == "append":
        binding.mom_mx_kv_append(st["k"], st["v"], st["slots"], st["cache"], case["page"], positions=st["positions"],
                                 inv_freq=st["inv_freq"], interleaved=case["interleaved"], q=st["q"], q_out=st["q_out"])
        binding.mom_mx_kv_read(st["cache"], case["page"], st["slots"], st["k_out"], st["v_out"])
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    if case["kind"] == "attend":
        if "workspace" not in st:
            (n, hq, d), hkv = st["q"].shape, st["cache"].shape[1]
            st["workspace"] = torch.empty(binding.mom_mx_attention_workspace_bytes(n, case["seqs"], hq, hkv, d, case["kv"]),
                                          dtype=torch.uint8, device=st["q"].device)
        binding.mom_mx_attention(st["q"], st["cache"], case["page"], st["table"], st["lens"], case["kv"], st["out"], st["workspace"],
                                 q_starts=st["starts"], window=case["window"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if case["kind"] == "gateup":
        binding.mom_mx_gateup(st["x"], *st["w"], *st["w_up"], st["out"])
    else:
        binding.mom_mx_matvec(st["x"], *st["w"], st["out"], residual=st.get("residual"))
    return {"out": st["out"]}


def work(case):
    kind = case["kind"]
    if kind == "append":
        hq, hkv, d = HEADS[case["heads"]]
        n = case["seqs"] * case["tokens"]
        four = 2 * hkv * (d // 2 + d // 32)
        # queries in and out, keys and values in, the cache written and read, keys and values out
        return {"bytes": n * (4 * hq * d + 4 * hkv * d + 2 * four + 4 * hkv * d + 4 + 8), "flops": n * (hq + hkv) * int(case["rot"] * d) * 3}
    if kind == "attend":
        hq, hkv, d = HEADS[case["heads"]]
        seqs, tokens, kv, window = case["seqs"], case["tokens"], case["kv"], case["window"]
        if case["ragged"]:       # on average
            kv, tokens = (kv + min(kv, max(tokens, kv // 8))) / 2, tokens - (tokens - tokens // 2 - 1) / 2
        reach = min(kv, window) if window else kv
        pairs = tokens * reach if window and window < kv else tokens * kv - tokens * (tokens - 1) / 2
        read = min(kv, reach + tokens - 1)
        return {"bytes": int(seqs * (read * hkv * (d + d // 16) + tokens * hq * (4 * d + 4))), "flops": int(seqs * pairs * hq * 4 * d)}
    n, k, m = case["N"], case["K"], case["M"]
    weights = (2 if kind == "gateup" else 1) * n * (k // 2 + k // 32)
    out = {"fp32": 4, "bf16": 2, "residual": 4}[case.get("out", "bf16")]
    return {"bytes": weights + 2 * m * k + out * m * n, "flops": 2 * m * n * k * (2 if kind == "gateup" else 1)}


# The same from the definitions, in 64 bits

def _element(nibble):
    """e2m1 by its bits: without an exponent m / 2, else 2^(e - 1) (1 + m / 2)."""
    n = nibble.long()
    e, m = (n >> 1) & 3, (n & 1).double()
    mag = torch.where(e == 0, m * 0.5, torch.pow(2.0, (e - 1).double()) * (1.0 + m * 0.5))
    return torch.where(n >= 8, -mag, mag)


def _nearest(block):
    """The values [..., 32] in 64 bits that blocks [..., 32] become: the nearest of all sixteen times a power of two."""
    top = block.abs().amax(-1, keepdim=True)
    s = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 4
    s = s + (top > 7.0 * torch.pow(2.0, s)).double()       # the smallest power that leaves at most 7: within three of that
    s = s + (top > 7.0 * torch.pow(2.0, s)).double()
    s = s + (top > 7.0 * torch.pow(2.0, s)).double()
    a = block.abs() / torch.pow(2.0, s)
    mags = _element(torch.arange(8, device=block.device))
    off = (a.unsqueeze(-1) - mags).abs()
    near = off.amin(-1, keepdim=True)
    tied = off == near
    even = torch.arange(8, device=block.device) % 2 == 0
    pick = torch.where(tied & even, 2, tied.long()).argmax(-1)
    return torch.copysign(mags[pick], block) * torch.pow(2.0, s)


def _token_values(cache, page, d, head, slot):
    """Key and value [T, d] of the slots [T] of one head in 64 bits, by the address of every nibble."""
    flat, dev = cache.view(-1), cache.device
    base = ((slot // page) * cache.shape[1] + head)[:, None] * cache.shape[2]
    at, dim = (slot % page)[:, None], torch.arange(d, device=dev)[None]
    kb = flat[base + at * (d // 2) + dim // 2].long()
    k = _element((kb >> (4 * (dim % 2))) & 15) * torch.pow(2.0, flat[base + page * d // 2 + at * (d // 32) + dim // 32].double() - 127)
    to = base + page * (d // 2 + d // 32)
    vb = flat[to + at // 4 * (2 * d) + dim % 16 * (d // 8) + dim // 32 * 4 + at % 4].long()
    v = _element((vb >> (4 * (dim // 16 % 2))) & 15) * torch.pow(2.0, flat[to + page * d // 2 + at // 4 * (d // 8) + dim // 32 * 4 + at % 4].double() - 127)
    return k, v


def _exact_attend(st, case):
    q, page, window = st["q"].double(), case["page"], case["window"]
    hq, hkv, d = HEADS[case["heads"]]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    starts, lens = st["starts"].tolist(), st["lens"].tolist()
    for b in range(case["seqs"]):
        lo, hi, n = starts[b], starts[b + 1], lens[b]
        j = torch.arange(n, device=q.device)
        slot = st["table"][b].long()[j // page] * page + j % page
        for h in range(hkv):
            k, v = _token_values(st["cache"], page, d, h, slot)
            for r in range(lo, hi, 512):
                e = min(hi, r + 512)
                p = torch.arange(n - (hi - r), n - (hi - e), device=q.device)[:, None]
                off = (j > p) | (j <= p - window) if window else j > p
                for head in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    s = (q[r:e, head] @ k.t().contiguous()).mul_(d ** -0.5).masked_fill_(off, -math.inf)
                    z = torch.logsumexp(s, -1)
                    lse[r:e, head] = z
                    out[r:e, head] = torch.nan_to_num(torch.exp(s - z[:, None]), nan=0.0) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "attend":
        return _exact_attend(st, case)
    if kind == "append":
        half = st["inv_freq"].numel()
        angle = st["positions"].double()[:, None, None] * st["inv_freq"].double()
        turn = torch.polar(torch.ones_like(angle), angle)
        got = {}
        for name in ("q", "k"):
            x = st[name].double()
            y = x.clone()
            lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
            z = torch.complex(x[..., lo], x[..., hi]) * turn
            y[..., lo], y[..., hi] = z.real, z.imag
            got[name] = y
        for name, x in (("k", got["k"]), ("v", st["v"].double())):
            got[name] = torch.cat([_nearest(r.unflatten(-1, (-1, 32))).flatten(-2) for r in x.split(512)])
        return {"q": got["q"], "k": got["k"], "v": got["v"]}

    def product(w):
        x, parts, rows = st["x"].double(), [], max(1, (1 << 26) // case["K"])
        for r in range(0, case["N"], rows):
            b = w[0][r:r + rows].long()
            v = torch.stack((_element(b & 15), _element(b >> 4)), -1).flatten(-2)
            v *= torch.pow(2.0, w[1][r:r + rows].double() - 127).repeat_interleave(32, -1)
            parts.append(x @ v.t().contiguous())
        return torch.cat(parts, -1)

    y = product(st["w"])
    if kind == "gateup":
        y = y * torch.sigmoid(y) * product(st["w_up"])
    if "residual" in st:
        y = y + st["residual"].double()
    return {"out": y}
