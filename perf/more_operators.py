"""The operators of drafted tokens over the four-bit cache, as measurable cases.

A step with drafts: some rows (new tokens) of every sequence form a tree, row 0 its root; all of them attend over the cache at once,
the target's logits of all of them come out, and a walk down the tree decides which of them stay.  Kinds:

    plan     from the rows' parents: which rows each row sees (bits), its position, its slot in the cache
    attend   attention of the rows over the paged cache: all that was there before them, and of the new ones what their bits say
    verify   the drafted tokens against the target's probabilities, from given random numbers: which rows stay, and the next token
    keep     the rows' keys and values appended, those that stay moved together, and what the cache then holds of them read back

Vocabularies and heads are those of the library's benchmark workloads:

    llama   V = 128256, 32 query heads, 8 key heads of 128
    qwen    V = 152064, 28 query heads, 4 key heads of 128
    odd     V = 32001 (ragged)

A cache is a tensor [pages, key heads, block bytes] of uint8; elements are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) in blocks of 32 with a
common scale 2^(b - 127) held as one byte b.  A block of P tokens of D dimensions holds, one after the other: the key codes [P][D / 2] (low
nibble first), the key scales [P][D / 32], the value codes [P / 4][16][D / 32][4] whose byte (q, l, g, t) has dimension 32 g + l of token
4 q + t in its low nibble and dimension 32 g + 16 + l in its high one, and the value scales [P / 4][D / 32][4].
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
VOCABS = {"llama": 128256, "qwen": 152064, "odd": 32001}
HEADS = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (8, 8, 64), "shared": (16, 1, 64), "wide": (16, 4, 256)}
MOST_VERIFIED = 32 * 8 * 128256      # logits of the largest verification


def _plan(name, seqs, rows, branch, kv, page, ragged=False):
    return {"name": name, "kind": "plan", "seqs": seqs, "rows": rows, "branch": branch, "kv": kv, "page": page, "ragged": ragged}


def _attend(name, heads, seqs, rows, branch, kv, page, ragged=False, window=0):
    return {"name": name, "kind": "attend", "heads": heads, "seqs": seqs, "rows": rows, "branch": branch, "kv": kv, "page": page,
            "ragged": ragged, "window": window}


def _verify(name, vocab, seqs, rows, branch, draft, temperature, bf16=False, ragged=False, mixed=False):
    return {"name": name, "kind": "verify", "V": vocab, "seqs": seqs, "rows": rows, "branch": branch, "draft": draft,
            "temperature": temperature, "bf16": bf16, "ragged": ragged, "mixed": mixed}


def _keep(name, heads, seqs, rows, kv, page, ragged=False):
    return {"name": name, "kind": "keep", "heads": heads, "seqs": seqs, "rows": rows, "kv": kv, "page": page, "ragged": ragged}


def listed():
    return [
        # the tree of one sequence: all latency
        _plan("plan_16", 1, 16, 4, 32767, 64),
        # the trees of a batch, each sequence with its own
        _plan("plan_batch_48", 48, 64, 4, 8192, 16, ragged=True),
        # a small tree after a short prompt: all latency
        _attend("tree_317", "llama", 1, 8, 3, 317, 16),
        # a serving batch, every sequence of its own length up to 8192 with a small tree
        _attend("tree_batch_32", "llama", 32, 8, 2, 8192, 64, ragged=True),
        # as many rows as the products in four bits take, after a long context
        _attend("tree_131072", "llama", 1, 16, 4, 131072, 64),
        # wide trees, seven query heads to a key head, odd lengths, a sliding window
        _attend("tree_window_61", "qwen", 5, 61, 4, 16001, 16, ragged=True, window=4096),
        # one sequence, four tokens drafted in a chain by a model whose probabilities are at hand
        _verify("verify_5", VOCABS["llama"], 1, 5, 1, True, 1.0),
        # a batch of such chains
        _verify("verify_batch_32", VOCABS["llama"], 32, 8, 1, True, 0.8),
        # trees with several children a row, logits in bf16
        _verify("verify_tree_16", VOCABS["qwen"], 8, 16, 3, True, 1.0, bf16=True),
        # drafts without probabilities (looked up in the text), some sequences greedy, a ragged vocabulary
        _verify("verify_lookup_7", VOCABS["odd"], 11, 7, 2, False, 0.7, ragged=True, mixed=True),
        # what stays of one sequence's tree
        _keep("keep_16", "llama", 1, 16, 32767, 64),
        # what stays of a batch's
        _keep("keep_batch_48", "qwen", 48, 8, 8192, 16, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["plan", "attend", "attend", "attend", "attend", "verify", "verify", "verify", "verify", "keep", "keep"])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256])
    ragged = rng.random() < 0.6
    if kind == "verify":
        rows = rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 2, 16), _log_int(rng, 2, 16), _log_int(rng, 2, 64)])
        V = rng.choice([VOCABS["llama"], VOCABS["qwen"], VOCABS["odd"], _log_int(rng, 2, 160000), _log_int(rng, 1000, 160000)])
        seqs = min(rng.choice([1, 1, _log_int(rng, 2, 64)]), max(1, MOST_VERIFIED // (rows * V)))
        return {"kind": kind, "V": V, "seqs": seqs, "rows": rows, "branch": rng.choice([1, 1, 2, 3, 4]), "draft": rng.random() < 0.7,
                "temperature": rng.choice([0.0, 0.6, 1.0, 1.3]), "bf16": rng.random() < 0.3, "ragged": ragged, "mixed": rng.random() < 0.3}
    rows = rng.choice([_log_int(rng, 1, 16), _log_int(rng, 2, 64), _log_int(rng, 2, 200)])
    seqs = rng.choice([1, 1, _log_int(rng, 2, 64)])
    if kind == "plan":
        return {"kind": kind, "seqs": seqs, "rows": rows, "branch": rng.randint(1, 6), "kv": max(rows, _log_int(rng, 1, 32768)), "page": page, "ragged": ragged}
    heads = rng.choice(["llama", "llama", "qwen", "qwen", "small", "shared", "wide"])
    if kind == "keep":
        return {"kind": kind, "heads": heads, "seqs": seqs, "rows": rows, "kv": max(rows, _log_int(rng, 1, 32768)), "page": page, "ragged": ragged}
    # no more keys than the largest listed cases have, in all and times the rows that ask for them
    most = min(131072 // seqs, (1 << 22) // (seqs * rows))
    return {"kind": kind, "heads": heads, "seqs": seqs, "rows": rows, "branch": rng.randint(1, 6), "kv": max(rows, _log_int(rng, 1, max(1, most))),
            "page": page, "ragged": ragged, "window": rng.choice([0, 0, 0, _log_int(rng, 1, 8192)])}


# Four bits

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _encode(x):
    """Codes 0 to 15 and scale bytes (uint8) of x [..., 32 n]: the power of two that brings the largest magnitude of a block to at most 7, and the
    nearest codes, ties to the even one."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    s = torch.where(top > 0, e - 3 + (m > 0.875).to(e.dtype), -125).clamp(-125, 125)
    a = torch.ldexp(b.abs(), -s)
    c = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * (b < 0).byte()
    return c.to(torch.uint8).flatten(-2), (s + 127).squeeze(-1).to(torch.uint8)


def _decode(codes, scales):
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    s = torch.where(scales < 255, torch.exp2(scales.float() - 127.0), float("nan"))
    return (table[codes.long()].unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


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


def _where(cache, page, d, slots):
    heads = torch.arange(cache.shape[1], device=cache.device)
    return ((slots // page)[:, None, None], heads[None, :, None]), [p[:, None, :] for p in _places(page, d, slots % page, cache.device)]


def _store(cache, page, d, slots, k, v):
    """k, v [T, heads, d] into the cache."""
    at, (kc, ks, vc, vs) = _where(cache, page, d, slots)
    codes, scales = _encode(k)
    cache[at + (kc,)] = codes[..., 0::2] | (codes[..., 1::2] << 4)
    cache[at + (ks,)] = scales
    codes, scales = _encode(v)
    c = codes.unflatten(-1, (-1, 2, 16))
    cache[at + (vc,)] = (c[..., 0, :] | (c[..., 1, :] << 4)).flatten(-2)
    cache[at + (vs,)] = scales


def _load(cache, page, d, slots):
    """k, v [T, heads, d] in 32 bits as the cache holds them."""
    at, (kc, ks, vc, vs) = _where(cache, page, d, slots)
    b = cache[at + (kc,)]
    k = _decode(torch.stack((b & 15, b >> 4), -1).flatten(-2), cache[at + (ks,)])
    b = cache[at + (vc,)].unflatten(-1, (-1, 16))
    return k, _decode(torch.stack((b & 15, b >> 4), -2).flatten(-3), cache[at + (vs,)])


# Inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _pages_of(gen, seqs, kv, page):
    """A table [seqs, pages of a sequence] over a pool in any order, with a few pages that nobody has."""
    each = -(-kv // page)
    pool = torch.randperm(seqs * each + 3, generator=gen, device=DEV).to(torch.int32)
    return pool[:seqs * each].view(seqs, each).contiguous(), seqs * each + 3


def _row_counts(case):
    """Rows of every sequence: all of them, or between half and all."""
    rows = case["rows"]
    return [rows - (b % (rows - rows // 2) if case["ragged"] else 0) for b in range(case["seqs"])]


def _tree(rng, rows, branch):
    """Parents of a tree of `rows` rows with up to `branch` children a row, the newer rows the likelier parents."""
    parents, free = [-1], [branch]
    for i in range(1, rows):
        open_rows = [j for j in range(max(0, i - 4 * branch), i) if free[j]] or [j for j in range(i) if free[j]]
        p = open_rows[max(rng.randrange(len(open_rows)), rng.randrange(len(open_rows)))]
        free[p] -= 1
        parents.append(p)
        free.append(branch)
    return parents


def _seen(parents):
    """Which rows each row of a tree sees: itself and those above it."""
    seen = np.zeros((len(parents), len(parents)), dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def _words(case):
    return -(-case["rows"] // 32)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _starts(counts):
    return [0] + np.cumsum(counts).tolist()


def _lengths(gen, case, least):
    """Tokens of every sequence in the cache, `least` [seqs] new ones among them."""
    kv, seqs = case["kv"], case["seqs"]
    if not case["ragged"]:
        return [kv] * seqs
    lens = torch.randint(kv // 8, kv + 1, (seqs,), generator=gen, device=DEV).tolist()
    return [kv] + [max(n, m) for n, m in zip(lens[1:], least[1:])]


def prepare(case, seed):
    gen, rng = _generator(seed), random.Random(seed)
    counts = _row_counts(case)
    st = {"case": case, "counts": counts, "starts": _ints(_starts(counts))}
    kind, seqs, n = case["kind"], case["seqs"], sum(counts)
    if kind != "keep":
        trees = [_tree(rng, m, case["branch"]) for m in counts]
        st["parents"] = _ints([p for t in trees for p in t])
    if kind != "verify":
        page, kv = case["page"], case["kv"]
        st["lens"] = _ints(_lengths(gen, case, counts))
        st["table"], pages = _pages_of(gen, seqs, kv, page)
    if kind == "plan":
        st["masks"] = torch.empty((n, _words(case)), dtype=torch.int32, device=DEV)
        st["positions"] = torch.empty(n, dtype=torch.int32, device=DEV)
        st["slots"] = torch.empty(n, dtype=torch.int64, device=DEV)
    elif kind == "attend":
        hq, hkv, d = HEADS[case["heads"]]
        # what is left of earlier sequences lies behind the last token of a page and in the pages that nobody has
        cache = torch.randint(0, 256, (pages, hkv, _block_bytes(page, d)), generator=gen, device=DEV, dtype=torch.uint8)
        for b, length in enumerate(st["lens"].tolist()):
            for r in range(0, length, 16384):
                at = torch.arange(r, min(r + 16384, length), device=DEV)
                k, v = (torch.randn((at.numel(), hkv, d), generator=gen, device=DEV) for _ in range(2))
                _store(cache, page, d, st["table"][b].long()[at // page] * page + at % page, k, v)
        st["cache"] = cache
        # one plan serves all layers of a step: it is at hand
        masks = np.zeros((n, 32 * _words(case)), dtype=np.uint64)
        for lo, t in zip(_starts(counts), trees):
            masks[lo:lo + len(t), :len(t)] = _seen(t)
        words = (masks.reshape(n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1, dtype=np.uint64)
        st["masks"] = torch.from_numpy(words.astype(np.uint32).view(np.int32)).to(DEV)
        st["q"] = torch.randn((n, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        st["out"] = torch.empty((n, hq, d), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((n, hq), dtype=torch.float32, device=DEV)
    elif kind == "verify":
        V, dtype = case["V"], torch.bfloat16 if case["bf16"] else torch.float32
        # logits as a model's: a few tokens have most of the weight; the drafting model's are those with an error
        logits = torch.randn((n, V), generator=gen, device=DEV) * 3.0
        st["target"] = logits.to(dtype, copy=True)
        logits += torch.randn((n, V), generator=gen, device=DEV) * 0.7
        t = [0.0 if case["mixed"] and b % 3 == 1 else case["temperature"] for b in range(seqs)]
        st["temperatures"] = torch.tensor(t, dtype=torch.float32, device=DEV)
        # every drafted token is drawn from the drafting model at its parent
        row_t = torch.repeat_interleave(st["temperatures"], _ints(counts, torch.int64))
        st["tokens"] = torch.zeros(n, dtype=torch.int32, device=DEV)
        base = torch.repeat_interleave(st["starts"][:-1].long(), _ints(counts, torch.int64))
        above = (base + st["parents"].long().clamp(min=0))
        for r in range(0, n, 64):
            l = logits[above[r:r + 64]].to(dtype).float()
            noise = -torch.log(-torch.log(torch.rand(l.shape, generator=gen, device=DEV).clamp(min=1e-30)))
            st["tokens"][r:r + 64] = (l + row_t[r:r + 64, None] * noise).argmax(-1).to(torch.int32)
        st["draft"] = logits.to(dtype) if case["draft"] else None
        del logits
        st["uniforms"] = torch.rand(n, generator=gen, device=DEV)
        st["rows"], st["out"] = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(2))
        st["kept"] = torch.empty(seqs, dtype=torch.int32, device=DEV)
    else:
        hq, hkv, d = HEADS[case["heads"]]
        st["cache"] = torch.randint(0, 256, (pages, hkv, _block_bytes(page, d)), generator=gen, device=DEV, dtype=torch.uint8)
        qkv = torch.randn((n, hq + 2 * hkv, d), generator=gen, device=DEV).to(torch.bfloat16)
        st["k"], st["v"] = qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        lens = st["lens"].tolist()
        at = _ints([lens[b] - m + i for b, m in enumerate(counts) for i in range(m)], torch.int64)
        seq = _ints([b for b, m in enumerate(counts) for _ in range(m)], torch.int64)
        st["slots"] = st["table"].long()[seq, at // page] * page + at % page
        # the root and some rows below it in rising order; the rest of a sequence's rows say -1
        path = [[0] + sorted(rng.sample(range(1, m), rng.randint(0, min(m - 1, 6)))) for m in counts]
        st["rows"] = _ints([r for m, p in zip(counts, path) for r in p + [-1] * (m - len(p))])
        st["kept"] = _ints([len(p) for p in path])
        st["new_lens"] = torch.empty(seqs, dtype=torch.int32, device=DEV)
        st["k_out"], st["v_out"] = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    return st


# The plain forms

def _row_owner(st, n):
    """Sequence and number within it of every row."""
    starts = st["starts"].long()
    b = torch.searchsorted(starts, torch.arange(n, device=starts.device), right=True) - 1
    return b, torch.arange(n, device=starts.device) - starts[b]


def _plain_plan(st):
    parents, page = st["parents"].long(), st["case"]["page"]
    n, words = st["masks"].shape
    b, i = _row_owner(st, n)
    first = st["starts"].long()[b]
    masks, depth = torch.zeros((n, words), dtype=torch.int64, device=DEV), torch.zeros(n, dtype=torch.int64, device=DEV)
    # one row up at a time, for as long as there is one
    at, live = i, torch.ones(n, dtype=torch.bool, device=DEV)
    for _ in range(st["case"]["rows"]):
        masks.scatter_add_(1, (at // 32)[:, None], torch.where(live, 1 << (at % 32), 0)[:, None])
        up = parents[first + at]
        live = live & (up >= 0)
        depth += live
        at = torch.where(live, up, at)
    base = (st["lens"].long() - (st["starts"][1:] - st["starts"][:-1]).long())[b]
    place = base + i
    slots = st["table"].long()[b, place // page] * page + place % page
    masks = torch.where(masks >= 1 << 31, masks - (1 << 32), masks).to(torch.int32)
    return {"masks": masks, "positions": (base + depth).to(torch.int32), "slots": slots}


def _plain_attend(st):
    case, q = st["case"], st["q"]
    page, window, kv, most = case["page"], case["window"], case["kv"], case["rows"]
    (n, hq, d), (seqs, each), hkv = q.shape, st["table"].shape, st["cache"].shape[1]
    group, words = hq // hkv, st["masks"].shape[1]
    at = torch.arange(kv, device=q.device)
    slots = st["table"].long()[:, at // page] * page + at % page
    k, v = _load(st["cache"], page, d, slots.flatten())
    lens, starts = st["lens"].long(), st["starts"].long()
    k, v = (t.view(seqs, kv, hkv, d).transpose(1, 2) for t in (k, v))
    live = at < lens[:, None]                                                     # [seqs, kv]
    v = torch.where(live[:, None, :, None], v, 0.0)
    # rows padded to the longest of their kind: [seqs, most]
    asked = starts[1:] - starts[:-1]
    row = (starts[:-1, None] + torch.arange(most, device=q.device)).clamp(max=n - 1)
    base = (lens - asked)[:, None, None]
    j = (at - base).clamp(min=0)                                                  # which of the new ones a token is: [seqs, 1, kv]
    words_of = st["masks"][row].gather(2, (j // 32).clamp(max=words - 1).expand(seqs, most, kv))
    seen = live[:, None] & ((at < base) | (((words_of >> (j % 32)) & 1) != 0))    # [seqs, most, kv]
    if window:
        behind = seen.flip(-1).to(torch.int32).cumsum(-1).flip(-1)                # of what a row sees, this token and those after it
        seen &= behind <= window
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
    b, i = _row_owner(st, n)
    return {"out": o.permute(0, 2, 1, 3, 4)[b, i].reshape(n, hq, d).to(torch.bfloat16), "lse": lse.permute(0, 2, 1, 3)[b, i].reshape(n, hq)}


def _softmax64(logits, temperature):
    """In 64 bits: a cumulative sum over the vocabulary has a border at every token."""
    x = logits.double() / temperature[:, None]
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_verify(st):
    case = st["case"]
    seqs, most, V = case["seqs"], case["rows"], case["V"]
    starts, parents, tokens = st["starts"].long(), st["parents"].long(), st["tokens"].long()
    n = parents.shape[0]
    asked, first = starts[1:] - starts[:-1], starts[:-1]
    greedy = st["temperatures"] <= 0
    t = torch.where(greedy, 1.0, st["temperatures"]).double()
    seq = torch.arange(seqs, device=DEV)
    # where the walk stands, what is left of the target's probabilities there, and the outputs
    cur = torch.zeros(seqs, dtype=torch.int64, device=DEV)
    p = _softmax64(st["target"][first], t)
    best = st["target"][first].float().argmax(-1)
    q = _softmax64(st["draft"][first], t) if case["draft"] else None
    r = p
    rows = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    out = torch.full((n + 1,), -1, dtype=torch.int64, device=DEV)      # one more: what is not to be stored goes there
    rows = torch.cat([rows, rows[:1]])
    rows[first] = 0
    count = torch.ones(seqs, dtype=torch.int64, device=DEV)
    for i in range(1, most):
        at = (first + i).clamp(max=n - 1)
        x = tokens[at]
        tried = (i < asked) & (parents[at] == cur)
        weight = q[seq, x] if case["draft"] else 1.0
        taken = tried & torch.where(greedy, x == best, st["uniforms"][at].double() * weight < r[seq, x])
        refused = tried & ~taken
        # what is left after a refusal: no number of it under zero, the sum one again
        if case["draft"]:
            less = (r - q).clamp(min=0.0)
        else:
            less = r.clone()
            less[seq, x] = 0.0
        total = less.sum(-1, keepdim=True)
        r = torch.where(refused[:, None] & (total > 0), less / total, r)
        # down to a row that is taken
        rows[torch.where(taken, first + count, n)] = i
        out[torch.where(taken, first + count - 1, n)] = x
        count += taken
        cur = torch.where(taken, i, cur)
        now = first + cur
        r = torch.where(taken[:, None], _softmax64(st["target"][now], t), r)
        best = torch.where(taken, st["target"][now].float().argmax(-1), best)
        if case["draft"]:
            q = torch.where(taken[:, None], _softmax64(st["draft"][now], t), q)
    below = r.cumsum(-1)
    u = st["uniforms"][first].double() * below[:, -1]
    drawn = torch.searchsorted(below, u[:, None], right=True).squeeze(-1).clamp(max=V - 1)
    out[first + count - 1] = torch.where(greedy, best, drawn)
    return {"rows": rows[:n].to(torch.int32), "tokens": out[:n].to(torch.int32), "counts": count.to(torch.int32)}


def _plain_keep(st):
    case, cache = st["case"], st["cache"]
    d, page, n = st["k"].shape[-1], case["page"], st["k"].shape[0]
    _store(cache, page, d, st["slots"], st["k"].float(), st["v"].float())
    b, i = _row_owner(st, n)
    stays = i < st["kept"].long()[b]
    source = st["slots"][st["starts"].long()[b] + torch.where(stays, st["rows"].long(), i)]
    # all of them read before any is written
    (read, offsets), (to, places) = _where(cache, page, d, source), _where(cache, page, d, st["slots"])
    moved = [cache[read + (o,)] for o in offsets]
    for o, m in zip(places, moved):
        cache[to + (o,)] = m
    k, v = _load(cache, page, d, st["slots"])
    asked = st["starts"][1:] - st["starts"][:-1]
    return {"lens": st["lens"] - asked + st["kept"], "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"plan": _plain_plan, "attend": _plain_attend, "verify": _plain_verify, "keep": _plain_keep}[kind](st)
    from paper_2504_12526_amd import binding
    case = st["case"]
    if kind == "plan":
        binding.mom_mx_tree(st["lens"], parents=st["parents"], q_starts=st["starts"], masks=st["masks"], positions=st["positions"],
                            slots=st["slots"], page_table=st["table"], page_tokens=case["page"])
        return {"masks": st["masks"], "positions": st["positions"], "slots": st["slots"]}
    if kind == "attend":
        if "workspace" not in st:
            (n, hq, d), hkv = st["q"].shape, st["cache"].shape[1]
            st["workspace"] = torch.empty(binding.mom_mx_tree_attention_workspace_bytes(n, case["seqs"], hq, hkv, d, case["kv"]),
                                          dtype=torch.uint8, device=st["q"].device)
        binding.mom_mx_tree_attention(st["q"], st["cache"], case["page"], st["table"], st["lens"], case["kv"], st["masks"], st["out"],
                                      st["workspace"], q_starts=st["starts"], window=case["window"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "verify":
        if "workspace" not in st:
            st["workspace"] = torch.empty(binding.mom_verify_drafts_workspace_bytes(st["target"].shape[0], case["seqs"], case["V"]),
                                          dtype=torch.uint8, device=st["target"].device)
        binding.mom_verify_drafts(st["target"], st["tokens"], st["uniforms"], st["rows"], st["out"], st["kept"], st["workspace"], draft=st["draft"],
                                  parents=st["parents"], max_children=case["branch"], q_starts=st["starts"], temperatures=st["temperatures"])
        return {"rows": st["rows"], "tokens": st["out"], "counts": st["kept"]}
    binding.mom_mx_kv_append(st["k"], st["v"], st["slots"], st["cache"], case["page"])
    binding.mom_mx_kv_keep(st["cache"], case["page"], st["k"].shape[-1], st["table"], st["lens"], st["rows"], st["kept"], st["new_lens"], q_starts=st["starts"])
    binding.mom_mx_kv_read(st["cache"], case["page"], st["slots"], st["k_out"], st["v_out"])
    return {"lens": st["new_lens"], "k": st["k_out"], "v": st["v_out"]}


def work(case):
    kind, counts = case["kind"], _row_counts(case)
    n = sum(counts)
    if kind == "plan":
        return {"bytes": n * (4 + 4 * _words(case) + 4 + 8) + 8 * case["seqs"], "flops": n}
    if kind == "verify":
        # a row of the drafting model is read where it has children
        inner = sum(-(-(m - 1) // case["branch"]) for m in counts) if case["draft"] and case["temperature"] > 0 else 0
        return {"bytes": (n + inner) * case["V"] * (2 if case["bf16"] else 4) + 20 * n, "flops": 4 * (n + inner) * case["V"]}
    hq, hkv, d = HEADS[case["heads"]]
    if kind == "keep":
        four = 2 * hkv * (d // 2 + d // 32)
        # keys and values in, the cache written and read, up to seven rows of a sequence moved, keys and values out
        return {"bytes": n * (4 * hkv * d + 2 * four + 4 * hkv * d + 8 + 4) + 2 * four * sum(min(m - 1, 6) for m in counts) // 2, "flops": n}
    seqs, kv, window, rows = case["seqs"], case["kv"], case["window"], n / case["seqs"]
    if case["ragged"]:           # on average
        kv = max(rows, (kv + kv / 8) / 2) if seqs > 1 else kv
    reach = min(kv, window + rows) if window else kv
    return {"bytes": int(seqs * (reach * hkv * (d + d // 16) + rows * hq * (4 * d + 4))), "flops": int(seqs * rows * (min(kv, window) if window else kv) * hq * 4 * d)}


# The same from the definitions, in 64 bits

def _element(nibble):
    """e2m1 by its bits: without an exponent m / 2, else 2^(e - 1) (1 + m / 2)."""
    n = nibble.long()
    e, m = (n >> 1) & 3, (n & 1).double()
    mag = torch.where(e == 0, m * 0.5, torch.pow(2.0, (e - 1).double()) * (1.0 + m * 0.5))
    return torch.where(n >= 8, -mag, mag)


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


def _nearest(x):
    """The values in 64 bits that blocks of 32 of x [..., 32 n] become: the nearest of all eight magnitudes times a power of two."""
    block = x.double().unflatten(-1, (-1, 32))
    top = block.abs().amax(-1, keepdim=True)
    s = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 4
    for _ in range(3):                                       # the smallest power that leaves at most 7: within three of that
        s = s + (top > 7.0 * torch.pow(2.0, s)).double()
    a = block.abs() / torch.pow(2.0, s)
    mags = _element(torch.arange(8, device=x.device))
    off = (a.unsqueeze(-1) - mags).abs()
    tied = off == off.amin(-1, keepdim=True)
    even = torch.arange(8, device=x.device) % 2 == 0
    pick = torch.where(tied & even, 2, tied.long()).argmax(-1)
    return (torch.copysign(mags[pick], block) * torch.pow(2.0, s)).flatten(-2)


def _exact_plan(st, case):
    masks, positions, slots = [], [], []
    parents, page = st["parents"].tolist(), case["page"]
    lens, table, lo = st["lens"].tolist(), st["table"].tolist(), 0
    for b, m in enumerate(st["counts"]):
        for i in range(m):
            bits, j, steps = 0, i, 0
            while j >= 0:
                bits, j, steps = bits | 1 << j, parents[lo + j], steps + 1
            masks.append([bits >> 32 * w & 0xffffffff for w in range(_words(case))])
            at = lens[b] - m + i
            positions.append(lens[b] - m + steps - 1)
            slots.append(table[b][at // page] * page + at % page)
        lo += m
    masks = torch.from_numpy(np.array(masks, dtype=np.uint32).view(np.int32)).to(DEV)
    return {"masks": masks, "positions": _ints(positions), "slots": _ints(slots, torch.int64)}


def _exact_attend(st, case):
    q, page, window = st["q"].double(), case["page"], case["window"]
    hq, hkv, d = HEADS[case["heads"]]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    parents, lens, lo = st["parents"].tolist(), st["lens"].tolist(), 0
    for b, m in enumerate(st["counts"]):
        n = lens[b]
        j = torch.arange(n, device=q.device)
        slot = st["table"][b].long()[j // page] * page + j % page
        # a row of a tree: its own rows in front of it are those above it, and all of them come after what was there
        seen = torch.cat([torch.ones((m, n - m), dtype=torch.bool, device=q.device), torch.from_numpy(_seen(parents[lo:lo + m])).to(q.device)], 1)
        for i in range(m if window else 0):
            at = seen[i].nonzero().squeeze(-1)
            seen[i, at[:-window]] = False
        for h in range(hkv):
            k, v = _token_values(st["cache"], page, d, h, slot)
            for head in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                s = (q[lo:lo + m, head] @ k.t().contiguous()).mul_(d ** -0.5).masked_fill_(~seen, -math.inf)
                z = torch.logsumexp(s, -1)
                lse[lo:lo + m, head] = z
                out[lo:lo + m, head] = torch.nan_to_num(torch.exp(s - z[:, None]), nan=0.0) @ v
        lo += m
    return {"out": out, "lse": lse}


def _exact_verify(st, case):
    target, draft = st["target"], st["draft"]
    parents, tokens, u, temps = (st[k].tolist() for k in ("parents", "tokens", "uniforms", "temperatures"))
    rows, out, counts, lo = [], [], [], 0

    def chances(logits, t):
        x = logits.double().cpu().numpy() / t
        e = np.exp(x - x.max())
        return e / math.fsum(e)

    for b, m in enumerate(st["counts"]):
        t, path, got, at = temps[b], [0], [], 0
        while True:
            children = [i for i in range(m) if i > 0 and parents[lo + i] == at]
            if t <= 0:
                best = int(np.argmax(target[lo + at].float().cpu().numpy()))
                down = [i for i in children if tokens[lo + i] == best][:1]
            else:
                p, down = chances(target[lo + at], t), []
                q = chances(draft[lo + at], t) if draft is not None and children else None
                for i in children:
                    x = tokens[lo + i]
                    if u[lo + i] * (1.0 if q is None else q[x]) < p[x]:
                        down = [i]
                        break
                    left = np.maximum(p - q, 0.0) if q is not None else np.where(np.arange(len(p)) == x, 0.0, p)
                    if left.sum() > 0:
                        p = left / math.fsum(left)
            if not down:
                break
            at = down[0]
            path.append(at)
            got.append(tokens[lo + at])
        if t > 0:
            below = np.cumsum(p)
            best = min(int(np.searchsorted(below, u[lo] * below[-1], side="right")), len(p) - 1)
        got.append(best)
        rows += path + [-1] * (m - len(path))
        out += got + [-1] * (m - len(got))
        counts.append(len(path))
        lo += m
    return {"rows": _ints(rows), "tokens": _ints(out), "counts": _ints(counts)}


def _exact_keep(st, case):
    k, v = (_nearest(st[name]) for name in ("k", "v"))
    ko, vo, lens, lo = k.clone(), v.clone(), [], 0
    rows, kept = st["rows"].tolist(), st["kept"].tolist()
    for b, m in enumerate(st["counts"]):
        for i in range(kept[b]):
            ko[lo + i], vo[lo + i] = k[lo + rows[lo + i]], v[lo + rows[lo + i]]
        lens.append(int(st["lens"][b]) - m + kept[b])
        lo += m
    return {"lens": _ints(lens), "k": ko, "v": vo}


def exact(case, seed):
    st = prepare(case, seed)
    return {"plan": _exact_plan, "attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep}[case["kind"]](st, case)
