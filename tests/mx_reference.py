"""The four-bit operators written out in 64 bits on the CPU, element by element where that says best what is meant."""
import math

import torch

MAGS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
BF16_HALF = 2.0 ** -8        # half a step of bf16, relative
F32_HALF = 2.0 ** -24


def encode(x):
    """Codes [..., n] (0 to 15) and scale bytes [..., n / 32] of x [..., n]: the smallest power of two that leaves at most 7 (at least
    2^-125, at most 2^125), the nearest element, ties to the even code; NaN for a block with an infinity or a NaN."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    fine = torch.isfinite(b).all(-1)
    top = torch.where(fine & (top > 0), top, 1e-300)
    e = torch.ceil(torch.log2(top / 7)).long()
    e = torch.where(top > 7 * torch.pow(2.0, e.double()), e + 1, e)
    e = torch.where(top <= 7 * torch.pow(2.0, e.double() - 1), e - 1, e).clamp(-125, 125)
    a = b.abs() * torch.pow(2.0, -e.double()).unsqueeze(-1)
    off = (a.unsqueeze(-1) - MAGS).abs()
    low = off.amin(-1, keepdim=True)
    tie = off == low
    # of two tied neighbours one is even
    code = torch.where(tie, torch.tensor([2, 1, 2, 1, 2, 1, 2, 1]), 0).argmax(-1)
    code = code + 8 * torch.signbit(b).long()
    code = torch.where(fine.unsqueeze(-1), code, 0)
    return code.flatten(-2), torch.where(fine, e + 127, 255)


def decode(codes, scales):
    c = codes.long()
    v = torch.where(c >= 8, -MAGS[c & 7], MAGS[c & 7]).unflatten(-1, (-1, 32))
    s = torch.where(scales.long() < 255, torch.pow(2.0, scales.double() - 127), math.nan)
    return (v * s.unsqueeze(-1)).flatten(-2)


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8)


def unpack(b):
    b = b.long()
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def block_bytes(P, D):
    return P * (D // 2 + D // 32) * 2


def put(block, P, D, at, kc, ks, vc, vs):
    """Token `at` of a block (uint8 [block_bytes]): key codes and scales, value codes and scales."""
    G = D // 32
    block[at * (D // 2):(at + 1) * (D // 2)] = pack(kc)
    to = P * (D // 2)
    block[to + at * G:to + (at + 1) * G] = ks.to(torch.uint8)
    to += P * G
    c = vc.view(G, 2, 16)
    q, t = divmod(at, 4)
    quads = block[to:to + P * (D // 2)].view(P // 4, 16, G, 4)
    quads[q, :, :, t] = (c[:, 0] | (c[:, 1] << 4)).t().to(torch.uint8)
    to += P * (D // 2)
    block[to:].view(P // 4, G, 4)[q, :, t] = vs.to(torch.uint8)


def get(cache, P, D, page, at):
    """Keys and values [heads, D] in 64 bits of one token of the cache [pages, heads, bytes]."""
    G, b = D // 32, cache[page]
    k = decode(unpack(b[:, at * (D // 2):(at + 1) * (D // 2)]), b[:, P * (D // 2) + at * G:P * (D // 2) + (at + 1) * G])
    to, (q, t) = P * (D // 2 + G), divmod(at, 4)
    c = b[:, to:to + P * (D // 2)].reshape(-1, P // 4, 16, G, 4)[:, q, :, :, t].long().transpose(1, 2)      # [heads, G, 16]
    codes = torch.stack((c & 15, c >> 4), 2).flatten(1)
    return k, decode(codes, b[:, to + P * (D // 2):].reshape(-1, P // 4, G, 4)[:, q, :, t])


def rotate(x, positions, inv_freq, interleaved):
    """x [T, heads, D] in 64 bits, its first 2 len(inv_freq) dimensions rotated."""
    y, half = x.double().clone(), inv_freq.numel()
    if half == 0:
        return y
    angle = positions.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(angle), torch.sin(angle)
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    return y


def append(cache, P, k, v, slots):
    """k, v [T, heads, D] in 64 bits into a copy of the cache."""
    cache, D = cache.clone(), k.shape[-1]
    kc, ks = encode(k)
    vc, vs = encode(v)
    for i, slot in enumerate(slots.tolist()):
        if 0 <= slot < cache.shape[0] * P:
            for h in range(cache.shape[1]):
                put(cache[slot // P, h], P, D, slot % P, kc[i, h], ks[i, h], vc[i, h], vs[i, h])
    return cache


def attention(q, cache, P, table, lens, starts, scale, window=0, most=1 << 30):
    """out [T, Hq, D], lse [T, Hq] in 64 bits, and for each the error that products and sums in fp32 and weights in bf16 may have."""
    (T, Hq, D), Hkv = q.shape, cache.shape[1]
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    out_err, lse_err = torch.zeros_like(out), torch.zeros_like(lse)
    for b, n in enumerate(lens.tolist()):
        lo, hi = int(starts[b]), int(starts[b + 1])
        n = max(0, min(n, most, table.shape[1] * P))
        held = [j for j in range(n) if 0 <= int(table[b, j // P]) < cache.shape[0]]
        if not held:
            continue
        j = torch.tensor(held)
        kv = [get(cache, P, D, int(table[b, t // P]), t % P) for t in held]
        k, v = torch.stack([x for x, _ in kv], 1), torch.stack([x for _, x in kv], 1)             # [Hkv, n, D]
        for i in range(lo, hi):
            p = n - (hi - lo) + (i - lo)
            sees = (j <= p) & ((j > p - window) if window else torch.ones_like(j, dtype=torch.bool))
            if not sees.any():
                continue
            for h in range(Hq):
                kh, vh = k[h // (Hq // Hkv)][sees], v[h // (Hq // Hkv)][sees]
                x = q[i, h].double()
                s = scale * (kh @ x)
                lse[i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[i, h])
                out[i, h] = w @ vh
                # a score is off by D roundings of its sum and a few of its own, its weight by as much, relative, and by the
                # roundings of exp and of the sum of n weights; a weight for the product by a rounding to bf16 more
                ds = float((abs(scale) * (kh.abs() @ x.abs())).max()) * (D + 4) * 2 * F32_HALF
                rel = 2 * ds + (len(w) + 16) * 2 * F32_HALF
                # (weights under 2^-126 of the largest have no normal number in 32 bits and may be 0)
                out_err[i, h] = (w @ vh.abs()) * (rel + BF16_HALF) + out[i, h].abs() * BF16_HALF + vh.abs().sum(0) * 2.0 ** -126
                lse_err[i, h] = ds + (len(w) + 16) * 2 * F32_HALF + lse[i, h].abs() * 4 * F32_HALF
    return out, lse, out_err, lse_err


def product(x, codes, scales):
    """y [M, N] in 64 bits of x [M, K] and a weight in four bits, and the error that sums in fp32 may have."""
    w = decode(unpack(codes), scales)
    return x.double() @ w.t(), (x.double().abs() @ w.abs().t()) * x.shape[1] * 2 * F32_HALF
