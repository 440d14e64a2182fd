"""Drafted tokens in a tree written out in 64 bits on the CPU, a row at a time."""
import math

import numpy as np
import torch

import mx_reference as ref


def above(parents, lo, i):
    """The row above row i of a sequence whose rows begin at lo; -1: none."""
    p = i - 1 if parents is None else int(parents[lo + i])
    return p if 0 <= p < i else -1


def climb(parents, lo, i):
    """Row i and those above it, from below."""
    path = []
    while i >= 0:
        path.append(i)
        i = above(parents, lo, i)
    return path


def spans(starts, T):
    """First row and one past the last of each sequence."""
    s = [min(max(int(x), 0), T) for x in starts]
    return [(s[b], max(s[b], s[b + 1])) for b in range(len(s) - 1)]


def tree(parents, starts, T, lens, words, table=None, P=16):
    """Masks [T][words] (as whole numbers), positions and slots [T]; None for rows of no sequence."""
    masks, positions, slots = [None] * T, [None] * T, [None] * T
    for b, (lo, hi) in enumerate(spans(starts, T)):
        for i in range(hi - lo):
            path = climb(parents, lo, i)
            bits = sum(1 << j for j in path)
            masks[lo + i] = [(bits >> (32 * w)) & 0xffffffff for w in range(words)]
            base = int(lens[b]) - (hi - lo)
            positions[lo + i] = base + len(path) - 1
            place = base + i
            slots[lo + i] = -1
            if table is not None and 0 <= place < table.shape[1] * P and int(table[b, place // P]) >= 0:
                slots[lo + i] = int(table[b, place // P]) * P + place % P
    return masks, positions, slots


def attention(q, cache, P, table, lens, starts, masks, scale, window=0, most=1 << 30):
    """out [T, Hq, D], lse [T, Hq] in 64 bits for rows with masks [T, words] (int32), and for each the error that products and sums in fp32 and weights in bf16 may have; rows
    of no sequence are NaN."""
    (T, Hq, D), Hkv = q.shape, cache.shape[1]
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    out_err, lse_err = torch.zeros_like(out), torch.zeros_like(lse)
    for b, (lo, hi) in enumerate(spans(starts, T)):
        m, n = hi - lo, max(0, min(int(lens[b]), most, table.shape[1] * P))
        held = {j for j in range(n) if 0 <= int(table[b, j // P]) < cache.shape[0]}
        kv = {j: ref.get(cache, P, D, int(table[b, j // P]), j % P) for j in held}
        for i in range(lo, hi):
            words = [int(w) & 0xffffffff for w in masks[i].tolist()]
            sees = [j for j in range(n) if j < n - m or (words[(j - n + m) // 32] >> ((j - n + m) % 32) & 1 if (j - n + m) // 32 < len(words) else 0)]
            if window:
                sees = sees[-window:]
            sees = [j for j in sees if j in held]
            if not sees:
                continue
            k, v = torch.stack([kv[j][0] for j in sees], 1), torch.stack([kv[j][1] for j in sees], 1)             # [Hkv, n, D]
            for h in range(Hq):
                kh, vh, x = k[h // (Hq // Hkv)], v[h // (Hq // Hkv)], q[i, h].double()
                s = scale * (kh @ x)
                lse[i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[i, h])
                out[i, h] = w @ vh
                # a score is off by D roundings of its sum and a few of its own, its weight by as much, relative, and by the roundings of exp and of the sum of
                # n weights; a weight for the product by a rounding to bf16 more
                ds = float((abs(scale) * (kh.abs() @ x.abs())).max()) * (D + 4) * 2 * ref.F32_HALF
                rel = 2 * ds + (len(w) + 16) * 2 * ref.F32_HALF
                out_err[i, h] = (w @ vh.abs()) * (rel + ref.BF16_HALF) + out[i, h].abs() * ref.BF16_HALF + vh.abs().sum(0) * 2.0 ** -126
                lse_err[i, h] = ds + (len(w) + 16) * 2 * ref.F32_HALF + lse[i, h].abs() * 4 * ref.F32_HALF
    return out, lse, out_err, lse_err


def chances(logits, t):
    """softmax(logits / t): NaN as minus infinity, infinity as the largest number; zeros where there is nothing."""
    x = logits.double().numpy().copy()
    x[np.isnan(x)] = -math.inf
    x = np.minimum(x, 3.4028234663852886e38)
    if not len(x) or x.max() == -math.inf:
        return np.zeros_like(x)
    e = np.where(x == -math.inf, 0.0, np.exp((x - x.max()) / t))
    return e / e.sum()


def largest(logits):
    x = logits.double().numpy().copy()
    x[np.isnan(x)] = -math.inf
    x = np.minimum(x, 3.4028234663852886e38)
    return int(np.argmax(x)) if len(x) and x.max() > -math.inf else -1


def verify(target, draft, tokens, parents, max_children, starts, temperatures, uniforms, known=512):
    """Rows, tokens and counts that come out (None for rows of no sequence), by the definition; `known` rows of a sequence at most are tried."""
    T, V = target.shape
    rows, out, counts = [None] * T, [None] * T, []
    for b, (lo, hi) in enumerate(spans(starts, T)):
        if hi == lo:
            counts.append(0)
            continue
        t = 1.0 if temperatures is None else float(temperatures[b])
        greedy = not t > 0
        path, got, at = [0], [], 0
        while True:
            children = [i for i in range(1, min(hi - lo, known)) if above(parents, lo, i) == at and 0 <= int(tokens[lo + i]) < V][:max_children]
            down = None
            if greedy:
                best = largest(target[lo + at])
                down = next((i for i in children if int(tokens[lo + i]) == best), None)
            else:
                p = chances(target[lo + at], t)
                r = p.copy()
                q = None if draft is None or not children else chances(draft[lo + at], t)
                for i in children:
                    x, u = int(tokens[lo + i]), float(uniforms[lo + i])
                    if u * (1.0 if q is None else q[x]) < r[x]:
                        down = i
                        break
                    if q is None:
                        r[x] = 0.0
                    else:
                        r = np.maximum(r - q, 0.0)
                    if r.sum() > 0:
                        r = r / r.sum()
                    else:
                        r = p.copy()
            if down is None:
                break
            at = down
            path.append(at)
            got.append(int(tokens[lo + at]))
        if greedy:
            got.append(best)
        elif r.sum() == 0:
            got.append(-1)
        else:
            below = np.cumsum(r)
            past = np.nonzero((below > float(uniforms[lo]) * below[-1]) & (r > 0))[0]
            got.append(int(past[0]) if len(past) else int(np.nonzero(r)[0][-1]))
        n = hi - lo
        rows[lo:hi] = path + [-1] * (n - len(path))
        out[lo:hi] = got + [-1] * (n - len(got))
        counts.append(len(path))
    return rows, out, counts


def keep(cache, P, D, table, lens, starts, rows, counts, most=1 << 30):
    """The cache and the lengths after the rows that stay have been moved together."""
    cache, G = cache.clone(), D // 32
    pages, new = cache.shape[0], []
    most = min(most, table.shape[1] * P)

    def parts(block, at):
        """Views of what token `at` has in a block: key codes, key scales, value codes, value scales."""
        q, t = divmod(at, 4)
        to = P * (D // 2 + G)
        return (block[at * (D // 2):(at + 1) * (D // 2)], block[P * (D // 2) + at * G:P * (D // 2) + (at + 1) * G],
                block[to:to + P * (D // 2)].view(P // 4, 16, G, 4)[q, :, :, t], block[to + P * (D // 2):].view(P // 4, G, 4)[q, :, t])

    for b, (lo, hi) in enumerate(spans(starts, len(rows))):
        m = hi - lo
        count = min(max(int(counts[b]), 0), m)
        base = int(lens[b]) - m
        new.append(max(base + count, 0))
        for i in range(count):
            r = int(rows[lo + i])
            if not (i < r < m) or base + i < 0 or base + r >= most:
                continue
            p0, p1 = int(table[b, (base + r) // P]), int(table[b, (base + i) // P])
            if not (0 <= p0 < pages and 0 <= p1 < pages):
                continue
            for h in range(cache.shape[1]):
                src, dst = parts(cache[p0, h], (base + r) % P), parts(cache[p1, h], (base + i) % P)
                for s, d in zip(src, dst):
                    d.copy_(s.clone())
    return cache, new
