"""Attention in 64 bits over keys and values that are at hand as numbers, whole matrices at a time (for lengths that mx_reference.attention, element by
element, is too slow for), and how far sums in 32 bits may be off before the result's one rounding to bf16."""
import math

import torch

BF16_HALF = 2.0 ** -8        # half a step of bf16, relative
F32_HALF = 2.0 ** -24
# What the weights lose on their way to the second product, relative.  Rounded to bf16: half a step.  With what that took off (at most half a step)
# multiplied too, in bf16 by cutting off its lower bits: a step of it, 2^-7 of 2^-8.
ROUNDED, WITH_REST = BF16_HALF, 2.0 ** -15


def attention(q, keys, values, starts, lens, scale, window=0, weights=ROUNDED):
    """q [T, Hq, D]; keys, values: of each sequence [its tokens, Hkv, D] in 64 bits; starts [B + 1], lens [B].  out, lse and the bounds of their errors,
    that of out without its last rounding.  Rows of no sequence are NaN."""
    T, Hq, D = q.shape
    out, lse = torch.full((T, Hq, D), math.nan, dtype=torch.float64), torch.full((T, Hq), math.nan, dtype=torch.float64)
    out_err, lse_err = torch.zeros_like(out), torch.zeros_like(lse)
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        if lo == hi:
            continue
        k, v = keys[b][:n], values[b][:n]
        group = Hq // k.shape[1]
        j, p = torch.arange(n), torch.arange(n - (hi - lo), n)[:, None]
        sees = (j <= p) & (j > p - window) if window else j <= p
        count = sees.sum(-1).double()
        for h in range(Hq):
            kh, vh, x = k[:, h // group], v[:, h // group], q[lo:hi, h].double()
            s = (scale * (x @ kh.t())).masked_fill(~sees, -math.inf)
            z = torch.logsumexp(s, -1)
            w = torch.nan_to_num(torch.exp(s - z[:, None]), nan=0.0)
            out[lo:hi, h], lse[lo:hi, h] = w @ vh, z
            # a score is off by D roundings of its sum and a few of its own, its weight by as much, relative, and by the roundings of exp and of
            # the sum of the weights; weights under 2^-126 of the largest may be 0
            ds = (abs(scale) * (x.abs() @ kh.abs().t())).masked_fill(~sees, 0.0).amax(-1) * (D + 4) * 2 * F32_HALF
            rel = 2 * ds + (count + 16) * 2 * F32_HALF
            out_err[lo:hi, h] = (w @ vh.abs()) * (rel + weights)[:, None] + sees.double() @ vh.abs() * 2.0 ** -126
            lse_err[lo:hi, h] = ds + (count + 16) * 2 * F32_HALF + torch.nan_to_num(z.abs(), posinf=0.0) * 4 * F32_HALF
    return out, lse, out_err, lse_err


def outside(got, want, err):
    """How many elements of `got` (bf16) are not the rounding of any number that is off from `want` by at most `err` (roundings keep the order)."""
    low, high = ((want + s * err).float().to(torch.bfloat16).double() for s in (-1, 1))
    got = got.double().cpu()
    return int((~((got >= low) & (got <= high))).sum())
