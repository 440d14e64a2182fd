"""The bounds of tests/mx_attention_bounds.py, on the CPU: what they let pass and what they catch, with mistakes planted in a model of the arithmetic."""
import math

import pytest
import torch

import mx_attention_bounds as bounds


def _model(q, k, v, scale, rest):
    """One query token after all of k, v [n, 1, D]: weights in fp32, rounded to bf16 for the product; `rest` of what that took off is added."""
    s = (q[0].float() @ k[:, 0].float().t()) * scale
    e = torch.exp(s - s.amax(-1, keepdim=True))
    p = e.to(torch.bfloat16).float()
    return ((p.double() + rest(e - p).double()) @ v[:, 0] / e.double().sum(-1, keepdim=True)).float().to(torch.bfloat16)[None]


def _cut(r):
    return (r.view(torch.int32) & -65536).view(torch.float32)


CASES = [(8, 64, 64), (16, 128, 64), (4, 128, 70), (8, 256, 60), (20, 256, 50)]


def _case(Hq, D, n):
    gen = torch.Generator().manual_seed(1)
    q = (torch.randn((1, Hq, D), generator=gen) * 0.1).to(torch.bfloat16)
    k, v = (torch.randn((n, 1, D), generator=gen).to(torch.bfloat16).double() for _ in range(2))
    return q, k, v, 1 / math.sqrt(D)


@pytest.mark.parametrize("Hq,D,n", CASES)
def test_weights_with_what_their_rounding_took_off(Hq, D, n):
    q, k, v, scale = _case(Hq, D, n)
    want, _, err, _ = bounds.attention(q, [k], [v], [0, 1], [n], scale, weights=bounds.WITH_REST)
    assert bounds.outside(_model(q, k, v, scale, _cut), want, err) == 0
    # without it, with the wrong half of its bits, and subtracted
    for rest in (torch.zeros_like, lambda r: (r.view(torch.int32) << 16).view(torch.float32).nan_to_num(0.0, 0.0, 0.0).clamp(-1, 1), lambda r: -_cut(r)):
        assert bounds.outside(_model(q, k, v, scale, rest), want, err) > want.numel() // 50


@pytest.mark.parametrize("Hq,D,n", CASES)
def test_weights_rounded_to_bf16(Hq, D, n):
    q, k, v, scale = _case(Hq, D, n)
    want, _, err, _ = bounds.attention(q, [k], [v], [0, 1], [n], scale)
    assert bounds.outside(_model(q, k, v, scale, torch.zeros_like), want, err) == 0
    assert bounds.outside(_model(q, k, v * 1.02, scale, torch.zeros_like), want, err) > 0


def test_the_matrices_say_what_the_elements_say():
    """Against tests/mx_reference.py, which goes through a cache token by token."""
    import mx_reference as ref
    gen = torch.Generator().manual_seed(2)
    Hq, Hkv, D, P, lens, starts = 4, 2, 64, 16, [40, 9, 3], [0, 7, 8, 13]
    cache = torch.zeros((8, Hkv, ref.block_bytes(P, D)), dtype=torch.uint8)
    table = torch.arange(9).view(3, 3).clamp(max=7).to(torch.int32)
    keys, values = [], []
    for b, n in enumerate(lens):
        cache = ref.append(cache, P, torch.randn((n, Hkv, D), generator=gen).double(), torch.randn((n, Hkv, D), generator=gen).double(), b * 48 + torch.arange(n))
        kv = [ref.get(cache, P, D, int(table[b, t // P]), t % P) for t in range(n)]
        keys.append(torch.stack([k for k, _ in kv]))
        values.append(torch.stack([v for _, v in kv]))
    q = torch.randn((13, Hq, D), generator=gen).to(torch.bfloat16)
    for window in (0, 5):
        want = ref.attention(q, cache, P, table, torch.tensor(lens), starts, -0.3, window)
        got = bounds.attention(q, keys, values, starts, lens, -0.3, window)
        for a, b in zip(got[:2], want[:2]):
            seen = torch.isfinite(b)
            assert torch.equal(a[~seen], b[~seen]) and float((a - b)[seen].abs().max()) < 1e-12
