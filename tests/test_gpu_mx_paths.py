"""Attention over the four-bit cache where a call's shares, page numbers and forms meet: against 64 bits (tests/mx_attention_bounds.py), on keys and
values that mom_mx_kv_append stores and mom_mx_kv_read reads back."""
import math

import pytest
import torch

import mx_attention_bounds as bounds
import mx_reference as ref
from paper_2504_12526_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _fill(gen, Hkv, D, P, lens, max_kv, values=1.0):
    """A cache whose pages are in any order, noise (NaN among it) wherever nothing is stored; the table, and each sequence's keys and values."""
    each = -(-max_kv // P)
    pool = torch.randperm(sum(-(-n // P) for n in lens) + 3, generator=gen)
    table, used = torch.full((len(lens), each), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        table[b, :-(-n // P)] = pool[used:used + -(-n // P)]
        used += -(-n // P)
    cache = torch.randint(0, 256, (len(pool), Hkv, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8).to(DEV)
    slots = torch.cat([table[b].long()[torch.arange(n) // P] * P + torch.arange(n) % P for b, n in enumerate(lens)]).to(DEV)
    k, v = (torch.randn((len(slots), Hkv, D), generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    binding.mom_mx_kv_append(k, v * values, slots, cache, P)
    binding.mom_mx_kv_read(cache, P, slots, k, v)
    return cache, table, [t.double() for t in k.cpu().split(lens)], [t.double() for t in v.cpu().split(lens)]


def _run(q, cache, P, table, lens, max_kv, starts=None, scale=None, window=0):
    (T, Hq, D), Hkv = q.shape, cache.shape[1]
    out, lse = torch.full((T, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((T, Hq), 3.0, device=DEV)
    n = binding.mom_mx_attention_workspace_bytes(T, table.shape[0], Hq, Hkv, D, max_kv)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None            # NaN wherever nothing is written
    starts = None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
    binding.mom_mx_attention(q.to(DEV), cache, P, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), max_kv, out, ws, q_starts=starts, scale=scale,
                             window=window, lse=lse)
    return out, lse, n


def _near(lse, z, err):
    lse, seen = lse.double().cpu(), torch.isfinite(z)
    assert torch.equal(lse[~seen], z[~seen]) and float(((lse - z).abs() - err)[seen].max()) <= 0


def _compare(seed, Hq, Hkv, D, P, lens, asked, max_kv=None, window=0, shared=None, listed=True, std=1.0, weights=bounds.ROUNDED):
    gen = torch.Generator().manual_seed(seed)
    max_kv = max(lens) if max_kv is None else max_kv
    cache, table, keys, values = _fill(gen, Hkv, D, P, lens, max_kv)
    starts = [0] + torch.tensor(asked).cumsum(0).tolist()
    q = (torch.randn((starts[-1], Hq, D), generator=gen) * std).to(torch.bfloat16)
    out, lse, workspace = _run(q, cache, P, table, lens, max_kv, starts if listed else None, None, window)
    if shared is not None:
        assert (workspace > 0) == shared
    want, z, err, z_err = bounds.attention(q, keys, values, starts, lens, 1 / math.sqrt(D), window, weights)
    assert bounds.outside(out, want, err) == 0
    _near(lse, z, z_err)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 1, 64), (4, 2, 256)])
@pytest.mark.parametrize("starts,T", [([0, 2, 5], 9), ([3, 4, 6], 8), ([1, 1, 3], 3)])
def test_tokens_of_no_sequence_are_left_alone_where_shares_are_joined(Hq, Hkv, D, starts, T):
    gen = torch.Generator().manual_seed(1)
    lens = [3000, 40]
    cache, table, keys, values = _fill(gen, Hkv, D, 16, lens, 3000)
    q = torch.randn((T, Hq, D), generator=gen).to(torch.bfloat16)
    out, lse, workspace = _run(q, cache, 16, table, lens, 3000, starts)
    assert workspace > 0
    want, z, err, z_err = bounds.attention(q, keys, values, starts, lens, 1 / math.sqrt(D))
    inside = slice(starts[0], starts[-1])
    assert bounds.outside(out[inside], want[inside], err[inside]) == 0
    _near(lse[inside], z[inside], z_err[inside])
    none = [i for i in range(T) if not starts[0] <= i < starts[-1]]
    assert (out[none] == 3).all() and (lse[none] == 3).all()


def test_rows_of_no_sequence_beside_a_chunk_in_shares():
    gen = torch.Generator().manual_seed(2)
    starts, T, lens, D = [20, 120], 150, [3000], 128
    cache, table, keys, values = _fill(gen, 1, D, 64, lens, 3000)
    q = torch.randn((T, 4, D), generator=gen).to(torch.bfloat16)
    out, lse, workspace = _run(q, cache, 64, table, lens, 3000, starts)
    assert workspace > 0
    want, _, err, _ = bounds.attention(q, keys, values, starts, lens, 1 / math.sqrt(D))
    assert bounds.outside(out[20:120], want[20:120], err[20:120]) == 0
    none = list(range(20)) + list(range(120, T))
    assert (out[none] == 3).all() and (lse[none] == 3).all()


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("lens,asked,max_kv,window", [([3000], [100], 3000, 0), ([3000], [100], 3000, 700), ([700], [100], 3000, 0), ([2900, 60, 1500], [90, 70, 101], 2900, 0),
                                                      ([2000], [90], 2000, 1)])
def test_many_rows_in_shares(D, P, lens, asked, max_kv, window):
    """Parts of the tokens, empty ones among them, for wavefronts with and without rows; past 1024 tokens the page numbers are looked up again."""
    _compare(3, 4, 1, D, P, lens, asked, max_kv, window, shared=True)


@pytest.mark.parametrize("D,P", [(64, 16), (128, 128), (256, 16)])
def test_many_rows_in_one_share_past_1024_tokens(D, P):
    _compare(4, 130, 130, D, P, [1300], [258], shared=False)


@pytest.mark.parametrize("Hq,Hkv,D,m,listed,shared", [(8, 8, 64, 1, True, False), (8, 8, 128, 1, False, False), (8, 8, 256, 1, True, False),
                                                      # (of 20 rows each; the workspace is the larger one of sequences with and without starts)
                                                      (12, 3, 64, 5, True, None), (12, 3, 128, 5, True, None), (16, 4, 128, 5, False, None)])
def test_more_than_32_steps_of_a_wavefront(Hq, Hkv, D, m, listed, shared):
    """Many tiles and one sequence of more than 8192 tokens, in one share: the page numbers are looked up again."""
    B = 64
    _compare(5, Hq, Hkv, D, 16, [9300] + [m + (7 * b) % 50 for b in range(1, B)], [m] * B, listed=listed, shared=shared)


@pytest.mark.parametrize("D", [64, 128])
def test_more_than_32_steps_of_a_wavefront_in_shares(D):
    B = 63
    _compare(7, 2, 1, D, 256, [72000] + [1 + 5 * b for b in range(1, B)], [1] * B, shared=True)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (4, 1, 64), (7, 1, 128)])
@pytest.mark.parametrize("lens,asked,max_kv,window", [([2500, 300], [7, 9], 2500, 0), ([2500, 300], [7, 9], 2500, 1300), ([400], [12], 2500, 0)])
def test_a_few_rows_in_shares(Hq, Hkv, D, lens, asked, max_kv, window):
    _compare(8, Hq, Hkv, D, 16, lens, asked, max_kv, window, shared=True)


@pytest.mark.parametrize("Hq,Hkv,D,lens,asked", [(8, 1, 64, [64], [1]), (16, 1, 128, [64], [1]), (4, 2, 128, [70, 33, 64], [1, 1, 1]), (8, 1, 256, [60], [1]), (20, 1, 256, [50], [1]),
                                                 (4, 1, 64, [64], [3]), (4, 4, 256, [64] * 15, [1] * 15), (40, 10, 128, [61] * 6, [1] * 6)])
def test_few_tiles_of_few_rows_have_the_rounding_of_the_result_alone(Hq, Hkv, D, lens, asked):
    """Up to 16 rows a sequence (any number up to 256 where there are 256 dimensions) and fewer than 64 tiles: weights near one another, so that what they lose
    by their rounding to bf16 shows in the result."""
    _compare(9, Hq, Hkv, D, 16, lens, asked, std=0.1, weights=bounds.WITH_REST)


@pytest.mark.parametrize("kind", ["keys", "values"])
def test_append_of_numbers_below_the_smallest_scale(kind):
    """Subnormal bf16 numbers, which 2^-125 brings to at most half a step of the largest, and zeros."""
    D, P = 64, 16
    bits = torch.arange(0, 256, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros(4, 1, D, dtype=torch.bfloat16)
    x[0, 0, :], x[1, 0, :], x[2, 0, :], x[3, 0, :] = bits[:64], bits[64:128], -bits[128:192], bits[192:256]
    y = torch.ones_like(x)
    k, v = (x, y) if kind == "keys" else (y, x)
    cache = torch.zeros(1, 1, ref.block_bytes(P, D), dtype=torch.uint8)
    got = cache.to(DEV)
    binding.mom_mx_kv_append(k.to(DEV), v.to(DEV), torch.arange(4).to(DEV), got, P)
    assert torch.equal(got.cpu(), ref.append(cache, P, k.double(), v.double(), torch.arange(4)))


def test_quantize_of_numbers_below_the_smallest_scale():
    w = torch.arange(0, 256, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(4, 64).clone()
    codes, scales = torch.empty((4, 32), dtype=torch.uint8, device=DEV), torch.empty((4, 2), dtype=torch.uint8, device=DEV)
    binding.mom_mx_quantize(w.to(DEV), codes, scales)
    c, s = ref.encode(w.double())
    assert torch.equal(codes.cpu(), ref.pack(c)) and torch.equal(scales.cpu(), s.to(torch.uint8))


def test_a_table_beside_the_result():
    """Rows of a page table that lie apart: what lies between and behind them is not the table's, and may be the result's."""
    gen = torch.Generator().manual_seed(10)
    D, P, lens, starts = 64, 16, [64, 37], [0, 1, 2]
    cache, table, keys, values = _fill(gen, 1, D, P, lens, 64)
    buf = torch.full((4096,), -1, dtype=torch.int32, device=DEV)
    wide = buf[:128 + 4].as_strided((2, 4), (128, 1))         # four pages a row, 128 entries from row to row
    wide.copy_(table)
    out = buf[136:136 + 2 * 2 * D // 2].view(torch.bfloat16).view(2, 2, D)
    q = torch.randn((2, 2, D), generator=gen).to(torch.bfloat16)
    binding.mom_mx_attention(q.to(DEV), cache, P, wide, torch.tensor(lens, dtype=torch.int32, device=DEV), 64, out, None)
    want, _, err, _ = bounds.attention(q, keys, values, starts, lens, 1 / math.sqrt(D))
    assert bounds.outside(out, want, err) == 0


def test_a_table_without_pages():
    """No pages yet: nothing is seen."""
    cache = torch.zeros((1, 1, ref.block_bytes(16, 64)), dtype=torch.uint8, device=DEV)
    q, out, lse = torch.ones((2, 2, 64), dtype=torch.bfloat16, device=DEV), torch.full((2, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((2, 2), 3.0, device=DEV)
    binding.mom_mx_attention(q, cache, 16, torch.empty((2, 0), dtype=torch.int32, device=DEV), torch.tensor([5, 0], dtype=torch.int32, device=DEV), 64, out, None, lse=lse)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("M", [1, 5, 16])
@pytest.mark.parametrize("N,K", [(300, 1056), (70, 64), (40, 4096), (33, 14336), (32900, 96)])
@pytest.mark.parametrize("offset", [1, 6, 13])
def test_scales_at_any_byte(M, N, K, offset):
    """Rows cut out of a larger weight: codes on 16 bytes, scales anywhere."""
    gen = torch.Generator().manual_seed(11)
    x = torch.randn((M, K), generator=gen).to(torch.bfloat16).to(DEV)
    codes = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8).to(DEV)
    scales = torch.randint(118, 126, (N, K // 32), generator=gen, dtype=torch.uint8).to(DEV)
    moved = torch.full((scales.numel() + 32,), 255, dtype=torch.uint8, device=DEV)[offset:offset + scales.numel()].view_as(scales)
    moved.copy_(scales)
    want, got = (torch.empty((M, N), device=DEV) for _ in range(2))
    binding.mom_mx_matvec(x, codes, scales, want)
    binding.mom_mx_matvec(x, codes, moved, got)
    assert torch.isfinite(want).all() and torch.equal(got, want)
    want, got = (torch.empty((M, N), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    binding.mom_mx_gateup(x, codes, scales, codes, scales, want)
    binding.mom_mx_gateup(x, codes, moved, codes, moved, got)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
