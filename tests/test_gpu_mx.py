"""The four-bit operators on the GPU, through the C ABI, against tests/mx_reference.py: at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import mx_reference as ref
from paper_2504_12526_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen) * std).to(torch.bfloat16)


def _noise(gen, pages, heads, P, D):
    """A cache full of whatever was there before, NaN scales among it."""
    return torch.randint(0, 256, (pages, heads, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8)


def _within(got, want, err, what=""):
    got, want = got.double().cpu(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, "NaN", int(torch.isnan(got).sum()), int(torch.isnan(want).sum()))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), (what, "infinities")
    fine = torch.isfinite(want)
    off = ((got - want).abs() - err)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), int((off > 0).sum()))


# Append and read

def _append_case(T, Hq, Hkv, D, P, rot, interleaved, far, seed, strided=True):
    gen = _gen(seed)
    qkv = _normal(gen, T, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if not strided:
        q, k, v = (t.contiguous() for t in (q, k, v))
    pages = -(-T // P) + 2
    slots = torch.randperm(pages * P, generator=gen)[:T]
    positions = torch.randint(0, far + 1, (T,), generator=gen).to(torch.int32)
    inv_freq = (500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float()
    return qkv, q, k, v, slots, positions, inv_freq, _noise(gen, pages, Hkv, P, D)


def _on_gpu(qkv, q, k, v):
    """The same slices of the same tensor on the GPU where they are slices of one."""
    if q.is_contiguous() and k.is_contiguous():
        return tuple(t.to(DEV) for t in (q, k, v))
    g, a, b = qkv.to(DEV), q.shape[1], q.shape[1] + k.shape[1]
    return g[:, :a], g[:, a:b], g[:, b:]


@pytest.mark.parametrize("T,Hq,Hkv,D,P,rot,interleaved,far", [
    (1, 32, 8, 128, 16, 128, False, 32767),
    (5, 28, 4, 128, 64, 128, False, 1048575),
    (3, 8, 8, 64, 32, 64, True, 131071),
    (37, 5, 1, 64, 16, 32, False, 4095),
    (9, 4, 2, 256, 128, 256, False, 262143),
    (7, 6, 3, 256, 256, 96, True, 1000),
    (130, 7, 3, 128, 16, 16, True, 458751),
    (600, 4, 2, 128, 32, 128, False, 458751),
    (21, 3, 3, 128, 16, 0, False, 10),
])
def test_append_and_read(T, Hq, Hkv, D, P, rot, interleaved, far):
    qkv, q, k, v, slots, positions, inv_freq, cache = _append_case(T, Hq, Hkv, D, P, rot, interleaved, far, 1)
    if T > 4:
        slots[1], slots[3] = -1, cache.shape[0] * P          # padding: stored nowhere
    gq, gk, gv = _on_gpu(qkv, q, k, v)
    gc, q_out = cache.to(DEV), torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    rotation = {} if rot == 0 else {"positions": positions.to(DEV), "inv_freq": inv_freq.to(DEV), "interleaved": interleaved}
    binding.mom_mx_kv_append(gk, gv, slots.to(DEV), gc, P, q=gq, q_out=q_out, **rotation)
    want_k = ref.rotate(k, positions, inv_freq, interleaved)
    want = ref.append(cache, P, want_k, v.double(), slots)
    assert torch.equal(gc.cpu(), want)                        # every byte of the cache, those of other tokens too
    want_q = ref.rotate(q, positions, inv_freq, interleaved)
    # rounded once, by way of fp32; a difference of two products may cancel, which 64 bits carry
    _within(q_out, want_q, want_q.abs() * (ref.BF16_HALF + 2 * ref.F32_HALF) + 1e-14)
    ko, vo = (torch.full((T, Hkv, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    binding.mom_mx_kv_read(gc, P, slots.to(DEV), ko, vo)
    for i, slot in enumerate(slots.tolist()):
        held = 0 <= slot < cache.shape[0] * P
        wk, wv = ref.get(want, P, D, slot // P, slot % P) if held else (torch.zeros(Hkv, D).double(),) * 2
        assert torch.equal(ko[i].double().cpu(), wk) and torch.equal(vo[i].double().cpu(), wv), (i, slot)


def test_append_of_a_long_prompt_fills_its_pages():
    """One head, 16640 tokens in order: every wavefront a token of its own, and offsets of many pages."""
    T, Hkv, D, P = 16640, 1, 64, 64
    qkv, q, k, v, _, positions, inv_freq, cache = _append_case(T, 1, Hkv, D, P, D, False, 16639, 3)
    slots = torch.arange(T)
    gq, gk, gv = _on_gpu(qkv, q, k, v)
    gc = cache.to(DEV)
    binding.mom_mx_kv_append(gk, gv, slots.to(DEV), gc, P, positions=positions.to(DEV), inv_freq=inv_freq.to(DEV))
    ko, vo = (torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    binding.mom_mx_kv_read(gc, P, slots.to(DEV), ko, vo)
    assert torch.equal(ko.double().cpu(), ref.decode(*ref.encode(ref.rotate(k, positions, inv_freq, False))))
    assert torch.equal(vo.double().cpu(), ref.decode(*ref.encode(v.double())))


def test_append_of_infinities_nan_zeros_and_extremes():
    T, H, D, P = 8, 1, 64, 16
    gen = _gen(4)
    k, v = _normal(gen, T, H, D), _normal(gen, T, H, D)
    for t in (k, v):
        t[0, 0, 3] = math.nan
        t[1, 0, 40] = math.inf
        t[2, 0, 8] = -math.inf
        t[3] = 0.0
        t[4, 0, :32] = torch.finfo(torch.bfloat16).max
        t[5, 0, :32] = torch.finfo(torch.bfloat16).tiny
        t[6, 0, 32:] = -0.0
        t[6, 0, 33] = 7.0
        t[7, 0, :32] = torch.tensor([7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 4)
    slots, cache = torch.arange(T) + 3, _noise(gen, 1, H, P, D)
    gc = cache.to(DEV)
    binding.mom_mx_kv_append(k.to(DEV), v.to(DEV), slots.to(DEV), gc, P)
    assert torch.equal(gc.cpu(), ref.append(cache, P, k.double(), v.double(), slots))
    ko, vo = (torch.empty((T, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    binding.mom_mx_kv_read(gc, P, slots.to(DEV), ko, vo)
    for o in (ko.cpu(), vo.cpu()):
        assert o[0, 0, :32].isnan().all() and not o[0, 0, 32:].isnan().any() and o[1, 0, 32:].isnan().all() and o[2, 0, :32].isnan().all()
        assert (o[3] == 0).all() and (o[4, 0, :32] == 6 * 2.0 ** 125).all() and (o[7, 0, 0] == 6)


def test_append_rotates_dense_queries_in_place():
    T, Hq, Hkv, D, P = 6, 3, 1, 128, 16
    qkv, q, k, v, slots, positions, inv_freq, cache = _append_case(T, Hq, Hkv, D, P, 128, False, 5000, 5, strided=False)
    gq, gk, gv = _on_gpu(qkv, q, k, v)
    gc, q_out = cache.to(DEV), torch.empty_like(gq)
    args = dict(positions=positions.to(DEV), inv_freq=inv_freq.to(DEV))
    binding.mom_mx_kv_append(gk, gv, slots.to(DEV), gc, P, q=gq, q_out=q_out, **args)
    binding.mom_mx_kv_append(gk, gv, slots.to(DEV), gc, P, q=gq, q_out=gq, **args)
    assert torch.equal(gq.view(torch.int16), q_out.view(torch.int16))


def test_append_rotates_infinities_and_nan():
    """An infinity stays one, opposite ones and NaN are NaN, in the two dimensions that they turn into and nowhere else."""
    T, D, P = 4, 64, 16
    gen = _gen(6)
    q, k = _normal(gen, T, 1, D), _normal(gen, T, 1, D)
    q[0, 0, 3], q[1, 0, 40], q[2, 0, 5], q[3, 0, 7], q[3, 0, 39] = math.inf, -math.inf, math.nan, math.inf, math.inf
    positions, inv_freq = torch.tensor([1, 5, 9, 100], dtype=torch.int32), (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float()
    q_out = torch.empty_like(q, device=DEV)
    binding.mom_mx_kv_append(k.to(DEV), k.to(DEV), torch.arange(T).to(DEV), torch.zeros(1, 1, ref.block_bytes(P, D), dtype=torch.uint8, device=DEV), P,
                             positions=positions.to(DEV), inv_freq=inv_freq.to(DEV), q=q.to(DEV), q_out=q_out)
    want = ref.rotate(q, positions, inv_freq, False)
    assert torch.isinf(want[:2]).sum() == 4 and torch.isnan(want).sum() >= 2
    _within(q_out, want, want.abs() * (ref.BF16_HALF + 2 * ref.F32_HALF) + 1e-14)


# Attention

def _sequences(gen, Hkv, D, P, lens, extra=3, values=1.0):
    """A cache with sequences of these lengths on pages in any order, what was there before behind and between them; the table."""
    each = max(1, max(-(-n // P) for n in lens))
    pool = torch.randperm(len(lens) * each + extra, generator=gen)
    table = pool[:len(lens) * each].view(len(lens), each).to(torch.int32)
    cache = _noise(gen, len(pool), Hkv, P, D)
    for b, n in enumerate(lens):
        if n:
            slots = table[b].long()[torch.arange(n) // P] * P + torch.arange(n) % P
            cache = ref.append(cache, P, torch.randn((n, Hkv, D), generator=gen).double(), torch.randn((n, Hkv, D), generator=gen).double() * values, slots)
    return cache, table


def _attend(q, cache, P, table, lens, max_kv, starts=None, scale=None, window=0, with_lse=True, stream=None):
    (T, Hq, D), (_, Hkv, _) = q.shape, cache.shape
    out = torch.full((T, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, Hq), 3.0, dtype=torch.float32, device=DEV) if with_lse else None
    n = binding.mom_mx_attention_workspace_bytes(T, table.shape[0], Hq, Hkv, D, max_kv)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None            # NaN wherever nothing is written
    binding.mom_mx_attention(q, cache, P, table, lens, max_kv, out, ws, q_starts=starts, scale=scale, window=window, lse=lse, stream=stream)
    return out, lse


def _compare(gen, Hq, Hkv, D, P, lens, asked, window=0, scale=None, starts=True, max_kv=None, table_of=None, q=None, cache_table=None):
    cache, table = cache_table or _sequences(gen, Hkv, D, P, lens)
    if table_of:
        table = table_of(table, cache)
    T = sum(asked)
    if q is None:
        q = _normal(gen, T, Hq, D)
    at = torch.tensor([0] + asked).cumsum(0)
    max_kv = max(lens) if max_kv is None else max_kv
    out, lse = _attend(q.to(DEV), cache.to(DEV), P, table.to(DEV), torch.tensor(lens, dtype=torch.int32).to(DEV), max_kv,
                       at.to(torch.int32).to(DEV) if starts else None, scale, window)
    want = ref.attention(q, cache, P, table, torch.tensor(lens), at, 1 / math.sqrt(D) if scale is None else scale, window, max_kv)
    _within(out, want[0], want[2], "out")
    _within(lse, want[1], want[3], "lse")
    return out, lse


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 16), (7, 1, 128, 64), (4, 4, 64, 32), (16, 1, 64, 16), (2, 2, 256, 128), (20, 1, 256, 16), (24, 1, 128, 256), (40, 1, 64, 16)])
@pytest.mark.parametrize("lens", [[1], [2, 31], [32, 33, 17], [100, 1, 257]])
def test_one_token_a_sequence(Hq, Hkv, D, P, lens):
    _compare(_gen(10), Hq, Hkv, D, P, lens, [1] * len(lens))
    _compare(_gen(11), Hq, Hkv, D, P, lens, [1] * len(lens), starts=False)


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 16), (7, 1, 128, 64), (3, 3, 64, 16), (4, 1, 256, 32)])
@pytest.mark.parametrize("lens,asked,window", [
    ([5], [5], 0), ([40, 37], [3, 7], 0), ([130], [65], 0), ([70, 9, 300], [1, 9, 20], 0), ([140, 80], [33, 2], 20), ([200], [17], 1), ([257], [9], 64), ([90], [90], 31),
])
def test_several_tokens_a_sequence(Hq, Hkv, D, P, lens, asked, window):
    _compare(_gen(12), Hq, Hkv, D, P, lens, asked, window)


@pytest.mark.parametrize("Hq,Hkv,D,P,n,m,window", [(4, 1, 128, 16, 400, 300, 0), (2, 1, 64, 64, 333, 333, 0), (8, 1, 128, 32, 260, 129, 50), (1, 1, 256, 16, 200, 150, 0), (3, 1, 128, 16, 290, 280, 0)])
def test_a_chunk_of_a_prompt(Hq, Hkv, D, P, n, m, window):
    _compare(_gen(13), Hq, Hkv, D, P, [n], [m], window)


@pytest.mark.parametrize("Hq,Hkv,D,P,lens,asked,window", [
    (4, 1, 128, 64, [5000], [1], 0), (2, 2, 64, 16, [3000, 1, 700], [1, 1, 1], 0), (4, 1, 256, 256, [2100], [2], 0), (4, 2, 128, 16, [2500], [3], 1100), (2, 1, 64, 32, [1500], [90], 0),
])
def test_long_sequences_are_shared_out(Hq, Hkv, D, P, lens, asked, window):
    assert binding.mom_mx_attention_workspace_bytes(sum(asked), len(lens), Hq, Hkv, D, max(lens)) > 0
    _compare(_gen(14), Hq, Hkv, D, P, lens, asked, window)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 8, 64), (8, 8, 128), (8, 4, 256)])
def test_many_short_sequences(Hq, Hkv, D):
    """More tiles than 768: a workgroup has four wavefronts, with 256 dimensions eight."""
    B = 1100 // Hkv
    _compare(_gen(25), Hq, Hkv, D, 16, [1 + (7 * b) % 45 for b in range(B)], [1] * B)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (6, 1, 128), (4, 2, 256)])
def test_many_sequences_of_their_own_numbers_of_tokens(Hq, Hkv, D):
    """More than 64 sequences, some without tokens: tiles are counted over several rounds."""
    asked = [(5 * b) % 12 if b % 7 else 0 for b in range(150)]
    _compare(_gen(26), Hq, Hkv, D, 16, [a + (11 * b) % 60 for b, a in enumerate(asked)], asked)


def test_rows_that_see_nothing():
    gen = _gen(15)
    # no tokens at all; fewer in the cache than asked about (the first stand before the beginning); lengths that are none
    cache, table = _sequences(gen, 2, 128, 16, [0, 3, 20])
    for lens in ([0, 3, 20], [-5, 0, 1], [0, 0, 0]):
        out, lse = _compare(gen, 8, 2, 128, 16, lens, [2, 5, 1], cache_table=(cache, table), max_kv=20)
        assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all()
    out, lse = _compare(gen, 8, 2, 128, 16, [0, 0, 0], [2, 5, 1], cache_table=(cache, table), max_kv=0)
    assert (out == 0).all()


def test_lengths_above_the_table_and_above_max_kv():
    gen = _gen(16)
    cache, table = _sequences(gen, 1, 64, 16, [64, 48])
    _compare(gen, 4, 1, 64, 16, [1000, 48], [1, 2], cache_table=(cache, table), max_kv=5000)       # what the table holds counts
    _compare(gen, 4, 1, 64, 16, [64, 48], [1, 2], cache_table=(cache, table), max_kv=40)


def test_pages_that_are_none():
    gen = _gen(17)
    for bad in (-1, -2147483648, 2147483647, None):
        def broken(table, cache):
            table = table.clone()
            table[0, 1] = cache.shape[0] if bad is None else bad
            table[1, 0] = cache.shape[0] if bad is None else bad
            return table
        _compare(gen, 4, 2, 128, 16, [70, 16, 33], [2, 1, 40], table_of=broken)


def test_table_rows_that_lie_apart():
    gen = _gen(18)
    cache, table = _sequences(gen, 1, 64, 16, [64, 37])
    wide = torch.full((2, 9), -1, dtype=torch.int32)
    wide[:, :4] = table
    q, lens = _normal(gen, 2, 2, 64), torch.tensor([64, 37], dtype=torch.int32)
    out, lse = _attend(q.to(DEV), cache.to(DEV), 16, wide.to(DEV)[:, :4], lens.to(DEV), 64)
    want = ref.attention(q, cache, 16, table, lens, [0, 1, 2], 0.125)
    _within(out, want[0], want[2])
    _within(lse, want[1], want[3])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_is_not_seen_does_not_reach_a_row(D):
    """NaN keys and values of later tokens leave the earlier rows alone, and reach the rows that see them; beside shares and windows."""
    gen = _gen(19)
    for lens, asked, window in (([60], [40], 0), ([100], [100], 0), ([100], [90], 13), ([700], [3], 0), ([90, 64], [2, 5], 40)):
        cache, table = _sequences(gen, 1, D, 16, lens)
        k, v = _normal(gen, 1, 1, D).double(), _normal(gen, 1, 1, D).double()
        v[0, 0, 35] = math.nan                                    # a block of the dimensions
        slot = lambda b, t: torch.tensor([int(table[b, t // 16]) * 16 + t % 16])
        cache = ref.append(cache, 16, k, v, slot(0, lens[0] - 1))                       # the last token of all
        cache = ref.append(cache, 16, k, v, slot(0, max(0, lens[0] - asked[0] // 2 - 1)))
        out, _ = _compare(gen, 4, 1, D, 16, lens, asked, window, cache_table=(cache, table))
        assert torch.isnan(out[asked[0] - 1, :, 32:64]).all() and not torch.isnan(out[:, :, :32]).any()
        if asked[0] > 2:
            assert not torch.isnan(out[0]).any()
        k[0, 0, 1] = math.inf
        cache = ref.append(cache, 16, k, torch.zeros_like(v), slot(0, lens[0] - 1))
        _compare(gen, 4, 1, D, 16, lens, asked, window, cache_table=(cache, table))


def test_scores_of_every_size():
    gen = _gen(20)
    D, P, lens, asked = 128, 16, [300], [3]
    for std, scale in ((60.0, None), (1.0, 0.0), (1.0, -0.3), (1e-20, None), (8.0, 1.0)):
        cache, table = _sequences(gen, 1, D, P, lens)
        q = _normal(gen, 3, 4, D, std=std)
        _compare(gen, 4, 1, D, P, lens, asked, scale=scale, q=q, cache_table=(cache, table))
    # scores that rise all the way: the running maximum moves in every step
    n = 300
    k = torch.zeros(n, 1, D, dtype=torch.float64)
    k[:, 0, 0] = torch.arange(n).double()
    cache = ref.append(_noise(gen, 19, 1, P, D), P, k, torch.randn((n, 1, D), generator=gen).double(), torch.arange(n))
    table = torch.arange(19, dtype=torch.int32)[None]
    q = torch.zeros(1, 4, D, dtype=torch.bfloat16)
    q[0, :, 0] = torch.tensor([1.0, -1.0, 30.0, -30.0])
    _compare(gen, 4, 1, D, P, [n], [1], q=q, cache_table=(cache, table))


def test_tokens_of_no_sequence_are_left_alone_and_starts_are_kept_in_bounds():
    gen = _gen(21)
    cache, table = _sequences(gen, 1, 64, 16, [50, 20])
    q, lens = _normal(gen, 9, 2, 64), torch.tensor([50, 20], dtype=torch.int32)
    for starts in ([2, 5, 7], [2, 2, 6], [0, 9, 9]):
        out, lse = _attend(q.to(DEV), cache.to(DEV), 16, table.to(DEV), lens.to(DEV), 50, torch.tensor(starts, dtype=torch.int32).to(DEV))
        want = ref.attention(q, cache, 16, table, lens, starts, 0.125)
        _within(out[starts[0]:starts[-1]], want[0][starts[0]:starts[-1]], want[2][starts[0]:starts[-1]])
        outside = [i for i in range(9) if not starts[0] <= i < starts[-1]]
        assert (out[outside] == 3).all() and (lse[outside] == 3).all()


def test_without_lse_and_with_queries_of_a_projection():
    gen = _gen(22)
    cache, table = _sequences(gen, 2, 128, 32, [77])
    qkv, lens = _normal(gen, 3, 12, 128), torch.tensor([77], dtype=torch.int32)
    out, _ = _attend(qkv.to(DEV)[:, :8], cache.to(DEV), 32, table.to(DEV), lens.to(DEV), 77, with_lse=False)
    want = ref.attention(qkv[:, :8], cache, 32, table, lens, [0, 3], 128 ** -0.5)
    _within(out, want[0], want[2])


def test_pages_past_two_gigabytes():
    """A pool of over 4 GiB with the sequence on its last pages."""
    gen, P, D, Hkv, n = _gen(23), 256, 256, 32, 300
    block = ref.block_bytes(P, D)
    pages = ((1 << 32) + (1 << 26)) // (block * Hkv)
    small, table = _sequences(gen, Hkv, D, P, [n], extra=0)
    cache = torch.zeros((pages, Hkv, block), dtype=torch.uint8, device=DEV)
    cache[-2:] = small.to(DEV)
    q, lens = _normal(gen, 1, Hkv, D), torch.tensor([n], dtype=torch.int32)
    out, lse = _attend(q.to(DEV), cache, P, (table + pages - 2).to(DEV), lens.to(DEV), n)
    want = ref.attention(q, small, P, table, lens, [0, 1], 1 / 16)
    _within(out, want[0], want[2])
    k, v = _normal(gen, 2, Hkv, D), _normal(gen, 2, Hkv, D)
    slots = torch.tensor([pages * P - 1, pages * P - P - 2])
    binding.mom_mx_kv_append(k.to(DEV), v.to(DEV), slots.to(DEV), cache, P)
    ko, vo = torch.empty_like(k, device=DEV), torch.empty_like(v, device=DEV)
    binding.mom_mx_kv_read(cache, P, slots.to(DEV), ko, vo)
    assert torch.equal(ko.double().cpu(), ref.decode(*ref.encode(k.double()))) and torch.equal(vo.double().cpu(), ref.decode(*ref.encode(v.double())))


def test_the_same_bits_every_time():
    gen = _gen(24)
    cache, table = _sequences(gen, 1, 128, 16, [3000])
    q, lens = _normal(gen, 2, 4, 128).to(DEV), torch.tensor([3000], dtype=torch.int32).to(DEV)
    first = _attend(q, cache.to(DEV), 16, table.to(DEV), lens, 3000)
    for _ in range(5):
        again = _attend(q, cache.to(DEV), 16, table.to(DEV), lens, 3000)
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])


# Products

def _weight(gen, N, K, std=0.05):
    codes, scales = ref.encode(_normal(gen, N, K, std=std).double())
    return ref.pack(codes), scales.to(torch.uint8)


@pytest.mark.parametrize("N,K", [(1, 32), (16, 64), (17, 96), (33, 128), (50, 160), (300, 1056), (129, 2080), (64, 4096), (2049 * 16 + 5, 64), (40, 14336), (33, 32768), (32800, 2208), (20, 8224)])
@pytest.mark.parametrize("M", [1, 2, 5, 16])
def test_products(N, K, M):
    gen = _gen(30)
    x, w, w2, res = _normal(gen, M, K), _weight(gen, N, K), _weight(gen, N, K), _normal(gen, M, N)
    g, g2 = tuple(t.to(DEV) for t in w), tuple(t.to(DEV) for t in w2)
    want, err = ref.product(x, *w)
    out = torch.full((M, N), 3.0, device=DEV)
    binding.mom_mx_matvec(x.to(DEV), *g, out)
    _within(out, want, err)
    half = torch.full((M, N), 3.0, dtype=torch.bfloat16, device=DEV)
    binding.mom_mx_matvec(x.to(DEV), *g, half)
    _within(half, want, err + (want.abs() + err) * ref.BF16_HALF)
    binding.mom_mx_matvec(x.to(DEV), *g, half, residual=res.to(DEV))
    both = want + res.double()
    _within(half, both, err + 2 * ref.F32_HALF * both.abs() + (both.abs() + err) * ref.BF16_HALF)
    inplace = res.to(DEV)
    binding.mom_mx_matvec(x.to(DEV), *g, inplace, residual=inplace)
    assert torch.equal(inplace.view(torch.int16), half.view(torch.int16))
    up, up_err = ref.product(x, *w2)
    s = want * torch.sigmoid(want)
    y = s * up
    binding.mom_mx_gateup(x.to(DEV), *g, *g2, half)
    # silu rises by at most 1.1; its exponential and reciprocal are good to a few steps of fp32
    tol = 1.1 * err * (up.abs() + up_err) + s.abs() * up_err + y.abs() * 2.0 ** -20
    _within(half, y, tol + (y.abs() + tol) * ref.BF16_HALF)


def test_product_of_nan_and_infinities():
    gen = _gen(31)
    N, K = 40, 96
    x, (codes, scales) = _normal(gen, 2, K), _weight(gen, N, K)
    scales[3, 1] = 255
    out = torch.empty((2, N), device=DEV)
    binding.mom_mx_matvec(x.to(DEV), codes.to(DEV), scales.to(DEV), out)
    want, err = ref.product(x, codes, scales)
    _within(out, want, err)
    assert torch.isnan(out[:, 3]).all() and int(torch.isnan(out).sum()) == 2
    x[1, 5] = math.inf
    scales[3, 1] = 120
    codes[:, 2] = 0x22                                                # no zeros against the infinity
    binding.mom_mx_matvec(x.to(DEV), codes.to(DEV), scales.to(DEV), out)
    assert torch.isinf(out[1]).all() and torch.isfinite(out[0]).all()


@pytest.mark.parametrize("N,K", [(1, 32), (3, 96), (257, 1056), (64, 4096)])
def test_quantize(N, K):
    gen = _gen(32)
    w = _normal(gen, N, K, std=0.02)
    w[0, :4] = torch.tensor([0.0, -0.0, 7.0, math.nan if K > 32 else 1.0])
    codes, scales = torch.empty((N, K // 2), dtype=torch.uint8, device=DEV), torch.empty((N, K // 32), dtype=torch.uint8, device=DEV)
    binding.mom_mx_quantize(w.to(DEV), codes, scales)
    c, s = ref.encode(w.double())
    assert torch.equal(codes.cpu(), ref.pack(c)) and torch.equal(scales.cpu(), s.to(torch.uint8))


# Together

def test_steps_on_a_side_stream_and_in_a_graph():
    """Append and attend in a captured graph, replayed with new inputs between eager calls, and the same on another stream."""
    gen, Hq, Hkv, D, P, n = _gen(40), 8, 2, 128, 16, 600
    cache0, table = _sequences(gen, Hkv, D, P, [n])
    steps = [_normal(gen, 1, Hq + 2 * Hkv, D) for _ in range(4)]
    freq = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV)
    w = tuple(t.to(DEV) for t in _weight(gen, 64, Hq * D))

    def buffers():
        return {"cache": cache0.to(DEV), "table": table.to(DEV), "lens": torch.zeros(1, dtype=torch.int32, device=DEV), "slots": torch.zeros(1, dtype=torch.int64, device=DEV),
                "positions": torch.zeros(1, dtype=torch.int32, device=DEV), "qkv": torch.zeros(1, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device=DEV),
                "q": torch.empty(1, Hq, D, dtype=torch.bfloat16, device=DEV), "out": torch.empty(1, Hq, D, dtype=torch.bfloat16, device=DEV),
                "ws": torch.empty(binding.mom_mx_attention_workspace_bytes(1, 1, Hq, Hkv, D, n), dtype=torch.uint8, device=DEV), "y": torch.empty(1, 64, device=DEV)}

    def step(s):
        binding.mom_mx_kv_append(s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:], s["slots"], s["cache"], P, positions=s["positions"], inv_freq=freq, q=s["qkv"][:, :Hq], q_out=s["q"])
        binding.mom_mx_attention(s["q"], s["cache"], P, s["table"], s["lens"], n, s["out"], s["ws"])
        binding.mom_mx_matvec(s["out"].view(1, Hq * D), *w, s["y"])

    def feed(s, i):
        at = 500 + 7 * i
        s["qkv"].copy_(steps[i].to(DEV))
        s["lens"].fill_(at + 1)
        s["positions"].fill_(at)
        s["slots"].fill_(int(table[0, at // P]) * P + at % P)

    eager, graphed, sided = buffers(), buffers(), buffers()
    side = torch.cuda.Stream()
    step(graphed)                                  # loads the kernels
    graphed["cache"].copy_(cache0.to(DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    for i in range(4):
        for s in (eager, graphed, sided):
            feed(s, i)
        step(eager)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(sided)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for s in (graphed, sided):
            assert torch.equal(s["out"].view(torch.int16), eager["out"].view(torch.int16)) and torch.equal(s["y"], eager["y"]) and torch.equal(s["cache"], eager["cache"])
        want = ref.attention(eager["q"].cpu(), eager["cache"].cpu(), P, table, eager["lens"].cpu(), [0, 1], D ** -0.5)
        _within(eager["out"], want[0], want[2])
