"""Drafted tokens in a tree on the GPU, through the C ABI, against tests/draft_reference.py: at the sizes and masks where they can go wrong."""
import math
import random

import pytest
import torch

import draft_reference as dref
import mx_reference as ref
from paper_2504_12526_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen) * std).to(torch.bfloat16)


def _within(got, want, err, what=""):
    got, want = got.double().cpu(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, "NaN", int(torch.isnan(got).sum()), int(torch.isnan(want).sum()))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), (what, "infinities")
    fine = torch.isfinite(want)
    off = ((got - want).abs() - err)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), int((off > 0).sum()))


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype)


def _tree(rng, m, branch):
    return [-1 if i == 0 else rng.randrange(max(0, i - branch), i) for i in range(m)]


def _parents(rng, counts, branch, front=0, back=0):
    return [99] * front + [p for m in counts for p in _tree(rng, m, branch)] + [99] * back


def _starts(counts, front=0):
    s = [front]
    for m in counts:
        s.append(s[-1] + m)
    return s


# The tree's description

@pytest.mark.parametrize("counts,branch,words,P,front,back", [
    ([1], 1, 1, 16, 0, 0),
    ([16], 4, 1, 64, 0, 0),
    ([33], 3, 2, 16, 0, 0),
    ([5, 0, 64, 1, 31, 32], 4, 2, 16, 0, 0),
    ([7, 40, 3], 6, 1, 256, 2, 3),              # more rows than the words have bits, rows of no sequence at both ends
    ([200, 13], 9, 7, 32, 1, 0),
    ([512], 2, 16, 16, 0, 0),
    ([700], 5, 16, 128, 0, 1),                  # more rows than masks know
    ([3] * 130, 2, 1, 16, 0, 0),
])
def test_tree(counts, branch, words, P, front, back):
    rng = random.Random(1)
    T, B = front + sum(counts) + back, len(counts)
    parents = _ints(_parents(rng, counts, branch, front, back))
    lens = _ints([m + rng.randrange(0, 50) for m in counts])
    each = -(-(max(counts) + 50) // P)
    table = torch.randperm(B * each, generator=_gen(2)).to(torch.int32).view(B, each)
    table[0, 0] = -1
    starts = _ints(_starts(counts, front))
    masks, positions, slots = torch.full((T, words), 77, dtype=torch.int32), torch.full((T,), 77, dtype=torch.int32), torch.full((T,), 77, dtype=torch.int64)
    gm, gp, gs = masks.to(DEV), positions.to(DEV), slots.to(DEV)
    binding.mom_mx_tree(lens.to(DEV), parents=parents.to(DEV), q_starts=starts.to(DEV), masks=gm, positions=gp, slots=gs, page_table=table.to(DEV), page_tokens=P)
    want = dref.tree(parents, starts, T, lens, words, table, P)
    for i in range(T):
        assert [w & 0xffffffff for w in gm[i].tolist()] == (want[0][i] if want[0][i] is not None else [77] * words), i
    assert gp.tolist() == [77 if p is None else p for p in want[1]]
    assert gs.tolist() == [77 if s is None else s for s in want[2]]
    # one output alone
    alone = torch.full((T,), 77, dtype=torch.int32, device=DEV)
    binding.mom_mx_tree(lens.to(DEV), parents=parents.to(DEV), q_starts=starts.to(DEV), positions=alone)
    assert torch.equal(alone, gp)


def test_tree_of_chains_of_forests_and_of_parents_that_are_none():
    lens = _ints([40, 3, 12])
    masks, positions = torch.zeros((12, 1), dtype=torch.int32, device=DEV), torch.zeros(12, dtype=torch.int32, device=DEV)
    binding.mom_mx_tree(lens.to(DEV), masks=masks, positions=positions)
    want = dref.tree(None, [0, 4, 8, 12], 12, lens, 1)
    assert masks.flatten().tolist() == [w[0] for w in want[0]] == [1, 3, 7, 15] * 3 and positions.tolist() == want[1]
    assert positions.tolist()[4:8] == [-1, 0, 1, 2]                       # three tokens, four rows: the first is before the sequence
    # several roots, parents that come later, a row as its own, and what is no number of a row
    parents = _ints([5, -1, 0, 3, -1, 4, 4, 2 ** 31 - 1, -2 ** 31, 8, 9, 3])
    lens = _ints([50])
    binding.mom_mx_tree(lens.to(DEV), parents=parents.to(DEV), masks=masks, positions=positions)
    want = dref.tree(parents, [0, 12], 12, lens, 1)
    assert masks.flatten().tolist() == [w[0] for w in want[0]] and positions.tolist() == want[1]
    slots = torch.zeros(12, dtype=torch.int64, device=DEV)
    table = _ints([[4, 2, 7]])
    binding.mom_mx_tree(lens.to(DEV), slots=slots, page_table=table.to(DEV), page_tokens=16)       # 48 places for 50 tokens
    assert slots.tolist() == dref.tree(None, [0, 12], 12, lens, 1, table, 16)[2] and slots.tolist()[-2:] == [-1, -1]


# Attention

def _attend_case(counts, Hq, Hkv, D, P, lens, seed, front=0, back=0, strided=False):
    gen = _gen(seed)
    T, each = front + sum(counts) + back, max(1, max(-(-n // P) for n in lens))
    table = torch.randperm(len(counts) * each + 2, generator=gen).to(torch.int32)[:len(counts) * each].view(len(counts), each)
    pages = len(counts) * each + 2
    cache = torch.randint(0, 256, (pages, Hkv, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8)       # what was there before, NaN scales among it
    for b, n in enumerate(lens):
        slots = torch.tensor([int(table[b, j // P]) * P + j % P for j in range(n)])
        if n:
            cache = ref.append(cache, P, torch.randn(n, Hkv, D, generator=gen, dtype=torch.float64), torch.randn(n, Hkv, D, generator=gen, dtype=torch.float64), slots)
    q = _normal(gen, T, Hq + (3 if strided else 0), D)
    return q, cache, table, _ints(lens), _ints(_starts(counts, front))


def _masks(rng, counts, kind, words, front=0, back=0):
    rows = [[0x55555555] * words] * front
    for m in counts:
        tree = _tree(rng, m, 4)
        for i in range(m):
            if kind == "tree":
                bits = sum(1 << j for j in dref.climb(tree, 0, i))
            elif kind == "chain":
                bits = (2 << i) - 1
            else:
                bits = 0 if rng.random() < 0.2 else rng.getrandbits(32 * words)
            rows.append([(bits >> (32 * w)) & 0xffffffff for w in range(words)])
    rows += [[0x55555555] * words] * back
    return _ints([[w - (1 << 32) if w >> 31 else w for w in r] for r in rows]).view(-1, words)


def _attend(q, cache, P, table, lens, starts, masks, scale=None, window=0, max_kv=None, heads=None, **more):
    gq = q.to(DEV)
    q = q if heads is None else q[:, :heads]
    gq = gq if heads is None else gq[:, :heads]
    T, Hq, D = q.shape
    max_kv = table.shape[1] * P if max_kv is None else max_kv
    out, lse = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T, Hq), 7.0, device=DEV)
    need = binding.mom_mx_tree_attention_workspace_bytes(T, table.shape[0], Hq, cache.shape[1], D, max_kv)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=DEV) if need else None
    binding.mom_mx_tree_attention(gq, cache.to(DEV), P, table.to(DEV), lens.to(DEV), max_kv, masks.to(DEV), out, ws, q_starts=None if starts is None else starts.to(DEV),
                                  scale=scale, window=window, lse=lse, **more)
    return out, lse


def _check(q, cache, P, table, lens, starts, masks, scale=None, window=0, max_kv=None, heads=None):
    out, lse = _attend(q, cache, P, table, lens, starts, masks, scale, window, max_kv, heads)
    q = q if heads is None else q[:, :heads]
    T, _, D = q.shape
    most = 1 << 30 if max_kv is None else max_kv
    spans = starts.tolist() if starts is not None else [b * T // len(lens) for b in range(len(lens) + 1)]
    want, want_lse, err, lse_err = dref.attention(q, cache, P, table, lens, spans, masks, 1 / math.sqrt(D) if scale is None else scale, window, most)
    lo, hi = spans[0], spans[-1]
    _within(out[lo:hi], want[lo:hi], err[lo:hi], "out")
    _within(lse[lo:hi], want_lse[lo:hi], lse_err[lo:hi], "lse")
    for t in (out, lse):
        assert (t[:lo] == 7).all() and (t[hi:] == 7).all()
    return out, lse


@pytest.mark.parametrize("counts,Hq,Hkv,D,P,lens,kind,words,window", [
    ([1], 4, 1, 128, 16, [1], "tree", 1, 0),                             # one row that sees itself
    ([8], 8, 2, 128, 16, [77], "tree", 1, 0),
    ([16], 4, 4, 64, 64, [130], "tree", 1, 0),                           # a query head a key head
    ([5, 3, 8], 7, 1, 128, 16, [40, 3, 261], "tree", 1, 0),              # seven a key head; a sequence of rows alone
    ([33, 2], 2, 1, 256, 32, [33, 100], "tree", 2, 0),
    ([64], 4, 1, 128, 16, [200], "tree", 2, 0),                          # 256 rows
    ([70], 4, 1, 64, 16, [333], "tree", 3, 0),                           # more than 256: rows of their own
    ([70, 1], 4, 1, 128, 64, [90, 400], "tree", 3, 0),
    ([40], 8, 1, 256, 16, [170], "tree", 2, 0),
    ([9, 12], 4, 2, 128, 16, [70, 31], "random", 1, 0),                  # any masks, empty ones too
    ([70], 4, 1, 128, 16, [101], "random", 3, 0),
    ([12], 4, 1, 64, 16, [12], "random", 1, 0),                          # rows that see nothing
    ([50], 2, 1, 128, 16, [90], "tree", 1, 0),                           # rows past the mask's words are not seen
    ([8, 20], 4, 1, 128, 16, [100, 64], "tree", 1, 5),                   # windows shorter than some ways up the tree
    ([8, 20], 4, 1, 128, 16, [100, 64], "random", 1, 3),
    ([40], 8, 1, 64, 16, [300], "random", 2, 33),
    ([40], 2, 1, 256, 16, [300], "random", 2, 100),
    ([13], 4, 1, 128, 32, [70], "tree", 1, 1),
    ([6, 6], 3, 1, 128, 16, [4, 0], "tree", 1, 0),                       # more rows than tokens, and none
    ([6, 6], 3, 1, 128, 16, [4, 0], "tree", 1, 2),
    ([12], 4, 1, 128, 16, [3000], "tree", 1, 0),                         # cut into shares
    ([6], 4, 1, 256, 128, [2500], "random", 1, 0),
    ([80], 4, 1, 128, 16, [2100], "tree", 3, 0),
    ([20, 7], 4, 1, 64, 16, [1500, 2900], "tree", 1, 1200),
    ([256], 2, 1, 64, 16, [300], "tree", 8, 0),
])
def test_attention(counts, Hq, Hkv, D, P, lens, kind, words, window):
    q, cache, table, lens, starts = _attend_case(counts, Hq, Hkv, D, P, lens, 11)
    _check(q, cache, P, table, lens, starts, _masks(random.Random(3), counts, kind, words), window=window)


@pytest.mark.parametrize("counts,D", [([9, 4, 2], 128), ([70, 11], 64)])
def test_attention_with_rows_of_no_sequence_strided_queries_and_pages_that_are_none(counts, D):
    lens = [m + 60 for m in counts]
    q, cache, table, lens, starts = _attend_case(counts, 4, 1, D, 16, lens, 12, front=3, back=2, strided=True)
    table[0, 1], table[1, 2] = -1, cache.shape[0]
    masks = _masks(random.Random(4), counts, "tree", 3, 3, 2)
    _check(q, cache, 16, table, lens, starts, masks, heads=4)
    _check(q, cache, 16, table, lens, starts, masks, heads=4, window=20, scale=-0.3)
    _check(q, cache, 16, table, lens, starts, masks, heads=4, max_kv=70, scale=0.0)


@pytest.mark.parametrize("kv,Hkv", [(1700, 1), (1700, 8), (300, 4)])
def test_attention_of_more_sequences_than_a_wavefront_has_lanes(kv, Hkv):
    """Most of them short, some without rows, a few long and in shares."""
    rng = random.Random(7)
    counts = [rng.choice([0, 1, 3]) for _ in range(150)]
    lens = [m + rng.randrange(0, 20) for m in counts]
    for b in (0, 63, 64, 149):
        counts[b], lens[b] = 5, kv - b
    q, cache, table, lens, starts = _attend_case(counts, Hkv, Hkv, 64, 16, lens, 16)
    _check(q, cache, 16, table, lens, starts, _masks(rng, counts, "tree", 1))


def test_nan_in_shares():
    rng, D, P, n, m = random.Random(8), 64, 16, 2600, 7
    q, cache, table, lens, starts = _attend_case([m], 2, 1, D, P, [n], 17)
    bad = torch.ones(1, 1, D, dtype=torch.float64)
    bad[:, :, 32:] = math.nan
    for j in (n - m + 2, 700):
        slot = int(table[0, j // P]) * P + j % P
        cache = ref.append(cache, P, torch.ones(1, 1, D, dtype=torch.float64), bad, torch.tensor([slot]))
        out, _ = _check(q, cache, P, table, lens, starts, _masks(rng, [m], "tree", 1))
        assert out[:, :, 32:].isnan().any() and not out[:, :, :32].isnan().any()


@pytest.mark.parametrize("m", [6, 72])
def test_attention_of_sequences_with_as_many_rows_each(m):
    q, cache, table, lens, _ = _attend_case([m] * 3, 4, 1, 128, 16, [m, m + 40, m + 17], 13)
    _check(q, cache, 16, table, lens, None, _masks(random.Random(5), [m] * 3, "tree", 3))


@pytest.mark.parametrize("m", [5, 70])
def test_what_a_row_does_not_see_does_not_reach_it(m):
    """NaN in rows and in tokens before a window: they are NaN for those that see them alone."""
    rng, D, P, n = random.Random(6), 128, 16, m + 40
    q, cache, table, lens, starts = _attend_case([m], 4, 1, D, P, [n], 14)
    bad = torch.full((2, 1, D), math.nan, dtype=torch.float64)
    bad[:, :, 32:] = 1.0
    for j in (n - m + 1, n - m + 3):
        slot = int(table[0, j // P]) * P + j % P
        cache = ref.append(cache, P, torch.ones(1, 1, D, dtype=torch.float64), bad[:1], torch.tensor([slot]))
    masks = _masks(rng, [m], "tree", 3)
    out, _ = _check(q, cache, P, table, lens, starts, masks)
    sees = [bool(int(w[0]) & 0b1010) for w in masks]
    assert any(sees) and not all(sees)
    assert [bool(r) for r in out[:, 0, 0].isnan().tolist()] == sees and not out[:, :, 32:].isnan().any()
    _check(q, cache, P, table, lens, starts, masks, window=2)
    # keys
    slot = int(table[0, (n - m + 2) // P]) * P + (n - m + 2) % P
    cache = ref.append(cache, P, torch.full((1, 1, D), math.nan, dtype=torch.float64), torch.ones(1, 1, D, dtype=torch.float64), torch.tensor([slot]))
    _check(q, cache, P, table, lens, starts, masks)


@pytest.mark.parametrize("counts,lens", [([1, 1], [50, 900]), ([7, 7], [50, 900]), ([90], [500])])
def test_chains_are_those_of_the_other_call(counts, lens):
    q, cache, table, lens, starts = _attend_case(counts, 8, 2, 128, 16, lens, 15)
    out, _ = _check(q, cache, 16, table, lens, starts, _masks(random.Random(0), counts, "chain", 3))
    other = torch.empty_like(out)
    ws = torch.empty(max(1, binding.mom_mx_attention_workspace_bytes(sum(counts), len(counts), 8, 2, 128, table.shape[1] * 16)), dtype=torch.uint8, device=DEV)
    binding.mom_mx_attention(q.to(DEV), cache.to(DEV), 16, table.to(DEV), lens.to(DEV), table.shape[1] * 16, other, ws, q_starts=starts.to(DEV))
    # two results, each off by at most what the weights' rounding and its own allow
    want, _, err, _ = dref.attention(q, cache, 16, table, lens, starts.tolist(), _masks(random.Random(0), counts, "chain", 3), 1 / math.sqrt(128))
    _within(other, want, err)


def test_attention_and_slots_by_a_table_whose_rows_lie_apart():
    counts, lens, P, D = [6, 40, 3], [100, 90, 33], 16, 64
    q, cache, table, lens, starts = _attend_case(counts, 2, 1, D, P, lens, 18)
    masks = _masks(random.Random(9), counts, "tree", 2)
    wide = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    apart = wide.to(DEV)[:, :table.shape[1]]
    out, other = (torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    args = dict(q_starts=starts.to(DEV))
    for t, o in ((apart, out), (table.to(DEV), other)):
        binding.mom_mx_tree_attention(q.to(DEV), cache.to(DEV), P, t, lens.to(DEV), 112, masks.to(DEV), o, None, **args)
    assert torch.equal(out.view(torch.int16), other.view(torch.int16)) and not (out == 7).all()
    slots = [torch.empty(49, dtype=torch.int64, device=DEV) for _ in range(2)]
    for t, o in ((apart, slots[0]), (table.to(DEV), slots[1])):
        binding.mom_mx_tree(lens.to(DEV), slots=o, page_table=t, page_tokens=P, **args)
    assert torch.equal(*slots) and slots[0].min() >= 0


# Verification

def _logits(gen, T, V, bf16, draft, spread=2.0):
    target = torch.randn((T, V), generator=gen) * spread
    other = target + torch.randn((T, V), generator=gen) * 0.8 if draft else None
    dtype = torch.bfloat16 if bf16 else torch.float32
    return target.to(dtype), None if other is None else other.to(dtype)


def _draws(gen, parents, starts, draft, target, T, V, t):
    """A token for every row, drawn from what its parent says."""
    tokens = torch.zeros(T, dtype=torch.int32)
    for b, (lo, hi) in enumerate(dref.spans(starts, T)):
        for i in range(1, hi - lo):
            up = dref.above(parents, lo, i)
            p = torch.from_numpy(dref.chances((draft if draft is not None else target)[lo + max(up, 0)], t[b] if t[b] > 0 else 0.3))
            tokens[lo + i] = int(torch.multinomial(p, 1, generator=gen)) if p.sum() > 0 else 0
    return tokens


def _verify(target, tokens, uniforms, B, draft=None, parents=None, max_children=1, starts=None, temperatures=None):
    T, V = target.shape
    rows, out = (torch.full((T,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    counts = torch.full((B,), 77, dtype=torch.int32, device=DEV)
    ws = torch.randint(0, 256, (binding.mom_verify_drafts_workspace_bytes(T, B, V),), dtype=torch.uint8, device=DEV)
    g = [None if t is None else t.to(DEV) for t in (tokens, uniforms, draft, parents, starts, temperatures)]
    if draft is not None and not draft.is_contiguous():
        g[2] = torch.zeros((T, draft.stride(0)), dtype=draft.dtype, device=DEV)[:, :V].copy_(draft)
    gt = target.to(DEV)
    if not target.is_contiguous():
        gt = torch.zeros((T, target.stride(0)), dtype=target.dtype, device=DEV)[:, :V].copy_(target)
    binding.mom_verify_drafts(gt, g[0], g[1], rows, out, counts, ws, draft=g[2], parents=g[3], max_children=max_children, q_starts=g[4], temperatures=g[5])
    return rows.tolist(), out.tolist(), counts.tolist()


def _same(got, want):
    fill = lambda x: [77 if v is None else v for v in x]
    assert got[2] == want[2]
    assert got[0] == fill(want[0]) and got[1] == fill(want[1])


@pytest.mark.parametrize("V", [1, 2, 5, 31, 1000, 4095, 4096, 4097, 12289, 32001])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("bf16", [False, True])
def test_verify(V, draft, bf16):
    gen, rng = _gen(V + 2 * draft + bf16), random.Random(V)
    counts = [5, 1, 9, 0, 17, 2, 33]
    front, back = 1, 2
    T, B = front + sum(counts) + back, len(counts)
    starts = _ints(_starts(counts, front))
    parents = _ints(_parents(rng, counts, 3, front, back))
    temperatures = torch.tensor([1.0, 0.7, 1.4, 1.0, 0.9, 0.0, 1.0])
    target, other = _logits(gen, T, V, bf16, draft)
    tokens = _draws(gen, parents, starts, other, target, T, V, temperatures.tolist())
    uniforms = torch.rand(T, generator=gen)
    for children in (1, 2, 9):
        got = _verify(target, tokens, uniforms, B, other, parents, children, starts, temperatures)
        _same(got, dref.verify(target, other, tokens, parents, children, starts, temperatures, uniforms))


@pytest.mark.parametrize("B,m,V", [(1, 5, 70001), (70, 3, 777), (3, 100, 513), (1, 1, 300000), (2, 520, 50)])
@pytest.mark.parametrize("draft", [True, False])
def test_verify_chains(B, m, V, draft):
    gen = _gen(B * m)
    T = B * m
    target, other = _logits(gen, T, V, False, draft, spread=1.0 if m < 50 else 0.01)
    if m > 50 and draft:
        other = target + torch.randn(T, V, generator=gen) * 1e-3          # long ways down
    starts = [b * m for b in range(B + 1)]
    tokens = _draws(gen, None, starts, other, target, T, V, [1.0] * B)
    uniforms = torch.rand(T, generator=gen)
    # rows longer than the vocabulary, at any element
    pad = torch.zeros(T, V + 3)
    pad[:, :V] = target
    got = _verify(pad[:, :V], tokens, uniforms, B, other)
    want = dref.verify(target, other, tokens, None, 1, starts, None, uniforms)
    if m > binding.MOM_MAX_DRAFT_ROWS:
        assert max(want[2]) == binding.MOM_MAX_DRAFT_ROWS or not draft   # the way down ends where the rows are not known any more
    _same(got, want)


def test_verify_of_more_sequences_than_a_wavefront_has_lanes():
    gen, rng, V = _gen(18), random.Random(18), 300
    counts = [rng.choice([0, 1, 2, 6]) for _ in range(200)]
    T, B, starts = 3 + sum(counts) + 1, len(counts), _ints(_starts(counts, 3))
    parents = _ints(_parents(rng, counts, 2, 3, 1))
    for draft in (True, False):
        target, other = _logits(gen, T, V, False, draft)
        t = torch.tensor([0.0 if b % 7 == 3 else 0.5 + b / B for b in range(B)])
        tokens = _draws(gen, parents, starts, other, target, T, V, t.tolist())
        uniforms = torch.rand(T, generator=gen)
        _same(_verify(target, tokens, uniforms, B, other, parents, 3, starts, t), dref.verify(target, other, tokens, parents, 3, starts, t, uniforms))


def test_verify_of_logits_far_from_the_first():
    """Sums are relative to a row's first logit: far above it, far below it, infinite, and large ones whose products are rounded."""
    gen, V, B = _gen(19), 9001, 8
    target, other = _logits(gen, 2 * B, V, False, True)
    for x in (target, other):
        x[0:2, 0] = 2000.0
        x[2:4, 0] = -2000.0
        x[4:6, 0] = -math.inf
        x[6:8] *= 1e6
        x[8:10, 4096:] = -math.inf
        x[10:12] += 5e4
        x[12:14, 0], x[12:14, 5000] = math.nan, math.inf
        x[14:16, :8999] = -math.inf
    tokens, uniforms = torch.randint(0, V, (2 * B,), generator=gen).to(torch.int32), torch.rand(2 * B, generator=gen)
    tokens[1], tokens[7], tokens[13], tokens[15] = 0, int(target[6].argmax()), 5000, 9000
    for t in (None, torch.full((B,), 0.01), torch.full((B,), 300.0), torch.full((B,), math.inf)):
        for draft in (other, None):
            _same(_verify(target, tokens, uniforms, B, draft, None, 1, None, t), dref.verify(target, draft, tokens, None, 1, [2 * b for b in range(B + 1)], t, uniforms))


@pytest.mark.parametrize("bf16", [False, True])
def test_verify_of_trees_of_as_many_rows_whose_logits_lie_apart(bf16):
    gen, rng, V, B, m = _gen(21), random.Random(21), 9999, 5, 11
    T = B * m
    parents = _ints(_parents(rng, [m] * B, 3))
    target, other = _logits(gen, T, V, bf16, True)
    wide = [torch.zeros((T, V + k), dtype=t.dtype) for t, k in ((target, 7), (other, 1))]
    for w, t in zip(wide, (target, other)):
        w[:, :V] = t
    starts = [b * m for b in range(B + 1)]
    tokens, uniforms = _draws(gen, parents, starts, other, target, T, V, [1.0] * B), torch.rand(T, generator=gen)
    got = _verify(wide[0][:, :V], tokens, uniforms, B, wide[1][:, :V], parents, 3)
    _same(got, dref.verify(target, other, tokens, parents, 3, starts, None, uniforms))


def test_verify_of_a_star_with_many_children():
    gen, V, m = _gen(8), 600, 130
    parents = _ints([-1] + [0] * (m - 1))
    for draft in (False, True):
        target, other = _logits(gen, m, V, False, draft, spread=0.5)
        uniforms = torch.rand(m, generator=gen)
        tokens = _draws(gen, parents, [0, m], other, target, m, V, [1.0])
        for children in (1, 7, 129):
            # numbers that refuse most of them
            u = uniforms.clone()
            u[1:100] = 0.9999 if draft else 0.5
            _same(_verify(target, tokens, u, 1, other, parents, children), dref.verify(target, other, tokens, parents, children, [0, m], None, u))


def test_verify_at_the_edges():
    V, inf, nan = 9, math.inf, math.nan
    base = torch.tensor([0.5, 1.0, -1.0, 2.0, 0.0, 0.25, 2.0, -3.0, 1.5])
    target = base.repeat(24, 1)
    draft = target + torch.linspace(-0.5, 0.5, V)
    parents = _ints([-1, 0, 0] * 8)
    starts = _ints(range(0, 25, 3))
    tokens = _ints([0, 3, 3, 0, -1, 6, 0, V, 6, 0, 1, 2, 0, 1, 2, 0, 1, 2, 0, 3, 6, 0, 6, 3])
    uniforms = torch.tensor([0.3, 0.9, 0.9, 0.0, 0.0, 0.99, 1.0, 0.0, 0.0, 0.7, 0.4, 0.2, 2.0, 0.9, 0.9, nan, 0.9, 0.9, -1.0, 0.9, 0.9, 0.5, 0.999, 0.1])
    temperatures = torch.tensor([1.0, 1.0, 1.0, inf, 1.0, 1.0, 1.0, 1e-30])
    # logits that are infinite or none
    target[9, 2], target[10, 0], target[12, 4], target[15] = -inf, inf, nan, -inf
    target[16, 3], draft[18] = inf, -inf
    draft[21, 0] = inf
    for other in (draft, None):
        for temps in (temperatures, torch.tensor([0.0, -1.0, nan, 0.0, 0.0, 0.0, 0.0, 0.0]), None):
            _same(_verify(target, tokens, uniforms, 8, other, parents, 2, starts, temps), dref.verify(target, other, tokens, parents, 2, starts, temps, uniforms))


def test_verify_leaves_the_targets_probabilities():
    """What comes out is distributed as the target says, whatever the drafts: the first token over 60000 sequences, and the second where a first was taken."""
    gen, V, B = _gen(9), 6, 60000
    p, q = torch.randn(3, V, generator=gen) * 1.5, torch.randn(3, V, generator=gen) * 1.5
    parents = _ints([-1, 0, 0] * B)
    for draft in (True, False):
        target, other = p.repeat(B, 1), q.repeat(B, 1) if draft else None
        chance = torch.softmax(q[0].double(), 0)
        tokens = torch.multinomial(chance, 3 * B, replacement=True, generator=gen).to(torch.int32)
        if not draft:
            tokens[1::3], tokens[2::3] = 4, 1                             # looked up, not drawn
        uniforms = torch.rand(3 * B, generator=gen)
        _, out, counts = _verify(target, tokens, uniforms, B, other, parents, 2, _ints(range(0, 3 * B + 1, 3)))
        first = torch.tensor(out[0::3])
        want = torch.softmax(p[0].double(), 0)
        got = torch.bincount(first, minlength=V).double() / B
        # a frequency of B draws is off by sqrt(p (1 - p) / B); five of that six times over is one in some 300000
        assert ((got - want).abs() <= 5 * (want * (1 - want) / B).sqrt()).all(), (got, want)
        for row in (1, 2):
            here = torch.tensor([o for o, c, r in zip(out[1::3], counts, _second_rows(out, tokens.tolist(), counts)) if c == 2 and r == row])
            if len(here) < 100:
                continue
            want2 = torch.softmax(p[row].double(), 0)
            got2 = torch.bincount(here, minlength=V).double() / len(here)
            assert ((got2 - want2).abs() <= 5 * (want2 * (1 - want2) / len(here)).sqrt()).all(), (row, got2, want2)


def _second_rows(out, tokens, counts):
    """Which row a sequence of three went to (the first whose token it is)."""
    return [1 if out[3 * b] == tokens[3 * b + 1] else 2 for b in range(len(counts))]


# Keeping rows

@pytest.mark.parametrize("counts,Hkv,D,P,front,back", [
    ([8], 8, 128, 16, 0, 0),
    ([5, 1, 16, 0, 33], 2, 64, 16, 1, 2),
    ([64, 3], 3, 256, 32, 0, 0),
    ([150], 1, 128, 64, 0, 0),
    ([7] * 20, 4, 128, 256, 0, 0),
])
def test_keep(counts, Hkv, D, P, front, back):
    rng, gen = random.Random(10), _gen(10)
    T, B = front + sum(counts) + back, len(counts)
    lens = [m + rng.randrange(0, 40) for m in counts]
    lens[0] = counts[0]                                                   # rows from the sequence's beginning on
    each = -(-max(lens) // P)
    table = torch.randperm(B * each + 1, generator=gen).to(torch.int32)[:B * each].view(B, each)
    cache = torch.randint(0, 256, (B * each + 1, Hkv, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8)
    rows, kept = [55] * front, []
    for m in counts:
        path = [0] + sorted(rng.sample(range(1, m), rng.randrange(0, m))) if m else []
        rows += path + [-1] * (m - len(path))
        kept.append(len(path))
    rows = _ints(rows + [55] * back)
    starts, kept, lens = _ints(_starts(counts, front)), _ints(kept), _ints(lens)

    def check(table, kept, rows, cache=cache):
        gc, new = cache.to(DEV), torch.full((B,), 77, dtype=torch.int32, device=DEV)
        binding.mom_mx_kv_keep(gc, P, D, table.to(DEV), lens.to(DEV), rows.to(DEV), kept.to(DEV), new, q_starts=starts.to(DEV))
        want, want_lens = dref.keep(cache, P, D, table, lens, starts, rows, kept)
        assert torch.equal(gc.cpu(), want) and new.tolist() == want_lens
        return gc

    got = check(table, kept, rows)
    assert B == 1 or not torch.equal(got.cpu(), cache)
    check(table, torch.zeros_like(kept), rows)
    # pages that are none of the cache's, counts that are too high, all rows or none
    none = table.clone()
    none[0, -1], none[-1, 0] = -1, cache.shape[0]
    check(none, kept, rows)
    check(table, kept + 1000, rows)
    check(table, kept - 1000, rows)


def test_keep_of_sequences_with_as_many_rows_each_and_of_a_table_whose_rows_lie_apart():
    gen, P, D, B, m = _gen(11), 16, 64, 3, 6
    wide = torch.randperm(12, generator=gen).to(torch.int32).view(3, 4)
    table = wide[:, :2]
    cache = torch.randint(0, 256, (12, 2, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8)
    rows, kept, lens = _ints([0, 2, 5, -1, -1, -1] * 3), _ints([3, 2, 1]), _ints([30, 33, 36])       # the last two have more tokens than places
    gc, new = cache.to(DEV), torch.empty(B, dtype=torch.int32, device=DEV)
    binding.mom_mx_kv_keep(gc, P, D, wide.to(DEV)[:, :2], lens.to(DEV), rows.to(DEV), kept.to(DEV), new)
    want, want_lens = dref.keep(cache, P, D, table, lens, [0, 6, 12, 18], rows, kept)
    assert torch.equal(gc.cpu(), want) and new.tolist() == want_lens == [27, 29, 31]


# Together

def _step(st):
    """One step with drafts: everything on the current stream."""
    binding.mom_mx_tree(st["lens"], parents=st["parents"], q_starts=st["starts"], masks=st["masks"], positions=st["positions"], slots=st["slots"],
                        page_table=st["table"], page_tokens=st["P"])
    binding.mom_mx_kv_append(st["k"], st["v"], st["slots"], st["cache"], st["P"], positions=st["positions"], inv_freq=st["inv_freq"], q=st["q"], q_out=st["rotated"])
    binding.mom_mx_tree_attention(st["rotated"], st["cache"], st["P"], st["table"], st["lens"], st["most"], st["masks"], st["out"], st["ws"], q_starts=st["starts"])
    binding.mom_verify_drafts(st["target"], st["tokens"], st["uniforms"], st["rows"], st["next"], st["counts"], st["vws"], draft=st["draft"], parents=st["parents"],
                              max_children=3, q_starts=st["starts"])
    binding.mom_mx_kv_keep(st["cache"], st["P"], 128, st["table"], st["lens"], st["rows"], st["counts"], st["new_lens"], q_starts=st["starts"])


def _step_state(seed, counts=(9, 6, 14), lens=(300, 41, 1200), V=5000, P=16, Hq=8, Hkv=2, D=128):
    rng, gen = random.Random(seed), _gen(seed)
    T, B = sum(counts), len(counts)
    q, cache, table, lens, starts = _attend_case(list(counts), Hq, Hkv, D, P, list(lens), seed)
    parents = _ints(_parents(rng, counts, 3))
    target, draft = _logits(gen, T, V, False, True)
    st = {"P": P, "most": table.shape[1] * P, "lens": lens, "parents": parents, "starts": starts, "table": table, "cache": cache, "q": q, "k": _normal(gen, T, Hkv, D),
          "v": _normal(gen, T, Hkv, D), "inv_freq": (500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float(), "target": target, "draft": draft,
          "tokens": _draws(gen, parents, starts, draft, target, T, V, [1.0] * B), "uniforms": torch.rand(T, generator=gen)}
    st = {k: v.to(DEV) if torch.is_tensor(v) else v for k, v in st.items()}
    i32 = dict(dtype=torch.int32, device=DEV)
    st |= {"masks": torch.zeros((T, 1), **i32), "positions": torch.zeros(T, **i32), "slots": torch.zeros(T, dtype=torch.int64, device=DEV), "rotated": torch.zeros_like(st["q"]),
           "out": torch.zeros_like(st["q"]), "rows": torch.zeros(T, **i32), "next": torch.zeros(T, **i32), "counts": torch.zeros(B, **i32), "new_lens": torch.zeros(B, **i32),
           "ws": torch.empty(binding.mom_mx_tree_attention_workspace_bytes(T, B, Hq, Hkv, D, st["most"]), dtype=torch.uint8, device=DEV),
           "vws": torch.empty(binding.mom_verify_drafts_workspace_bytes(T, B, V), dtype=torch.uint8, device=DEV)}
    return st


def test_a_step_with_drafts_is_the_decoding_of_what_it_kept():
    """The last row that stays attends in the tree as it does as the last token of a sequence that the kept rows were appended to one by one."""
    st = _step_state(20)
    before = st["cache"].clone()
    _step(st)
    want = dref.verify(st["target"].cpu(), st["draft"].cpu(), st["tokens"].cpu(), st["parents"].cpu(), 3, st["starts"].cpu(), None, st["uniforms"].cpu())
    assert st["rows"].tolist() == want[0] and st["next"].tolist() == want[1] and st["counts"].tolist() == want[2] and max(want[2]) > 2
    starts = st["starts"].tolist()
    T = st["q"].shape[0]
    last = [starts[b] + want[0][starts[b] + c - 1] for b, c in enumerate(want[2])]
    kept = [starts[b] + want[0][starts[b] + i] for b, c in enumerate(want[2]) for i in range(c)]
    base = [int(n) - (starts[b + 1] - starts[b]) for b, n in enumerate(st["lens"].tolist())]
    places = [base[b] + i for b, c in enumerate(want[2]) for i in range(c)]
    seqs = [b for b, c in enumerate(want[2]) for _ in range(c)]
    slots = torch.tensor([int(st["table"][b, j // st["P"]]) * st["P"] + j % st["P"] for b, j in zip(seqs, places)], device=DEV)
    line = before.clone()
    at = torch.tensor(kept, device=DEV)
    rotated = torch.empty((len(kept),) + st["q"].shape[1:], dtype=torch.bfloat16, device=DEV)
    binding.mom_mx_kv_append(st["k"][at].contiguous(), st["v"][at].contiguous(), slots, line, st["P"], positions=torch.tensor(places, dtype=torch.int32, device=DEV),
                             inv_freq=st["inv_freq"], q=st["q"][at].contiguous(), q_out=rotated)
    assert st["new_lens"].tolist() == [base[b] + c for b, c in enumerate(want[2])]
    for b, c in enumerate(want[2]):
        for j in range(base[b] + c):
            page, t = int(st["table"][b, j // st["P"]]), j % st["P"]
            for x, y in zip(ref.get(st["cache"].cpu(), st["P"], 128, page, t), ref.get(line.cpu(), st["P"], 128, page, t)):
                assert torch.equal(x, y), (b, j)
    ends = torch.tensor([sum(want[2][:b + 1]) - 1 for b in range(len(want[2]))], device=DEV)
    out, lens = torch.empty((len(ends),) + st["q"].shape[1:], dtype=torch.bfloat16, device=DEV), st["new_lens"]
    ws = torch.empty(max(1, binding.mom_mx_attention_workspace_bytes(len(ends), len(ends), 8, 2, 128, st["most"])), dtype=torch.uint8, device=DEV)
    one = rotated[ends].contiguous()
    binding.mom_mx_attention(one, st["cache"], st["P"], st["table"], lens, st["most"], out, ws)
    want_out, _, err, _ = ref.attention(one.cpu(), st["cache"].cpu(), st["P"], st["table"].cpu(), lens.cpu(), list(range(len(ends) + 1)), 1 / math.sqrt(128))
    _within(out, want_out, err)
    _within(st["out"][torch.tensor(last, device=DEV)], want_out, err)
    assert T == st["rotated"].shape[0]


def test_captured_steps_that_share_their_workspaces():
    """Two graphs over the same workspaces, replayed in turn with eager work between them; each replay is the eager result."""
    states = [_step_state(30), _step_state(31, counts=(5, 12), lens=(700, 90), V=9001)]
    for name in ("ws", "vws"):
        big = max((st[name] for st in states), key=lambda t: t.numel())
        for st in states:
            st[name] = big
    outs = ("masks", "positions", "slots", "rotated", "out", "rows", "next", "counts", "new_lens", "cache")
    caches, wants = [st["cache"].clone() for st in states], []
    for st in states:
        _step(st)
        wants.append({k: st[k].clone() for k in outs})
    graphs = []
    side = torch.cuda.Stream()
    for st, c in zip(states, caches):
        st["cache"].copy_(c)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            _step(st)
        graphs.append(g)
    for turn in range(3):
        for st, c, g, want in zip(states, caches, graphs, wants):
            st["cache"].copy_(c)
            for k in outs[:-1]:
                st[k].zero_()
            st["ws"].fill_(255)
            st["vws"].fill_(255)
            g.replay()
            torch.cuda.synchronize()
            for k in outs:
                assert torch.equal(st[k].view(torch.int16) if st[k].dtype == torch.bfloat16 else st[k], want[k].view(torch.int16) if want[k].dtype == torch.bfloat16 else want[k]), (turn, k)


def test_two_streams_at_once():
    states = [_step_state(40 + i) for i in range(2)]
    wants = []
    for st in states:
        c = st["cache"].clone()
        _step(st)
        wants.append({k: st[k].clone() for k in ("out", "next", "cache")})
        st["cache"].copy_(c)
        st["out"].zero_()
        st["next"].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for st, s in zip(states, streams):
        with torch.cuda.stream(s):
            _step(st)
    torch.cuda.synchronize()
    for st, want in zip(states, wants):
        for k, w in want.items():
            assert torch.equal(st[k].view(torch.uint8), w.view(torch.uint8)), k
