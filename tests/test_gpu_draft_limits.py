"""Drafted tokens on the GPU where a call's inputs are not what they should be, or as large as they may be."""
import random

import pytest
import torch

import draft_reference as dref
import mx_reference as ref
from paper_2504_12526_amd import binding
from test_gpu_draft import DEV, _gen, _ints, _logits, _normal, _same, _tree, _verify

pytestmark = pytest.mark.gpu
GUARD = 1 << 20


def _guarded(nbytes):
    """A workspace and what lies behind it, which has to stay as it is."""
    whole = torch.full((nbytes + GUARD,), 0x5a, dtype=torch.uint8, device=DEV)
    return whole[:nbytes], whole[nbytes:]


@pytest.mark.parametrize("starts", [[0, 512, 100, 600, 50, 300, 10], [600, 0, 600, 0, 600, 0, 600], [-7, 40, 20, 2 ** 31 - 1, -2 ** 31, 599, 30]])
def test_starts_that_do_not_ascend_reach_nothing_out_of_range(starts):
    gen, rng, T, V, B, P, D = _gen(51), random.Random(51), 600, 20001, 6, 16, 64
    target, draft = (t.to(DEV) for t in _logits(gen, T, V, False, True))
    i32 = dict(dtype=torch.int32, device=DEV)
    parents, tokens = _ints(_tree(rng, T, 9)).to(DEV), torch.randint(0, V, (T,), generator=gen).to(DEV, torch.int32)
    uniforms, gs = torch.rand(T, generator=gen).to(DEV), _ints(starts).to(DEV)
    lens, table = _ints([600, 700, 650, 900, 600, 610]).to(DEV), torch.randperm(6 * 57, generator=gen).to(DEV, torch.int32).view(6, 57)
    cache = torch.randint(0, 256, (6 * 57 + 9, 1, ref.block_bytes(P, D)), generator=gen, dtype=torch.uint8).to(DEV)
    masks, positions, slots = torch.zeros((T, 16), **i32), torch.zeros(T, **i32), torch.zeros(T, dtype=torch.int64, device=DEV)
    binding.mom_mx_tree(lens, parents=parents, q_starts=gs, masks=masks, positions=positions, slots=slots, page_table=table, page_tokens=P)
    assert slots.max() < 6 * 57 * P
    q = _normal(gen, T, 4, D).to(DEV)
    out = torch.zeros_like(q)
    ws, behind = _guarded(binding.mom_mx_tree_attention_workspace_bytes(T, B, 4, 1, D, 57 * P))
    binding.mom_mx_tree_attention(q, cache, P, table, lens, 57 * P, masks, out, ws if ws.numel() else None, q_starts=gs)
    torch.cuda.synchronize()
    assert (behind == 0x5a).all()
    rows, next_tokens, counts, new_lens = torch.zeros(T, **i32), torch.zeros(T, **i32), torch.zeros(B, **i32), torch.zeros(B, **i32)
    ws, behind = _guarded(binding.mom_verify_drafts_workspace_bytes(T, B, V))
    for model in (draft, None):
        binding.mom_verify_drafts(target, tokens, uniforms, rows, next_tokens, counts, ws, draft=model, parents=parents, max_children=3, q_starts=gs)
        torch.cuda.synchronize()
        assert (behind == 0x5a).all() and counts.min() >= 0 and counts.max() <= binding.MOM_MAX_DRAFT_ROWS
    before = cache[6 * 57:].clone()
    binding.mom_mx_kv_keep(cache, P, D, table, lens, rows, counts, new_lens, q_starts=gs)
    assert torch.equal(cache[6 * 57:], before)
    # and the next call is right
    small, other = target[:40, :3000].cpu(), draft[:40, :3000].cpu()
    t, p, u = (tokens[:40] % 3000).cpu(), _ints(_tree(rng, 40, 5)), uniforms[:40].cpu()
    _same(_verify(small.contiguous(), t, u, 1, other.contiguous(), p, 3), dref.verify(small, other, t, p, 3, [0, 40], None, u))


def _deep(rng, m, kind):
    if kind == "chain":
        return list(range(-1, m - 1))
    if kind == "star":
        return [-1] + [rng.randrange(0, 3) for _ in range(m - 1)]
    if kind == "far":                                                     # ways up that skip whole blocks of rows, several roots, parents that are none
        return [rng.choice([-1, i - 1, i // 2, max(0, i - 300), i, 7]) if i % 97 else i + 5 for i in range(m)]
    return [-1 if i == 0 else rng.randrange(max(0, i - 3), i) for i in range(m)]


@pytest.mark.parametrize("counts,kind,words", [
    ([513], "chain", 16), ([3000, 2, 700], "deep", 16), ([2100, 512, 511], "far", 16), ([5000], "star", 3), ([1024, 768], "far", 1), ([4001], "chain", 2),
])
def test_trees_of_more_rows_than_masks_know(counts, kind, words):
    """What lies behind is climbed in steps that do not grow with the depth: masks and positions together, and each alone."""
    rng, T = random.Random(3), sum(counts) + 2
    parents = _ints([9] + [p for m in counts for p in _deep(rng, m, kind)] + [9])
    starts = [1]
    for m in counts:
        starts.append(starts[-1] + m)
    lens = _ints([m + 11 for m in counts])
    # what lies above: rows before this one, so their answers are there
    want_masks, want_positions = [[77] * words for _ in range(T)], [77] * T
    for b, (lo, hi) in enumerate(dref.spans(starts, T)):
        seen, depth = {}, {}
        for i in range(hi - lo):
            up = dref.above(parents, lo, i)
            seen[i] = seen.get(up, 0) | (1 << i if i < 32 * words else 0)
            depth[i] = depth.get(up, -1) + 1
            want_masks[lo + i], want_positions[lo + i] = [seen[i] >> 32 * w & 0xffffffff for w in range(words)], int(lens[b]) - (hi - lo) + depth[i]
    args = dict(parents=parents.to(DEV), q_starts=_ints(starts).to(DEV))
    fresh = lambda *s: torch.full(s, 77, dtype=torch.int32, device=DEV)
    masks, positions, alone, by_itself = fresh(T, words), fresh(T), fresh(T, words), fresh(T)
    binding.mom_mx_tree(lens.to(DEV), masks=masks, positions=positions, **args)
    binding.mom_mx_tree(lens.to(DEV), masks=alone, **args)
    binding.mom_mx_tree(lens.to(DEV), positions=by_itself, **args)
    assert [[w & 0xffffffff for w in r] for r in masks.tolist()] == want_masks and positions.tolist() == want_positions
    assert torch.equal(alone, masks) and torch.equal(by_itself, positions)


@pytest.mark.parametrize("listed", [True, False])
def test_a_chain_of_a_whole_prompt_and_a_tree_as_long(listed):
    m = 1 << 20
    lens = _ints([m + 5]).to(DEV)
    masks, positions = torch.full((m, 16), 77, dtype=torch.int32, device=DEV), torch.full((m,), 77, dtype=torch.int32, device=DEV)
    for parents in (None, torch.arange(-1, m - 1, dtype=torch.int32, device=DEV)):
        masks.fill_(77)
        positions.fill_(77)
        binding.mom_mx_tree(lens, parents=parents, q_starts=_ints([0, m]).to(DEV) if listed else None, masks=masks, positions=positions)
        assert torch.equal(positions, torch.arange(5, m + 5, dtype=torch.int32, device=DEV))
        i, j = torch.arange(m, device=DEV)[:, None], torch.arange(16, device=DEV) * 32
        bits = (i + 1 - j).clamp(0, 32)
        want = torch.where(bits == 32, -1, (1 << bits.clamp(max=31)) - 1).to(torch.int32)
        assert torch.equal(masks, torch.where(bits == 32, torch.full_like(want, -1), want))
