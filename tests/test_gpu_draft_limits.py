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
