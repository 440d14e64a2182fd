"""What is left of the target's probabilities after refusals, on the GPU: trees of many rows, whose sums several workgroups share."""
import random

import pytest
import torch

import draft_reference as dref
from test_gpu_draft import DEV, _gen, _ints, _logits, _same, _tree, _verify

pytestmark = pytest.mark.gpu


def _down_the_later_children(gen, parents, m, V, refused):
    """Logits, tokens and numbers of one tree: the first `refused` children of a row are refused, as drawn tokens with numbers next to 1 mostly are; the others are the token that the target prefers most,
    with small numbers, so that the walk goes on."""
    target, draft = _logits(gen, m, V, False, True)
    tokens, uniforms = torch.zeros(m, dtype=torch.int32), torch.rand(m, generator=gen)
    ranks = [0] * m
    for i in range(1, m):
        up = dref.above(parents, 0, i)
        if up < 0:
            continue
        ranks[i] = sum(dref.above(parents, 0, j) == up for j in range(1, i))
        p, q = torch.softmax(target[up].double(), 0), torch.softmax(draft[up].double(), 0)
        if ranks[i] < refused:
            tokens[i], uniforms[i] = int(torch.multinomial(q, 1, generator=gen)), 0.9999
        else:
            tokens[i], uniforms[i] = int((p - 1.5 * q).topk(ranks[i] - refused + 1)[1][-1]), 0.05
    return target, draft, tokens, uniforms


@pytest.mark.parametrize("m,V,shape", [(66, 131077, "even"), (200, 131077, "random"), (512, 131077, "even"), (512, 4097, "random"), (130, 20000, "even")])
@pytest.mark.parametrize("refused", [1, 2])
def test_verify_of_one_tree_of_many_rows(m, V, shape, refused):
    """Workgroups that share a chunk's rows each make the list of them: it has to be the same list, also where refused children lie in several wavefronts."""
    gen, rng = _gen(m + V), random.Random(m)
    parents = _ints([-1] + [(i - 1) // 3 for i in range(1, m)] if shape == "even" else _tree(rng, m, 40))
    target, draft, tokens, uniforms = _down_the_later_children(gen, parents, m, V, refused)
    want = dref.verify(target, draft, tokens, parents, 4, [0, m], None, uniforms)
    assert want[2][0] >= 2
    for _ in range(3):                                                    # (the workspace holds other numbers each time)
        _same(_verify(target, tokens, uniforms, 1, draft, parents, 4), want)
