"""What is left of the target's probabilities after refusals, on the GPU: trees of many rows, whose sums several workgroups share, and rests that are next to nothing."""
import math
import random

import numpy as np
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


# What refusals leave

HALF = 2.0 ** -53
# A weight is off by the power's Taylor sum (5.5e-16) and some ten roundings, the sum that it is divided by by a rounding for every number that a lane adds up (64 of a chunk, the steps
# over lanes and chunks: under 100 in all).  That holds for both models, and either has at most all of its mass where the difference counts.
SIDE = 5.5e-16 + 110 * HALF
OFF = 2 * SIDE
NOTHING = 2.0 ** -42


def _exactly(logits, t):
    """softmax(logits / t) in the 64 bits of mantissa that the host has."""
    x = logits.to(torch.float64).numpy().astype(np.longdouble) / np.longdouble(t)
    e = np.exp(x - x.max())
    return e / e.sum()


def _could_be(x, u, weights, total):
    """Whether token x may be drawn with the number u from weights that are off by OFF in all, in part or in whole."""
    below = np.cumsum(weights)
    at, lo, hi = u * total, below[x] - weights[x], below[x]
    return lo - 2 * OFF <= at <= hi + 2 * OFF


@pytest.mark.parametrize("V", [9, 5000, 32001])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("t", [1.0, 0.6])
def test_a_draft_that_agrees_with_the_target(V, bf16, t):
    """A refusal leaves nothing then: p is what the next child is held against, and what is drawn from."""
    gen, B = _gen(V), 24
    target, _ = _logits(gen, 3 * B, V, bf16, False, spread=3.0)
    target[:, V // 2] = -math.inf
    parents, starts = _ints([-1, 0, 0] * B), [3 * b for b in range(B + 1)]
    tokens, uniforms = torch.randint(0, V // 2, (3 * B,), generator=gen).to(torch.int32), torch.rand(3 * B, generator=gen)
    for b in range(B):
        first, second = 3 * b + 1, 3 * b + 2
        if b % 3 == 0:
            tokens[first] = V // 2                                        # masked in both
        else:
            uniforms[first] = float(b % 3)                                # 1 and 2
        # the second is taken, refused by its number, or masked
        if b % 4 == 1:
            uniforms[second] = 1.0
        elif b % 4 == 2:
            tokens[second] = V // 2
    temps = torch.full((B,), t)
    want = dref.verify(target, target, tokens, parents, 2, starts, temps, uniforms)
    assert {1, 2} == set(want[2]) and min(o for o in want[1][0::3]) >= 0
    for children in (1, 2):
        want = dref.verify(target, target, tokens, parents, children, starts, temps, uniforms)
        _same(_verify(target, tokens, uniforms, B, target, parents, children, None, temps), want)


@pytest.mark.parametrize("V", [9, 9001])
@pytest.mark.parametrize("drafted", [True, False])
def test_rows_of_one_token(V, drafted):
    """A probability of 1 and numbers of 1 and more: refused, nothing is left, and it is drawn from p."""
    B, hot = 6, [3, V - 1, 0, V // 2, 5, 1]
    target = torch.full((4 * B, V), -math.inf)
    for b in range(B):
        target[4 * b:4 * b + 4, hot[b]] = -3.0 + b
    parents, starts = _ints([-1, 0, 0, 0] * B), [4 * b for b in range(B + 1)]
    tokens = torch.zeros(4 * B, dtype=torch.int32)
    for b in range(B):
        tokens[4 * b + 1:4 * b + 4] = hot[b]
    tokens[1 + 4 * 4] = (hot[4] + 1) % V                                  # another token first
    uniforms = torch.tensor([0.3, 1.0, 0.5, 0.5, 0.0, 2.0, 2.0, 0.999, 0.999, 1.0, 1.0, 1.0, 1.0, 2.0, 2.0, 2.0, 0.5, 1.0, 1.0, 0.7, 2.0, 1.0, 2.0, 0.0])
    draft = target if drafted else None
    for children in (1, 2, 3):
        want = dref.verify(target, draft, tokens, parents, children, starts, None, uniforms)
        assert [want[1][4 * b] for b in range(B)] == hot
        _same(_verify(target, tokens, uniforms, B, draft, parents, children), want)


def test_models_that_differ_by_little():
    """Both have one token far above the others, a lower one is refused first: what is left is a part in 10^6 to 10^14, as right as 64 bits allow.  Every other sequence has two such tokens and differs where
    there is hardly any weight."""
    gen, V, B = _gen(31), 5000, 240
    target = torch.randn((2 * B, V), generator=gen)
    draft = target + 0.5 * torch.randn((2 * B, V), generator=gen)
    uniforms, tokens, temps = torch.rand(2 * B, generator=gen), torch.zeros(2 * B, dtype=torch.int32), torch.ones(B)
    for b in range(B):
        r, peak = 2 * b, int(torch.randint(1, V, (1,), generator=gen))
        temps[b] = (1.0, 0.8, 0.6, 0.45)[b % 4]
        height = float(temps[b]) * (18.0 + 24.0 * (b // 8) / (B // 8))
        if b // 4 % 2:
            draft[r] = target[r]
            draft[r, 7:9] += torch.tensor([1.0, -0.5])
            target[r, peak - 1], draft[r, peak - 1] = height - 0.25, height - 0.25
        target[r, 0] -= 4.0 * (b % 3)                                     # the first logit, which sums are relative to, differs
        target[r, peak], draft[r, peak] = height, height
        p, q = _exactly(target[r], float(temps[b])), _exactly(draft[r], float(temps[b]))
        lower = np.where(q > 1.05 * p, q, 0.0)
        tokens[r + 1], uniforms[r + 1] = int(lower.argmax()), 0.99999
    starts = [2 * b for b in range(B + 1)]
    rows, out, counts = _verify(target, tokens, uniforms, B, draft, None, 1, None, temps)
    wrong, kinds = [], [0, 0]
    for b in range(B):
        r, u = 2 * b, float(uniforms[2 * b])
        p, q = _exactly(target[r], float(temps[b])), _exactly(draft[r], float(temps[b]))
        x = int(tokens[r + 1])
        assert float(uniforms[r + 1]) * q[x] > p[x] * (1 + 1e-3)          # refused, and by a margin
        assert rows[r:r + 2] == [0, -1] and counts[b] == 1 and out[r + 1] == -1
        left = np.maximum(p - q, 0)
        rest = left.sum()
        kinds[int(rest > NOTHING)] += 1
        fits = [_could_be(out[r], u, left, rest), _could_be(out[r], u, p, 1.0)] if 0 <= out[r] < V else [False, False]
        # (a rest that is as near to the border as it may be off may be either)
        if not (any(fits) if abs(rest - NOTHING) <= OFF else fits[int(rest < NOTHING)]):
            wrong.append((b, out[r], float(rest)))
    assert not wrong, (len(wrong), wrong[:5])
    assert min(kinds) > 30
    # among them many whose rest is so large that the token is the definition's
    want = dref.verify(target, draft, tokens, None, 1, starts, temps, uniforms)
    sure = [b for b in range(B) if np.maximum(_exactly(target[2 * b], float(temps[b])) - _exactly(draft[2 * b], float(temps[b])), 0).sum() > 1e-7]
    assert len(sure) >= 10 and [out[2 * b] for b in sure] == [want[1][2 * b] for b in sure]


def test_a_child_after_refusals_that_leave_next_to_nothing():
    """The first child is a low one, the second the token that both models put nearly everything on: with a rest under 2^-42 it is held against p again."""
    gen, V, B = _gen(33), 5000, 16
    target = torch.randn((3 * B, V), generator=gen)
    draft = target + 0.5 * torch.randn((3 * B, V), generator=gen)
    peaks = torch.randint(0, V, (B,), generator=gen)
    tokens, uniforms = torch.zeros(3 * B, dtype=torch.int32), torch.rand(3 * B, generator=gen)
    for b in range(B):
        target[3 * b, peaks[b]] = draft[3 * b, peaks[b]] = 45.0
        p, q = _exactly(target[3 * b], 1.0), _exactly(draft[3 * b], 1.0)
        assert np.maximum(p - q, 0).sum() < NOTHING / 2
        tokens[3 * b + 1], uniforms[3 * b + 1] = int(np.where(q > 1.05 * p, q, 0.0).argmax()), 0.99999
        tokens[3 * b + 2], uniforms[3 * b + 2] = int(peaks[b]), 0.9 if b % 2 else 1.5
    rows, out, counts = _verify(target, tokens, uniforms, B, draft, _ints([-1, 0, 0] * B), 2)
    for b in range(B):
        assert counts[b] == (2 if b % 2 else 1) and out[3 * b] == int(peaks[b])
        assert rows[3 * b:3 * b + 3] == ([0, 2, -1] if b % 2 else [0, -1, -1])


@pytest.mark.parametrize("chunked", [False, True])
def test_tokens_taken_off_without_a_drafting_model(chunked):
    """What the refused tokens leave is summed without them where little is left: few tokens among many that are masked, and tokens far below the refused one."""
    gen, B = _gen(32), 40
    V = 20000 if chunked else 600
    target = torch.full((4 * B, V), -math.inf)
    tokens, uniforms = torch.zeros(4 * B, dtype=torch.int32), torch.rand(4 * B, generator=gen)
    for b in range(B):
        r, places = 4 * b, torch.randperm(V, generator=gen)[:5].sort()[0]
        if chunked:
            places = 4096 * torch.arange(5) + torch.randint(0, 3600, (5,), generator=gen)        # a chunk each
        if b % 2:
            target[r, places] = torch.tensor([0.1, 1.7, 0.9, 1.3, -0.4])
            tokens[r + 1:r + 4] = places[:3] if b % 4 == 1 else places[[2, 2, 4]]
            uniforms[r + 1:r + 4] = 0.995
        else:
            target[r] = torch.randn(V, generator=gen)
            target[r, places[0]] = 3.0 + 0.5 * b                          # all but 1e-9 of it at the most
            tokens[r + 1:r + 4] = int(places[0])
            uniforms[r + 1:r + 4] = 1.0
        if b % 8 > 4:
            uniforms[r] = 0.0
    parents, starts = _ints([-1, 0, 0, 0] * B), [4 * b for b in range(B + 1)]
    for children in (1, 2, 3):
        want = dref.verify(target, None, tokens, parents, children, starts, None, uniforms)
        _same(_verify(target, tokens, uniforms, B, None, parents, children), want)
