"""The order of beam selection where numbers are equal or nearly so."""
import math
import random

import pytest
import torch

import kv8_plain as k8
from test_gpu_beam import ints, normal, pick, starts

pytestmark = pytest.mark.gpu


def agrees(logits, scores, groups, beams, k, finished=None, pad=0):
    """Parents and tokens are the definition's, place by place."""
    parents, tokens, got = pick(logits, scores, groups, beams, k, finished, pad)
    want = k8.select(logits, scores, finished, pad, groups, beams, k)
    assert parents.tolist() == [[w[0] for w in g] for g in want]
    assert tokens.tolist() == [[w[1] for w in g] for g in want]
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [1, 16, 128])
@pytest.mark.parametrize("vocab,beams", [(40007, 1), (300, 3)])
def test_zeros_of_both_signs_are_equal(dtype, k, vocab, beams):
    """More of them than a part's list holds, and fewer; as the best logits and behind better ones."""
    r = random.Random(k)
    t = torch.arange(vocab)
    for negative in (t < 100, t % 2 == 0, t % 97 != 5):
        for better in (0, 7):
            x = torch.zeros(vocab)
            x[negative] = -0.0
            x[r.sample(range(vocab), better)] = 1.0
            agrees(x.repeat(beams, 1).to(dtype).cuda(), torch.full((beams,), -3.0, device="cuda"), 1, beams, k)
    x = torch.full((vocab,), -1.0)
    x[r.sample(range(vocab), 30)] = 0.0
    x[r.sample(range(vocab), 30)] = -0.0
    agrees(x.repeat(beams, 1).to(dtype).cuda(), torch.full((beams,), -3.0, device="cuda"), 1, beams, k)


def test_beams_are_told_apart_in_64_bits():
    """Rows of m zeros and nothing else: their sum of exponentials is m exactly, and two beams of different m whose scores differ by less
    than a step of 32 bits come in the order of score - log(m)."""
    r = random.Random(1)
    groups, vocab = 200, 5000
    x, scores, want = torch.full((2 * groups, vocab), -math.inf), torch.zeros(2 * groups), []
    for g in range(groups):
        m = r.sample(range(2, vocab), 2)
        near = torch.tensor(-r.uniform(9, 12))
        scores[2 * g] = near
        scores[2 * g + 1] = torch.tensor(float(near) - math.log(m[0]) + math.log(m[1]))
        both = [float(scores[2 * g + i]) - math.log(m[i]) for i in range(2)]
        assert 1e-12 < abs(both[0] - both[1]) < 2.0 ** -20
        for i in range(2):
            x[2 * g + i, r.sample(range(vocab), m[i])] = 0.0
        want.append([2 * g, 2 * g + 1] if both[0] > both[1] else [2 * g + 1, 2 * g])
    first = x.argmax(-1).tolist()
    parents, tokens, _ = pick(x.cuda(), scores.cuda(), groups, 2, 1)
    assert parents[:, 0].tolist() == [w[0] for w in want]
    assert tokens[:, 0].tolist() == [first[w[0]] for w in want]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [1, 5, 64])
@pytest.mark.parametrize("vocab,beams", [(40007, 1), (9001, 4), (33, 2)])
def test_scores_that_coincide_in_64_bits_go_to_the_lowest_tokens(dtype, k, vocab, beams):
    """A logit adds nothing to a score of -1e30, and one of 1e-25 nothing to any: different logits of one score, in descending order of beams
    that are clearly apart and of beams that are equal."""
    scores = torch.full((2 * beams,), -1e30)
    agrees(normal(2 * beams, vocab, dtype, vocab), scores.cuda(), 2, beams, k)
    tiny = normal(2 * beams, vocab, dtype, vocab + 1) * 1e-25
    agrees(tiny, torch.arange(2 * beams).neg().float().cuda(), 2, beams, k)
    some = tiny.clone()
    for b in range(2 * beams):
        some[b, [(7 * b + 11 * i) % vocab for i in range(3)]] = 0.5 + b
    agrees(some, torch.arange(2 * beams).neg().float().cuda(), 2, beams, k)
    mixed = normal(2 * beams, vocab, dtype, vocab + 2) - 6
    mixed[0::2] = tiny[0::2]
    agrees(mixed, (torch.arange(2 * beams) * -1e-2).cuda(), 2, beams, k)


def test_finished_beams_among_scores_that_coincide():
    """A finished beam is one candidate, at its own place, whatever its logits are."""
    x = normal(8, 3000, torch.float32, 3)
    agrees(x, torch.full((8,), -1e30, device="cuda"), 2, 4, 9, ints([0, 1, 0, 0, 1, 1, 0, 0]), pad=17)
    agrees(x, torch.full((8,), -1e30, device="cuda"), 1, 8, 128, ints([1, 1, 0, 1, 0, 0, 1, 1]), pad=2999)
    agrees(x * 1e-25, torch.tensor([-8.0, 0.0] * 4, device="cuda"), 2, 4, 9, ints([0, 1] * 4), pad=5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("groups,beams,k,vocab", [(3, 5, 16, 20000), (1, 64, 128, 9000), (16, 16, 16, 4099)])
def test_near_ties_are_candidates_of_the_definition(dtype, groups, beams, k, vocab):
    """Beams that hold the same logits in other orders, so that their candidates lie within the exponentials' error of one another: whatever
    order they come in, each is a candidate whose score is the one of its place, and none comes twice."""
    rows = groups * beams
    one = normal(groups, vocab, torch.float32, vocab).to(dtype)
    x = torch.stack([one[r // beams][torch.randperm(vocab, generator=torch.Generator().manual_seed(r)).cuda()] for r in range(rows)])
    scores = (starts(groups).repeat_interleave(beams) + torch.arange(rows, device="cuda") % 3 * 2.0 ** -21).contiguous()
    parents, tokens, got = pick(x, scores, groups, beams, k)
    exact = scores.double()[:, None] + torch.log_softmax(x.double(), -1)
    for g in range(groups):
        pairs = list(zip(parents[g].tolist(), tokens[g].tolist()))
        assert len(set(pairs)) == k and all(g * beams <= b < (g + 1) * beams and 0 <= t < vocab for b, t in pairs)
        mine = torch.stack([exact[b, t] for b, t in pairs])
        best = exact[g * beams:(g + 1) * beams].flatten().topk(k).values
        # each beam's sum is off by at most half of 2^-20 (see the scores' bound), so two that change places lie within all of it
        assert ((mine - best).abs() <= 2.0 ** -20).all() and (mine[1:] - mine[:-1] <= 2.0 ** -20).all()
        assert ((got[g].double() - mine).abs() <= mine.abs() * 2.0 ** -23 + 2.0 ** -21).all()
        assert (got[g, 1:] <= got[g, :-1]).all()
        # within a beam the order is exact
        for b in {b for b, _ in pairs}:
            own = [(-float(x[b, t]), t) for c, t in pairs if c == b]
            assert own == sorted(own)
