"""The order of beam selection where numbers are equal or nearly so."""
import random

import pytest
import torch

import kv8_plain as k8
from test_gpu_beam import pick

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
