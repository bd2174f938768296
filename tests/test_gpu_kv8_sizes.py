"""Attention over the 8-bit cache where scores are so large that their own rounding is worth many powers of two."""
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from test_gpu_kv8 import FORMATS, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 1), (8, 2, 4), (40, 8, 4), (21, 3, 51), (49, 1, 1), (16, 2, 16)])
@pytest.mark.parametrize("out_dtype", [tts.OUT_BF16, tts.OUT_FP32])
def test_scores_of_any_size(fmt, hq, hkv, rows, out_dtype):
    """Keys whose sizes differ by e^18 and more: scores up to 2^33, whose neighbours in fp32 are 2^9 apart.  Results stay finite and within the formula's
    bound; the row's largest token has all of its weight."""
    r, largest = random.Random(rows), 0.0
    for seed in range(3):
        c = k8.Cache8(fmt, hkv, [rows, 500 + rows, 1100 + rows, 1], prefix=16 * r.randrange(3), seed=seed, spread=6.0)
        q, out, lse = attend(c, hq, rows, seed=seed + 1, out_dtype=out_dtype, max_ctas=r.choice([0, 3]))
        largest = max(largest, lse.abs()[torch.isfinite(lse)].max().item())
        k8.assert_attention(c, q, rows, out, lse)
    assert largest > 2.0 ** 27                                      # (that these inputs are what the test is about)
