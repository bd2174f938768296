"""Attention over the 8-bit cache: what a row does not see does not change its result, whatever size it has."""
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from test_gpu_kv8 import FORMATS, attend

pytestmark = pytest.mark.gpu
# rows of one KV head: those of one block of the kernel for few, those of the kernel for many
SHAPES = [(8, 2, 1, 2), (8, 2, 4, 1), (40, 8, 4, 1), (12, 2, 8, 2), (16, 1, 4, 3), (14, 1, 8, 1), (40, 8, 24, 5), (3, 1, 60, 20)]


def scaled(c, tokens, factor):
    """The cache with V of the given tokens (counted from the end) of every branch so many times as large."""
    other = k8.Cache8.__new__(k8.Cache8)
    other.__dict__.update(c.__dict__)
    code, scale = k8.unpack(c.pool)
    for b, row in enumerate(c.rows):
        for back in tokens:
            t = c.prefix + c.lens[b] - back
            if t >= 0:
                scale[row[t // 16], :, 1, t % 16] *= factor
    other.pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1])
    return other


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows,back", SHAPES)
@pytest.mark.parametrize("power", [30, 60, 110])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_that_do_not_see_a_large_value(fmt, hq, hkv, rows, back, power, tree):
    """V of the `back` last tokens is 2^power times the others'.  Rows that see none of them are within the bound of the cache without them;
    the others within their own."""
    if rows == 1:
        back = 0                                                    # (a single token sees all: V of no token is large)
    r = random.Random(rows)
    lens = [rows, rows + 9, 40 + rows, 300 + rows]
    parents = [[r.randrange(-1, i) if i else -1 for i in range(rows)] for _ in lens] if tree else None
    c = k8.Cache8(fmt, hkv, lens, prefix=0, seed=rows + power)
    large = scaled(c, range(1, back + 1), 2.0 ** power)
    q, out, lse = attend(large, hq, rows, seed=1, parents=parents, out_dtype=tts.OUT_FP32)
    want, want_lse, bound, lse_bound = k8.attention(c, q, rows, parents)
    want2, _, bound2, _ = k8.attention(large, q, rows, parents)
    for b, n in enumerate(lens):
        hidden = ~k8.sees(rows, n, parents[b] if tree else None)[:, n - back:].any(-1) if back else torch.ones(rows, dtype=torch.bool)
        assert hidden[0] or back >= rows
        for i in range(rows):
            at = b * rows + i
            x, y = (want, bound) if hidden[i] else (want2, bound2)
            assert ((out[at].double() - x[at]).abs() <= y[at] + x[at].abs() * 2.0 ** -24).all(), (b, i, bool(hidden[i]))
    assert ((lse.double() - want_lse).abs() <= lse_bound).all()
