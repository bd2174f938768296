"""Attention over the 8-bit cache: what a row does not see does not change its result, whatever size it has."""
import math
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from test_gpu_kv8 import FORMATS, attend, context, ints

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


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 4), (40, 8, 4), (16, 1, 8), (8, 2, 40)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("into", ["k", "v"])
def test_appended_tokens_that_are_not_finite_spoil_the_rows_that_see_them_alone(fmt, hq, hkv, rows, bad, into):
    """The last tokens are appended, one of them with a NaN or an infinity in head 0: what does not see it is what it is without."""
    lens = [rows, 70 + rows]
    gen = torch.Generator().manual_seed(rows)
    new = torch.randn(2, 2 * rows, hkv, 128, generator=gen).bfloat16().cuda()
    spoilt = new.clone()
    spoilt["kv".index(into), rows - 2, 0, 5] = spoilt["kv".index(into), 2 * rows - 2, 0, 77] = bad
    q, results = None, []
    for kv in (new, spoilt):
        c = k8.Cache8(fmt, hkv, lens, prefix=0, seed=rows)
        ctx = context(hq, hkv, 2, rows, c.width, c.num_pages)
        ctx.tts_kv8_append(fmt, None, None, 0, kv[0], kv[1], hkv * 128, None, c.pool, c.table, 0, c.branch_lens, ints([0, rows, 2 * rows]), 2, 2 * rows, None)
        q, out, lse = attend(c, hq, rows, seed=2, q=q, ctx=ctx)
        results.append((out, lse))
    sees = torch.zeros(2 * rows, hq, dtype=torch.bool, device="cuda")
    sees[rows - 2:rows, :hq // hkv] = sees[2 * rows - 2:, :hq // hkv] = True
    (good, good_lse), (out, lse) = results
    assert out.isnan().all(-1).equal(sees) and torch.isfinite(good).all()
    assert torch.equal(out[~sees], good[~sees]) and torch.equal(lse[~sees], good_lse[~sees])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows,prefix", [(8, 2, 4, 8192), (10, 2, 1, 4096), (28, 2, 8, 8192), (8, 1, 16, 2048)])
def test_a_long_prefix(fmt, hq, hkv, rows, prefix):
    c = k8.Cache8(fmt, hkv, [rows, 37 + rows, 500 + rows, 130], prefix=prefix, seed=rows)
    q, out, lse = attend(c, hq, rows, seed=3)
    k8.assert_attention(c, q, rows, out, lse)
