"""Attention over the 8-bit cache with more rows to a KV head than one block of the other kernel takes: trees and long chains of large head
groups, against the formula in 64 bits."""
import math
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from test_gpu_kv8 import FORMATS, attend, context, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows", [(49, 1, 1), (7, 1, 7), (25, 1, 2), (32, 1, 4), (43, 1, 3), (16, 2, 16), (24, 3, 7), (16, 1, 64), (3, 3, 64), (128, 1, 2)])
def test_chains(fmt, hq, hkv, rows):
    """49, 50, 128, 129, 1024, .. rows to a KV head; tiles of 64 tokens that are full, one short, one over."""
    c = k8.Cache8(fmt, hkv, [rows, rows + 1, max(rows, 31), max(rows, 32), max(rows, 33), 112 + rows, 400, 1], prefix=32, seed=rows)
    q, out, lse = attend(c, hq, rows, seed=1)
    k8.assert_attention(c, q, rows, out, lse)


@pytest.mark.parametrize("max_ctas", [1, 2, 5, 37, 0])
def test_trees_cut_between_ctas(max_ctas):
    r = random.Random(1)
    rows = 25
    c = k8.Cache8(k8.E4M3, 2, [rows, 3000, 70, rows + 1, 1500], prefix=48, seed=2)
    parents = [[r.randrange(-1, i) if i else -1 for i in range(rows)] for _ in range(c.n)]
    q, out, lse = attend(c, 8, rows, seed=3, parents=parents, max_ctas=max_ctas, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, rows, out, lse, parents=parents)


def test_one_long_branch_in_many_parts():
    c = k8.Cache8(k8.INT8, 1, [20000], seed=4)
    q, out, lse = attend(c, 8, 8, seed=5, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 8, out, lse)


def test_many_short_branches():
    c = k8.Cache8(k8.INT8, 2, [1 + i % 90 for i in range(300)], seed=6)
    q, out, lse = attend(c, 14, 8, seed=7)
    k8.assert_attention(c, q, 8, out, lse)


def test_repeats_itself():
    c = k8.Cache8(k8.E4M3, 4, [2500, 40, 900], prefix=64, seed=8)
    ctx = context(32, 4, 3, 10, c.width, c.num_pages)
    q, out, lse = attend(c, 32, 10, seed=9, ctx=ctx)
    for _ in range(5):
        _, again, lse2 = attend(c, 32, 10, q=q, ctx=ctx)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("tree", [False, True])
def test_rows_that_see_nothing(tree):
    parents = [[-1 if i % 5 == 0 else i - 1 for i in range(64)]] * 3 if tree else None
    c = k8.Cache8(k8.E4M3, 2, [3, 0, 5], seed=10)
    q, out, lse = attend(c, 4, 64, seed=11, parents=parents)
    k8.assert_attention(c, q, 64, out, lse, parents=parents)
    assert not out[64:128].any() and (lse[64:128] == -math.inf).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_and_queries_of_very_different_size(fmt):
    """Scales of V rising by 2^6 a page, queries from 2^-60 to 6 times the usual and zeros, in one block of rows."""
    c = k8.Cache8(fmt, 1, [200, 133], seed=12, poison=False)
    code, scale = k8.unpack(c.pool)
    for row in c.rows:
        for i, page in enumerate(row):
            scale[page, :, 1] = 2.0 ** (-40 + 6 * i) * (1 + torch.arange(16, device="cuda") / 16)
    scale[c.rows[0][3], 0, :, 5] = 2.0 ** -120                      # a token of zeros as the append leaves it
    code[c.rows[0][3], 0, :, 5] = 0
    c.pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1])
    q = torch.randn(12, 10, 128, generator=torch.Generator().manual_seed(13)).bfloat16().cuda()
    q[0, 0], q[1, 1], q[2, 2] = q[0, 0] * 2.0 ** -60, 0, q[2, 2] * 6
    q, out, lse = attend(c, 10, 6, q=q, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 6, out, lse)


def test_bad_values_stay_where_they_are():
    c = k8.Cache8(k8.INT8, 2, [140], seed=14)
    q = torch.randn(16, 8, 128, generator=torch.Generator().manual_seed(15)).bfloat16().cuda()
    _, good, _ = attend(c, 8, 16, q=q)
    code, scale = k8.unpack(c.pool)
    scale[c.rows[0][8], 0, 1, 138 % 16] = math.nan                  # the second to last token, KV head 0: rows 14 and 15 see it
    c.pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1])
    _, out, _ = attend(c, 8, 16, q=q)
    spoilt = torch.zeros(16, 8, dtype=torch.bool, device="cuda")
    spoilt[14:, :4] = True
    assert out.isnan().all(-1).equal(spoilt) and torch.equal(out[~spoilt], good[~spoilt])
    q2 = q.clone()
    q2[0, 5, 3] = math.inf
    _, out, _ = attend(c, 8, 16, q=q2)
    spoilt[0, 5] = True
    assert torch.equal(out[~spoilt], good[~spoilt]) and not torch.isfinite(out[0, 5]).any()


def test_bad_lengths_and_pages_are_reported():
    c = k8.Cache8(k8.E4M3, 2, [140, 140, 140], seed=16)
    q, good, _ = attend(c, 8, 14, seed=17)
    for bad in (-1, 16 * c.width + 1, 2 ** 31 - 1):
        c.branch_lens = ints([140, bad, 140])
        _, out, lse = attend(c, 8, 14, q=q, status=-4)
        assert not out[14:28].any() and (lse[14:28] == -math.inf).all()
    c.branch_lens = ints([140, 140, 140])
    table = c.table
    for bad in (-1, c.num_pages, 2 ** 30):
        c.table = table.clone()
        c.table[1, 5] = bad
        _, out, _ = attend(c, 8, 14, q=q, status=-4)
        assert torch.equal(out[:14], good[:14]) and torch.equal(out[28:], good[28:]) and torch.isfinite(out).all()
    c.table = table
    c.pool[c.rows[1][5]] = 0                                        # such a page counts as 16 tokens of zeros
    _, zeros, _ = attend(c, 8, 14, q=q)
    assert torch.equal(zeros, out)


def test_behind_32_bit_offsets():
    c = k8.Cache8(k8.E4M3, 8, [100, 37], prefix=16, seed=18, num_pages=140000)
    assert c.first * 8 * k8.RECORD > 2 ** 32
    q, out, lse = attend(c, 64, 7, seed=19)
    k8.assert_attention(c, q, 7, out, lse)


def test_strided_queries_another_scale_and_few_rows_on_the_same_context():
    c = k8.Cache8(k8.INT8, 1, [90, 260], seed=20)
    fused = torch.randn(16, 12, 128, generator=torch.Generator().manual_seed(21)).bfloat16().cuda()
    ctx = context(8, 1, 2, 8, c.width, c.num_pages, softmax_scale=0.2)
    for rows in (8, 2, 8, 7):
        q, out, lse = attend(c, 8, rows, q=fused[:2 * rows, :8], ctx=ctx)
        k8.assert_attention(c, q, rows, out, lse, scale=0.2)


def test_captured_calls_replay_on_new_data():
    c = k8.Cache8(k8.E4M3, 2, [900, 170], prefix=16, seed=22)
    ctx = context(16, 2, 2, 8, c.width, c.num_pages)
    stream = torch.cuda.Stream()
    ctx.tts_set_stream(stream)
    q = torch.randn(16, 16, 128, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(16, 16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(2):
            ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, 16, c.branch_lens, None, 2, 8, out, lse)
    for lens in ([900, 170], [8, 170], [750, 9]):
        c.lens = lens
        c.branch_lens.copy_(ints(lens))
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        k8.assert_attention(c, q, 8, out, lse)
    assert ctx.tts_last_status() == 0


def test_a_call_that_gave_up_leaves_the_context_usable():
    c = k8.Cache8(k8.E4M3, 2, [6000, 40], prefix=16, seed=23)
    ctx = context(16, 2, 2, 8, c.width, c.num_pages)
    q, good, lse = attend(c, 16, 8, seed=24, ctx=ctx)
    ctx.tts_debug_wait_timeout(1000000)
    assert ctx.tts_last_status() == -5
    _, again, lse2 = attend(c, 16, 8, q=q, ctx=ctx)
    assert torch.equal(again, good) and torch.equal(lse2, lse)


@pytest.mark.parametrize("rows", [1, 8])
def test_as_many_branches_as_there_can_be(rows):
    """1024 of them, some of them empty but for the prefix, for both kernels (8 and 64 rows)."""
    c = k8.Cache8(k8.INT8, 1, [i % 23 if i % 7 else 0 for i in range(1024)], prefix=32, seed=25 + rows)
    q, out, lse = attend(c, 8, rows, seed=26)
    k8.assert_attention(c, q, rows, out, lse)


@pytest.mark.parametrize("hq,hkv,rows", [(8, 1, 1), (8, 1, 8)])
def test_two_streams_with_a_context_each(hq, hkv, rows):
    """The same pages read at the same time by two contexts on two streams."""
    c = k8.Cache8(k8.E4M3, hkv, [3000, 170, 900], prefix=16, seed=27)
    q = torch.randn(3 * rows, hq, 128, generator=torch.Generator().manual_seed(28)).bfloat16().cuda()
    _, want, _ = attend(c, hq, rows, q=q)
    streams, contexts, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for s in streams:
        ctx = context(hq, hkv, 3, rows, c.width, c.num_pages)
        ctx.tts_set_stream(s)
        contexts.append(ctx)
        outs.append(torch.zeros_like(want))
    torch.cuda.synchronize()
    for _ in range(20):
        for ctx, out in zip(contexts, outs):
            ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, 16, c.branch_lens, None, 3, rows, out, None)
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out in outs) and all(ctx.tts_last_status() == 0 for ctx in contexts)
