"""The 8-bit cache on the GPU: append, read, attention and the page calls, against plain implementations in 64 bits."""
import math
import random

import pytest
import torch

import cache_plain
import kv8_plain as k8
import paper_2505_19634_b200 as tts

pytestmark = pytest.mark.gpu
FORMATS = [k8.E4M3, k8.INT8]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def context(hq, hkv, branches, rows, width, pages, **more):
    return tts.TtsContext(hq, hkv, branches, rows, width, pages, **more)


# ------------------------------------------------------------------------------------------------ append
def append_case(fmt, hq, hkv, chunk, lens, prefix, seed, first_row=0, rows_behind=0, stride_extra=0):
    c = k8.Cache8(fmt, hkv, lens, prefix=prefix, seed=seed)
    gen = torch.Generator().manual_seed(seed + 1)
    starts = [first_row]
    for n in chunk:
        starts.append(starts[-1] + n)
    rows = starts[-1] + rows_behind
    fused = torch.randn(rows, hq + 2 * hkv + stride_extra, 128, generator=gen).bfloat16().cuda()
    return c, starts, rows, fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:hq + 2 * hkv]


def places(c, chunk, starts):
    """(row, page, token of the page) of every appended row."""
    for b, n in enumerate(chunk):
        for i in range(n):
            t = c.prefix + c.lens[b] - n + i
            yield starts[b] + i, c.rows[b][t // 16], t % 16


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,chunk,lens,prefix", [(8, 2, [4, 4, 4], [4, 20, 37], 32), (40, 8, [1], [1], 0), (12, 1, [0, 33, 1, 16], [5, 40, 17, 16], 0),
                                                      (5, 5, [7] * 40, [9] * 40, 16)])
def test_append_without_rotation_is_exact(fmt, hq, hkv, chunk, lens, prefix):
    """Codes and scales are those of the definition, bit for bit; every other byte of the pool stays."""
    c, starts, rows, _, k, v = append_case(fmt, hq, hkv, chunk, lens, prefix, 1, first_row=2, rows_behind=3, stride_extra=1)
    v[3 % rows, 0] = 0                                              # a vector of zeros
    k[2, 0, 5] = 30000.0                                            # one large element
    ctx = context(hq, hkv, c.n, 1, c.width, c.num_pages)
    want_code, want_scale = (x.clone() for x in k8.unpack(c.pool))
    for kv, x in enumerate((k, v)):
        s = k8.scales(x.float(), fmt)
        code = k8.codes(x.float(), s, fmt)
        for row, page, t in places(c, chunk, starts):
            want_code[page, :, kv, t], want_scale[page, :, kv, t] = code[row], s[row]
    want = k8.pack(want_code[:, :, 0], want_code[:, :, 1], want_scale[:, :, 0], want_scale[:, :, 1])
    ctx.tts_kv8_append(fmt, None, None, 0, k, v, k.stride(0), None, c.pool, c.table, prefix, c.branch_lens, ints(starts), c.n, rows, None)
    assert torch.equal(c.pool, want) and ctx.tts_last_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("pairs,interleaved,axes", [(64, False, 1), (64, True, 3), (20, False, 2), (20, True, 1), (1, False, 1)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (7, 7)])
def test_append_with_rotation(fmt, pairs, interleaved, axes, hq, hkv):
    """Keys: the code is a nearest one to the rotated key (fp32 rotation: off by at most 2^-21 of the pair's length); queries as tts_kv_append_rope."""
    chunk, lens, prefix = [5, 0, 18], [30, 4, 18], 16
    c, starts, rows, q, k, v = append_case(fmt, hq, hkv, chunk, lens, prefix, 3)
    r = random.Random(4)
    axis, freq = [r.randrange(axes) for _ in range(pairs)], [10.0 ** -r.uniform(0, 4) for _ in range(pairs)]
    axis[0] = axes - 1
    pos = torch.randint(-100, 1 << 20, (axes, rows), generator=torch.Generator().manual_seed(5), dtype=torch.int32).cuda()
    ctx = context(hq, hkv, c.n, 1, c.width, c.num_pages)
    q_out, q_want = torch.empty(rows, hq, 128, device="cuda", dtype=torch.bfloat16), torch.empty(rows, hq, 128, device="cuda", dtype=torch.bfloat16)
    before = c.pool.clone()
    rope = tts.TtsRope(axis, freq, interleaved)
    ctx.tts_kv8_append(fmt, rope, q, q.stride(0), k, v, k.stride(0), pos, c.pool, c.table, prefix, c.branch_lens, ints(starts), c.n, rows, q_out)
    pools = torch.zeros(2, c.num_pages, hkv, 16, 128, device="cuda", dtype=torch.bfloat16)
    ctx.tts_kv_append_rope(rope, q, q.stride(0), k, v, k.stride(0), pos, pools[0], pools[1], c.table, prefix, c.branch_lens, ints(starts), c.n, rows, q_want)
    assert ctx.tts_last_status() == 0 and torch.equal(q_out, q_want)
    code, scale = k8.unpack(c.pool)
    turned = cache_plain.rope_turn(k.cpu(), pos.cpu(), axis, freq, interleaved).cuda()
    long = (k.double().abs().amax(-1) * math.sqrt(2) * 2.0 ** -21)[..., None]
    got = k8.table(fmt, "cuda")
    rows_at = torch.tensor(list(places(c, chunk, starts)), device="cuda")
    row, page, t = rows_at.unbind(1)
    s = scale[page, :, 0, t].double()
    assert ((s - turned[row].abs().amax(-1) / k8.LARGEST[fmt]).abs() <= s * 2.0 ** -20).all()
    y = got[code[page, :, 0, t].long()]
    # half a step at the code's value 2^(e-1) <= |y| < 2^e: 2^(e-5), from |y| = 64 (e = 7) on 4, and 2^-10 below 2^-6.  The exponent is taken
    # from the number's bits: a device's log2(64) may come out below 6.
    half = torch.where(y == 0, 2.0 ** -10, torch.exp2((torch.frexp(y).exponent - 5).clamp_min(-10).double())) if fmt == k8.E4M3 else 0.5
    assert ((y * s[..., None] - turned[row]).abs() <= half * s[..., None] * (1 + 1e-5) + long[row] * 2).all()
    # values, and everything that took no token
    vs = k8.scales(v.float(), fmt)
    assert torch.equal(code[page, :, 1, t], k8.codes(v.float(), vs, fmt)[row]) and torch.equal(scale[page, :, 1, t], vs[row])
    old_code, old_scale = k8.unpack(before)
    written = torch.zeros(c.num_pages, 16, dtype=torch.bool, device="cuda")
    written[page, t] = True
    assert torch.equal(code.permute(0, 3, 1, 2, 4)[~written], old_code.permute(0, 3, 1, 2, 4)[~written])
    assert torch.equal(scale.permute(0, 3, 1, 2)[~written].view(torch.int32), old_scale.permute(0, 3, 1, 2)[~written].view(torch.int32))


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_nan_and_infinity(fmt):
    c, starts, rows, _, k, v = append_case(fmt, 8, 2, [3], [3], 0, 6)
    k[0, 0, 7], v[1, 1, 0], k[2, 1, 1] = math.nan, math.inf, -math.inf
    ctx = context(8, 2, 1, 1, c.width, c.num_pages)
    ctx.tts_kv8_append(fmt, None, None, 0, k, v, k.stride(0), None, c.pool, c.table, 0, c.branch_lens, ints(starts), 1, rows, None)
    code, scale = k8.unpack(c.pool[c.rows[0][0]])
    bad = torch.zeros(2, 2, 3, dtype=torch.bool, device="cuda")
    bad[0, 0, 0] = bad[1, 1, 1] = bad[1, 0, 2] = True               # head, K or V, token
    assert torch.equal(scale[:, :, :3].isnan(), bad) and not code[:, :, :3][bad].any()


def test_append_reports_what_has_no_place():
    c, starts, rows, _, k, v = append_case(k8.INT8, 8, 2, [2, 2], [2, 2], 0, 7)
    ctx = context(8, 2, 2, 1, c.width, c.num_pages)
    before = c.pool.clone()

    def call(table=None, lens=None, start=None):
        ctx.tts_kv8_append(k8.INT8, None, None, 0, k, v, k.stride(0), None, c.pool, c.table if table is None else table, 0,
                           c.branch_lens if lens is None else ints(lens), ints(starts if start is None else start), 2, rows, None)
        return ctx.tts_last_status()

    for more in ({"start": [2, 0, 4]}, {"start": [0, 2, 5]}, {"start": [-1, 2, 4]}):
        assert call(**more) == -4 and torch.equal(c.pool, before)
    assert call(table=torch.full_like(c.table, c.num_pages)) == -4 and torch.equal(c.pool, before)
    assert call(lens=[1, 1]) == -4 and torch.equal(c.pool, before)
    assert call(lens=[16 * c.width + 1] * 2) == -4


# -------------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hkv,pages", [(2, 1), (1, 37), (8, 300)])
def test_read(fmt, hkv, pages):
    gen = torch.Generator().manual_seed(pages)
    code = torch.randint(0, 256, (pages, hkv, 2, 16, 128), generator=gen, dtype=torch.uint8)
    code[0, 0, 0, :2] = torch.arange(256, dtype=torch.uint8).view(2, 128)
    scale = torch.exp(8 * torch.randn(pages, hkv, 2, 16, generator=gen))
    pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1]).cuda()
    r = random.Random(1)
    src, dst = r.sample(range(pages), pages), r.sample(range(pages + 2), pages)
    src[pages // 2] = -1 if pages > 1 else src[0]
    k, v = (torch.full((pages + 2, hkv, 16, 128), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ctx = context(hkv, hkv, 1, 1, 1, pages)
    ctx.tts_kv8_read(fmt, pool, ints(src), ints(dst), pages, k, v, pages + 2)
    want = [torch.full((pages + 2, hkv, 16, 128), 7.0).bfloat16() for _ in range(2)]
    x = (k8.table(fmt)[code.long()].float() * scale[..., None]).bfloat16()
    for s, d in zip(src, dst):
        if s >= 0:
            want[0][d], want[1][d] = x[s, :, 0], x[s, :, 1]
    assert ctx.tts_last_status() == 0
    torch.testing.assert_close(k.cpu(), want[0], rtol=0, atol=0, equal_nan=True)
    torch.testing.assert_close(v.cpu(), want[1], rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("src,dst", [(4, 0), (0, 3), (1 << 30, 0)])
def test_read_reports_pages_outside(src, dst):
    pool = torch.zeros(4, 2, k8.RECORD, dtype=torch.uint8, device="cuda")
    k, v = (torch.full((3, 2, 16, 128), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ctx = context(2, 2, 1, 1, 1, 4)
    ctx.tts_kv8_read(0, pool, ints([src, 1]), ints([dst, 1]), 2, k, v, 3)
    assert ctx.tts_last_status() == -4 and not k[1].any() and (k[[0, 2]] == 7).all() and (v[[0, 2]] == 7).all()


# --------------------------------------------------------------------------------------------- attention
def attend(c, hq, rows, seed=0, parents=None, q=None, lse=True, out_dtype=tts.OUT_BF16, max_ctas=0, ctx=None, scale=0.0, status=0):
    if q is None:
        q = torch.randn(c.n * rows, hq, 128, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
    ctx = ctx or context(hq, c.hkv, c.n, rows, c.width, c.num_pages, out_dtype=out_dtype, max_ctas=max_ctas, softmax_scale=scale)
    out = torch.full((c.n * rows, hq, 128), math.nan, device="cuda", dtype=torch.bfloat16 if out_dtype == tts.OUT_BF16 else torch.float32)
    logs = torch.full((c.n * rows, hq), math.nan, device="cuda") if lse else None
    ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, c.prefix, c.branch_lens, None if parents is None else ints(parents), c.n, rows, out, logs)
    assert ctx.tts_last_status() == status
    return q, out, logs


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 1), (8, 2, 4), (40, 8, 1), (40, 8, 4), (12, 1, 2), (8, 8, 1), (28, 4, 3), (16, 1, 2), (33, 3, 3), (5, 5, 64)])
def test_attention_of_chains(fmt, hq, hkv, rows):
    c = k8.Cache8(fmt, hkv, [rows, rows + 15, max(rows, 16), max(rows, 17), rows + 300, rows + 31], prefix=32, seed=rows)
    q, out, lse = attend(c, hq, rows, seed=1)
    k8.assert_attention(c, q, rows, out, lse)


@pytest.mark.parametrize("lens,prefix", [([1], 0), ([1, 2, 16, 17, 128, 129], 0), ([2000], 48), ([1] * 200, 0), ([5000, 1, 1], 16)])
def test_attention_of_single_tokens(lens, prefix):
    c = k8.Cache8(k8.E4M3, 2, lens, prefix=prefix, seed=len(lens))
    q, out, lse = attend(c, 8, 1, seed=2, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 1, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 6), (40, 8, 60), (8, 1, 64), (2, 2, 33), (16, 2, 2)])
def test_attention_of_trees(fmt, hq, hkv, rows):
    r = random.Random(rows)
    c = k8.Cache8(fmt, hkv, [rows, rows + 9, rows + 150], prefix=16, seed=rows)
    parents = [[r.randrange(-1, i) if i else -1 for i in range(rows)] for _ in range(c.n)]
    parents[0] = list(range(-1, rows - 1))                          # a chain
    parents[1] = [-1] * rows                                        # a star
    q, out, lse = attend(c, hq, rows, seed=3, parents=parents)
    k8.assert_attention(c, q, rows, out, lse, parents=parents)
    chain, _, _ = attend(c, hq, rows, q=q)
    q, out2, lse2 = attend(c, hq, rows, q=q)
    assert torch.equal(out2[:rows], out[:rows]) and torch.equal(lse2[:rows], lse[:rows])        # the first branch's chain
    del chain


@pytest.mark.parametrize("max_ctas", [1, 2, 7, 0])
def test_attention_does_not_depend_on_the_split(max_ctas):
    """One CTA works through all items; several cut items between them in many places."""
    c = k8.Cache8(k8.INT8, 3, [300, 3, 3, 50, 700], prefix=16, seed=9)
    q, out, lse = attend(c, 9, 3, seed=4, max_ctas=max_ctas, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 3, out, lse)


def test_attention_repeats_itself():
    c = k8.Cache8(k8.E4M3, 8, [900, 40, 2000], prefix=64, seed=10)
    ctx = context(40, 8, 3, 4, c.width, c.num_pages)
    q, out, lse = attend(c, 40, 4, seed=5, ctx=ctx)
    for _ in range(5):
        _, again, lse2 = attend(c, 40, 4, q=q, ctx=ctx)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("parents", [None, [[-1, 0, 0, 1, 3], [-1, -1, 1, 1, 0], [-1, 0, 1, 2, 3]]])
def test_attention_of_rows_that_see_nothing(parents):
    """Branches shorter than their rows, and empty ones: zeros and -infinity, whatever the slots hold."""
    c = k8.Cache8(k8.E4M3, 2, [3, 0, 5], prefix=0, seed=11)
    q, out, lse = attend(c, 8, 5, seed=6, parents=parents)
    k8.assert_attention(c, q, 5, out, lse, parents=parents)
    assert not out[5:10].any() and (lse[5:10] == -math.inf).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_of_strided_queries_and_another_scale(fmt):
    c = k8.Cache8(fmt, 2, [40, 90], prefix=0, seed=12)
    fused = torch.randn(4, 12, 128, generator=torch.Generator().manual_seed(7)).bfloat16().cuda()
    q, out, lse = attend(c, 8, 2, q=fused[:, :8], scale=0.3)
    k8.assert_attention(c, q, 2, out, lse, scale=0.3)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_of_tokens_and_queries_of_very_different_size(fmt):
    """Scales of V from 2^-40 to 2^40 of one another, rising along the branch; rows of tiny, huge and no queries side by side."""
    c = k8.Cache8(fmt, 2, [200, 33], prefix=0, seed=13, poison=False)
    code, scale = k8.unpack(c.pool)
    for b, row in enumerate(c.rows):
        for i, page in enumerate(row):
            scale[page, :, 1] = 2.0 ** (-40 + 6 * i) * (1 + torch.arange(16, device="cuda") / 16)
    scale[c.rows[0][3], 0, :, 5] = 2.0 ** -120                      # a token of zeros as the append leaves it
    code[c.rows[0][3], 0, :, 5] = 0
    c.pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1])
    q = torch.randn(4, 8, 128, generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
    q[0, 0], q[1, 1], q[2, 2] = q[0, 0] * 2.0 ** -60, 0, q[2, 2] * 6
    q, out, lse = attend(c, 8, 2, q=q, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 2, out, lse)


def test_attention_keeps_bad_values_where_they_are():
    """A token whose V (or K) holds a NaN spoils the rows that see it, and only their heads; a row of infinite queries only itself."""
    c = k8.Cache8(k8.INT8, 2, [40], prefix=0, seed=14)
    q = torch.randn(4, 8, 128, generator=torch.Generator().manual_seed(9)).bfloat16().cuda()
    _, good, _ = attend(c, 8, 4, q=q)
    code, scale = k8.unpack(c.pool)
    scale[c.rows[0][2], 0, 1, 38 % 16] = math.nan                   # the second to last token, KV head 0
    c.pool = k8.pack(code[:, :, 0], code[:, :, 1], scale[:, :, 0], scale[:, :, 1])
    _, out, _ = attend(c, 8, 4, q=q)
    spoilt = torch.zeros(4, 8, dtype=torch.bool, device="cuda")
    spoilt[2:, :4] = True
    assert out.isnan().all(-1).equal(spoilt) and torch.equal(out[~spoilt], good[~spoilt])
    q2 = q.clone()
    q2[0, 5, 3] = math.inf
    _, out, _ = attend(c, 8, 4, q=q2)
    spoilt[0, 5] = True
    assert torch.equal(out[~spoilt], good[~spoilt]) and not torch.isfinite(out[0, 5]).any()


def test_attention_reports_bad_lengths_and_pages():
    c = k8.Cache8(k8.E4M3, 2, [40, 40, 40], prefix=0, seed=15)
    q, good, _ = attend(c, 8, 1, seed=10)
    for bad in (-1, 16 * c.width + 1, 2 ** 31 - 1):
        c.branch_lens = ints([40, bad, 40])
        _, out, lse = attend(c, 8, 1, q=q, status=-4)
        assert not out[1].any() and (lse[1] == -math.inf).all()
        # the others may be cut elsewhere, since the list of pages is another: both results are within the formula's bound of the exact one
        want, _, bound, _ = k8.attention(c, q, 1)
        assert ((out.double() - want).abs() <= bound + want.abs() * 2.0 ** -8)[[0, 2]].all()
    c.branch_lens = ints([40, 40, 40])
    table = c.table
    for bad in (-1, c.num_pages, 2 ** 30):
        c.table = table.clone()
        c.table[1, 1] = bad
        _, out, _ = attend(c, 8, 1, q=q, status=-4)
        assert torch.equal(out[[0, 2]], good[[0, 2]]) and torch.isfinite(out).all()
    # such a page counts as 16 tokens of zeros
    c.table = table
    rec = c.pool.clone()
    c.pool[c.rows[1][1]] = 0
    _, zeros, _ = attend(c, 8, 1, q=q)
    assert torch.equal(zeros, out)
    c.pool = rec


def test_attention_behind_32_bit_offsets():
    """Pages whose byte offsets pass 2^32."""
    c = k8.Cache8(k8.INT8, 8, [100, 37], prefix=16, seed=16, num_pages=140000)
    assert c.first * 8 * k8.RECORD > 2 ** 32
    q, out, lse = attend(c, 8, 2, seed=11)
    k8.assert_attention(c, q, 2, out, lse)


def test_a_captured_call_replays_on_new_data():
    c = k8.Cache8(k8.E4M3, 2, [300, 70], prefix=16, seed=17)
    ctx = context(8, 2, 2, 4, c.width, c.num_pages)
    stream = torch.cuda.Stream()
    ctx.tts_set_stream(stream)
    q = torch.randn(8, 8, 128, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(8, 8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(2):
            ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, 16, c.branch_lens, None, 2, 4, out, lse)
    for lens in ([300, 70], [4, 70], [250, 5]):
        c.lens = lens
        c.branch_lens.copy_(ints(lens))
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        k8.assert_attention(c, q, 4, out, lse)
    assert ctx.tts_last_status() == 0


def test_a_call_that_gave_up_leaves_the_context_usable():
    """The counters of parts, left in disorder as by a call that did not end, are set right when the status is read."""
    c = k8.Cache8(k8.E4M3, 2, [3000, 40], prefix=16, seed=20)
    ctx = context(8, 2, 2, 4, c.width, c.num_pages)
    q, good, lse = attend(c, 8, 4, seed=13, ctx=ctx)
    ctx.tts_debug_wait_timeout(1000000)
    assert ctx.tts_last_status() == -5
    _, again, lse2 = attend(c, 8, 4, q=q, ctx=ctx)
    assert torch.equal(again, good) and torch.equal(lse2, lse)


def test_read_pages_serve_the_chunk_attention():
    """A long chunk on an 8-bit context: its pages read back as bf16, then tts_chunk_attn; the last rows agree with tts_kv8_attn's
    within what the rounding of the values to bf16 (2^-9 in K's scores and in V) and of both results moves."""
    c = k8.Cache8(k8.INT8, 2, [100, 45], prefix=32, seed=18, poison=False)
    ctx = context(8, 2, 2, 4, c.width, c.num_pages)
    ctx.tts_chunk_reserve(8)
    k, v = (torch.zeros(c.num_pages, 2, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    pages = sorted({p for row in c.rows for p in row})
    ctx.tts_kv8_read(c.fmt, c.pool, ints(pages), ints(pages), len(pages), k, v, c.num_pages)
    q, out, _ = attend(c, 8, 4, seed=12, ctx=ctx)
    chunk = torch.empty_like(out)
    ctx.tts_chunk_attn(q, q.stride(0), k, v, c.table, 32, c.branch_lens, ints([0, 4, 8]), 2, 8, chunk)
    want, _, bound, _ = k8.attention(c, q, 4)
    size = torch.stack([c.kv(b)[1].abs().amax() for b in range(2)]).repeat_interleave(4)[:, None, None]
    # scores: 2^-9 of sums of magnitudes of at most 30; probabilities in bf16 2^-8; V 2^-9; result 2^-8
    assert ((chunk.double() - want).abs() <= bound + size * (2 * 30 * 2.0 ** -9 + 2.0 ** -8 + 2.0 ** -9) + want.abs() * 2.0 ** -8).all()
    assert ((out.double() - want).abs() <= bound + want.abs() * 2.0 ** -8).all()


# ------------------------------------------------------------------------------------------------- pages
@pytest.mark.parametrize("layers,hkv", [(1, 1), (3, 2), (128, 1)])
def test_fork_copy_and_compact_of_records(layers, hkv):
    """The same books as the bf16 cache's calls, and whole records moved in every pool."""
    gen = torch.Generator().manual_seed(layers)
    num = 24
    pools = [torch.randint(0, 256, (num, hkv, k8.RECORD), generator=gen, dtype=torch.uint8).cuda() for _ in range(layers)]
    book = cache_plain.Book([[0, 5, 9, -1], [0, 7, -1, -1], [0, 3, 20, 11]], 16, [20, 16, 40], num)
    ctx = context(hkv, hkv, 6, 1, 4, num)
    handle = tts.TtsKv8Pools(pools)
    refs = ints(book.refs())
    want = [x.clone() for x in pools]
    children, copies = book.fork([2, 0, 0, 2, -1, 2], book.refs())
    table, lens = torch.empty(6, 4, dtype=torch.int32, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda")
    ctx.tts_kv8_fork(handle, ints(book.table), 16, ints(book.lens), 3, ints([2, 0, 0, 2, -1, 2]), 6, refs, table, lens, refs)
    for x in want:
        for s, d in copies:
            x[d] = x[s]
    assert table.tolist() == children.table and lens.tolist() == children.lens and refs.tolist() == children.refs()
    assert len(copies) == 3 and all(torch.equal(x, y) for x, y in zip(pools, want))
    after, page_map, used = children.compact(children.refs())
    got_map, n_used = torch.empty(num, dtype=torch.int32, device="cuda"), ints([0])
    ctx.tts_kv8_compact(handle, table, 6, refs, table, refs, got_map, n_used)
    for x in want:
        old = x.clone()
        for s, d in enumerate(page_map):
            if d >= 0:
                x[d] = old[s]
    live = sorted({e for row in after.table for e in row if e >= 0})
    assert table.tolist() == after.table and got_map.tolist() == page_map and n_used.item() == used and refs.tolist() == after.refs()
    assert all(torch.equal(x[live], y[live]) for x, y in zip(pools, want))
    ctx.tts_kv8_copy_pages(handle, ints([live[0], -1, live[1]]), ints([num - 1, 2, num - 2]), 3)
    assert all(torch.equal(x[num - 1], x[live[0]]) and torch.equal(x[num - 2], x[live[1]]) for x in pools) and ctx.tts_last_status() == 0


# ---------------------------------------------------------------------------------------------- refusals
def test_refusals():
    c = k8.Cache8(k8.E4M3, 2, [20, 20], prefix=16, seed=19)
    ctx = context(8, 2, 2, 4, c.width, c.num_pages)
    q = torch.zeros(8, 8, 128, device="cuda", dtype=torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(8, 8, device="cuda")
    kv, starts, pos = torch.zeros(8, 2, 128, device="cuda", dtype=torch.bfloat16), ints([0, 4, 8]), ints([[0] * 8])
    rope = tts.TtsRope([0], [1.0])

    def refused(status, call, *args):
        with pytest.raises(tts.TtsError) as e:
            call(*args)
        assert e.value.status == status

    attn = [0, q, 1024, c.pool, c.table, 16, c.branch_lens, None, 2, 4, out, lse]
    append = [0, rope, q, 1024, kv, kv, 256, pos, c.pool, c.table, 16, c.branch_lens, starts, 2, 8, out]
    pages = torch.zeros(2, 8, 2, 16, 128, device="cuda", dtype=torch.bfloat16)
    read = [0, c.pool, ints([0, 1]), ints([0, 1]), 2, pages[0], pages[1], 8]

    def each(call, good, bad):
        call(*good)
        for at, value, status in bad:
            refused(status, call, *[value if i == at else x for i, x in enumerate(good)])

    each(ctx.tts_kv8_attn, attn, [(0, 2, -2), (0, -1, -2), (1, None, -1), (1, q.data_ptr() + 2, -1), (2, 1016, -1), (2, 1025, -1), (3, None, -1), (3, c.pool.data_ptr() + 8, -1),
                                  (4, None, -1), (5, 8, -1), (5, -16, -1), (5, 16 * (c.width + 1), -1), (6, None, -1), (8, 0, -1), (8, 3, -1), (9, 0, -1), (9, 5, -1),
                                  (10, None, -1), (10, q, -1), (10, out.data_ptr() + 4, -1), (10, c.pool, -1), (11, out, -1), (11, c.branch_lens, -1), (11, lse.data_ptr() + 1, -1)])
    each(ctx.tts_kv8_append, append, [(0, 5, -2), (1, None, -1), (2, None, -1), (3, 1000, -1), (4, None, -1), (6, 128, -1), (6, 260, -1), (7, None, -1), (8, None, -1),
                                      (8, kv, -1), (9, None, -1), (10, 7, -1), (12, None, -1), (13, 3, -1), (14, -1, -1), (15, None, -1), (15, kv, -1), (15, q.data_ptr() + 16, -1)])
    each(ctx.tts_kv8_read, read, [(0, 9, -2), (1, None, -1), (2, None, -1), (3, None, -1), (4, -1, -1), (5, None, -1), (5, c.pool, -1), (6, pages[0], -1), (6, pages[0, 1], -1), (7, 0, -1)])
    pools = tts.TtsKv8Pools([c.pool])
    refused(-1, ctx.tts_kv8_copy_pages, pools, None, ints([0]), 1)
    refused(-1, ctx.tts_kv8_copy_pages, tts.TtsKv8Pools([]), ints([0]), ints([0]), 1)
    refused(-1, ctx.tts_kv8_copy_pages, tts.TtsKv8Pools([c.pool, c.pool.data_ptr() + 4224]), ints([0]), ints([1]), 1)
    refused(-1, ctx.tts_kv8_copy_pages, tts.TtsKv8Pools([c.pool] * 129), ints([0]), ints([1]), 1)
    ctx.tts_kv8_copy_pages(tts.TtsKv8Pools([c.pool, c.pool, c.pool]), ints([0]), ints([0]), 1)
    assert ctx.tts_last_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("max_ctas", [1, 3, 10])
def test_single_tokens_of_more_items_than_ctas(fmt, max_ctas):
    """Items cut between CTAs, several to a CTA, some of them a page long."""
    c = k8.Cache8(fmt, 3, [700, 1, 2500, 16, 17, 90, 1300], prefix=16, seed=21)
    q, out, lse = attend(c, 12, 1, seed=14, max_ctas=max_ctas, out_dtype=tts.OUT_FP32)
    k8.assert_attention(c, q, 1, out, lse)
    _, again, _ = attend(c, 12, 1, q=q, max_ctas=max_ctas, out_dtype=tts.OUT_FP32)
    assert torch.equal(again, out)
