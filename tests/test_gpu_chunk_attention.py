"""Attention of ragged chunks (tts_chunk_attn) against a plain implementation in 64 bits.

Tolerance of an output element.  Scores are fp32 sums of 128 exact products: at most 128 x 2^-23 of the sum of
their magnitudes, about 7 after the scale for N(0, 1) inputs, so 1.1e-4 in the exponent, plus 2^-22 of the
hardware's 2^x.  The probabilities are rounded to bf16 before the second contraction (2^-8 of each), the output to
bf16 (2^-8 of it) unless fp32 is asked for.  With A the softmax mean of |V|:
    |out - exact| <= 2^-8 |exact| + (2^-8 + 2^-12) A        (2^-12 covers the score error and fp32 sums)
and lse is off by at most 1.5e-4 (2^-12 with larger scores).
"""
import math

import pytest
import torch

import paper_2505_19634_b200 as tts
from cache_plain import PAGE, Cache, chunk_attention

pytestmark = pytest.mark.gpu


def context(c: Cache, rows=None, **kw):
    ctx = tts.TtsContext(c.hq, c.hkv, c.n, 1, c.width, c.num_pages, **kw)
    ctx.tts_chunk_reserve(rows or max(1, c.total_rows))
    return ctx


def call(ctx, c: Cache, out, lse=None, q=None, table=None, row_start=None, lens=None):
    q = c.q if q is None else q
    ctx.tts_chunk_attn(q, q.stride(0), c.k, c.v, c.table if table is None else table, c.prefix, c.branch_lens if lens is None else lens,
                       c.row_start if row_start is None else row_start, c.n, c.total_rows, out, lse)


def run(c: Cache, dtype=torch.bfloat16, ctx=None, **kw):
    own = ctx is None
    ctx = ctx or context(c, out_dtype=tts.OUT_FP32 if dtype == torch.float32 else tts.OUT_BF16, **kw)
    out = torch.full((c.total_rows, c.hq, 128), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((c.total_rows, c.hq), 7.0, device="cuda")
    call(ctx, c, out, lse)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    if own:
        ctx.close()
    return out, lse


def check(c: Cache, out, lse, scale=None, lse_tol=1.5e-4):
    want, want_lse, mean = chunk_attention(c, scale)
    mine = torch.zeros(c.total_rows, dtype=torch.bool, device="cuda")
    mine[c.starts[0]:c.starts[-1]] = True
    got = out.double()
    assert (got[~mine] == 7).all() and (lse[~mine] == 7).all()          # rows of no branch are left as they were
    got, want, mean, l, wl = got[mine], want[mine], mean[mine], lse.double()[mine], want_lse[mine]
    assert torch.isfinite(got).all()
    last = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -23
    off = (got - want).abs() - (last * want.abs() + (2.0 ** -8 + 2.0 ** -12) * mean)
    assert off.max() <= 0, f"outside the bound by {off.max().item():.3e}"
    rms = ((got - want).square().mean().sqrt() / want.square().mean().sqrt().clamp_min(1e-30)).item()
    assert rms <= 5e-3, rms
    empty = wl == -math.inf
    assert torch.equal(l == -math.inf, empty) and (got[empty] == 0).all()
    if (~empty).any():
        assert (l - wl)[~empty].abs().max() <= lse_tol
    return rms


HEADS = [(8, 2), (40, 8), (16, 2), (7, 1), (8, 8), (64, 1), (33, 1), (128, 1), (3, 3)]


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_head_layouts_ragged_chunks(hq, hkv):
    c = Cache(hq, hkv, chunk=[1, 37, 0, 130, 16, 5], lens=[77, 37, 50, 211, 1040, 5], prefix=48, seed=hq)
    check(c, *run(c))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 24, 25, 26, 49, 50, 51, 75, 76, 127, 128, 129, 255, 256, 257])
def test_lengths_around_pages_and_tiles(n):
    """One branch, a chunk that is its whole cache: every edge of pages (16), row tiles (25 and 50 tokens at five
    heads per KV head) and key tiles (128)."""
    c = Cache(5, 1, chunk=[n], lens=[n], seed=n)
    check(c, *run(c))
    c = Cache(5, 1, chunk=[1], lens=[n], seed=n)
    check(c, *run(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_branches_mixed(dtype):
    g = torch.Generator().manual_seed(3)
    chunk = [1 if i % 3 else int(torch.randint(1, 200, (1,), generator=g)) for i in range(40)]
    lens = [x + int(torch.randint(0, 900, (1,), generator=g)) for x in chunk]
    c = Cache(40, 8, chunk=chunk, lens=lens, prefix=64, seed=5)
    check(c, *run(c, dtype))


@pytest.mark.parametrize("hq,hkv,chunk,lens", [
    (8, 1, [1], [20000]),                # one token over a long cache: cut into many pieces
    (5, 1, [60], [9000]),                # two row tiles over a long cache, cut
    (40, 8, [1, 300], [9000, 6011]),
    (4, 4, [700], [700]),                # causal within the chunk, pieces of different lengths
])
@pytest.mark.parametrize("max_ctas", [0, 1, 13])
def test_pieces_of_long_branches(hq, hkv, chunk, lens, max_ctas):
    c = Cache(hq, hkv, chunk=chunk, lens=lens, seed=11)
    check(c, *run(c, max_ctas=max_ctas))
    check(c, *run(c, torch.float32, max_ctas=max_ctas))


def test_growing_scores_move_the_reference():
    """Scores that grow along the sequence: the running maximum moves in every tile and O is rescaled."""
    c = Cache(8, 2, chunk=[140, 1, 3], lens=[900, 1500, 1100], seed=2)
    c.q = (c.q.float().abs() + 0.1).bfloat16()
    for b, row in enumerate(c.rows):
        for i, page in enumerate(row):
            c.k[page] = (c.k[page].float().abs() * (0.02 * i)).bfloat16()
    c.k, c.v = c.k.nan_to_num(0.0), c.v
    # scores up to about 128 x 0.8 x 0.8 x 1.9 / 11.3 = 14 in magnitude: twice the error of the bound in the header
    check(c, *run(c), lse_tol=5e-4)


def test_rows_that_see_nothing_and_empty_branches():
    # branch 0: 30 new tokens but only 10 cached: its first 20 rows see nothing; branch 2 has no token at all
    c = Cache(8, 2, chunk=[30, 200, 0, 4, 1], lens=[10, 3, 0, 0, 1], seed=4, extra_blocks=2)
    out, lse = run(c)
    check(c, out, lse)
    assert (out[:20] == 0).all() and (lse[:20] == -math.inf).all() and torch.isfinite(lse[20:30]).all()


def test_nothing_visible_anywhere():
    c = Cache(5, 1, chunk=[3, 70], lens=[0, 0], seed=4, extra_blocks=1)
    out, lse = run(c)
    assert (out == 0).all() and (lse == -math.inf).all()
    c = Cache(5, 1, chunk=[0, 0], lens=[10, 20], seed=4, rows_behind=9)      # no branch brings a row
    out, lse = run(c)
    assert (out == 7).all() and (lse == 7).all()


def test_rows_before_and_behind_the_chunks_stay():
    c = Cache(16, 2, chunk=[5, 33], lens=[60, 33], seed=9, first_row=7, rows_behind=40)
    check(c, *run(c))


def test_strided_queries_of_a_fused_projection():
    c = Cache(16, 2, chunk=[5, 90, 1], lens=[60, 133, 300], seed=9)
    fused = torch.randn(c.total_rows, 16 + 4, 128, device="cuda").bfloat16()
    fused[:, :16] = c.q
    ctx = context(c)
    out, lse = torch.empty_like(c.q), torch.empty(c.total_rows, 16, device="cuda")
    call(ctx, c, out, lse, q=fused[:, :16])
    plain = torch.empty_like(out)
    call(ctx, c, plain)                                                     # without lse
    torch.cuda.synchronize()
    check(c, out, lse)
    assert torch.equal(out, plain)
    ctx.close()


def test_scale_of_the_context():
    c = Cache(8, 2, chunk=[40], lens=[300], seed=1)
    check(c, *run(c, softmax_scale=0.05), scale=0.05)


def test_same_results_every_time_and_on_another_stream():
    c = Cache(40, 8, chunk=[1, 300, 1], lens=[9000, 6011, 5000], seed=6)
    ctx = context(c)
    first, lse = run(c, ctx=ctx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.tts_set_stream(side)
    out = torch.empty_like(first)
    for _ in range(5):
        call(ctx, c, out)
        side.synchronize()
        assert torch.equal(out, first)
    ctx.close()


def test_captured_and_replayed_with_new_lengths():
    c = Cache(8, 2, chunk=[1, 64, 3], lens=[400, 500, 900], seed=8)
    ctx = context(c)
    out, lse = torch.zeros_like(c.q), torch.zeros(c.total_rows, c.hq, device="cuda")
    call(ctx, c, out, lse)
    side = torch.cuda.Stream()
    ctx.tts_set_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(ctx, c, out, lse)
    # shorter branches: the replay reads the lengths that the device holds then
    c.lens = [300, 64, 700]
    c.rows = [r[:-(-n // PAGE)] for r, n in zip(c.rows, c.lens)]
    c.branch_lens.copy_(torch.tensor(c.lens))
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(c, out, lse)
    assert ctx.tts_last_status() == 0
    ctx.close()


def test_agrees_with_the_verify_attention_of_the_same_rows():
    """Four rows per branch: what tts_verify_attn computes, within twice the rounding of either."""
    c = Cache(40, 8, chunk=[4] * 6, lens=[100, 4, 257, 900, 31, 64], prefix=128, seed=12, poison=False)
    ctx = tts.TtsContext(c.hq, c.hkv, c.n, 4, c.width, c.num_pages, out_dtype=tts.OUT_FP32)
    ctx.tts_chunk_reserve(c.total_rows)
    a, b = (torch.empty(c.total_rows, c.hq, 128, device="cuda") for _ in range(2))
    call(ctx, c, a)
    ctx.tts_verify_attn(c.q, c.k, c.v, c.table, c.prefix, c.branch_lens, c.n, 3, tts.MASK_CAUSAL, b)
    torch.cuda.synchronize()
    _, _, mean = chunk_attention(c)
    assert ((a - b).abs().double() <= 2 * (2.0 ** -8 + 2.0 ** -12) * mean).all()
    ctx.close()


def test_refusals():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    ctx = tts.TtsContext(8, 2, 2, 1, c.width, c.num_pages)
    out = torch.full_like(c.q, 3.0)

    def status(**kw):
        a = dict(q=c.q, stride=8 * 128, k=c.k, v=c.v, table=c.table, prefix=0, lens=c.branch_lens, starts=c.row_start, n=2, rows=7, out=out, lse=None) | kw
        try:
            ctx.tts_chunk_attn(a["q"], a["stride"], a["k"], a["v"], a["table"], a["prefix"], a["lens"], a["starts"], a["n"], a["rows"], a["out"], a["lse"])
        except tts.TtsError as e:
            return e.status
        return 0

    assert status() == -1                                     # nothing reserved yet
    with pytest.raises(tts.TtsError):
        ctx.tts_chunk_reserve(0)
    ctx.tts_chunk_reserve(7)
    ctx.tts_chunk_reserve(5)                                  # a smaller number is covered
    with pytest.raises(tts.TtsError):
        ctx.tts_chunk_reserve(8)
    bad = [dict(q=None), dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(starts=None), dict(out=None), dict(stride=8 * 128 - 8),
           dict(stride=8 * 128 + 4), dict(stride=0), dict(prefix=8), dict(prefix=-16), dict(prefix=16 * (c.width + 1)), dict(n=0), dict(n=3),
           dict(rows=8), dict(rows=-1), dict(q=c.q.data_ptr() + 2), dict(out=out.data_ptr() + 8), dict(k=c.k.data_ptr() + 4), dict(lens=c.branch_lens.data_ptr() + 1)]
    for kw in bad:
        assert status(**kw) == -1, kw
    assert status(rows=0) == 0                                # nothing to do
    torch.cuda.synchronize()
    assert (out == 3).all() and ctx.tts_last_status() == 0
    assert status() == 0
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    ctx.close()
    wide = tts.TtsContext(129, 1, 2, 1, 4, 4)
    with pytest.raises(tts.TtsError) as e:
        wide.tts_chunk_reserve(4)
    assert e.value.status == -2
    wide.close()


@pytest.mark.parametrize("starts,lens", [([0, 5, 3], [30, 40]), ([0, 3, 8], [30, 40]), ([-1, 3, 7], [30, 40]), ([0, 3, 7], [30, -1]), ([0, 3, 7], [1000, 40])])
def test_malformed_rows_or_lengths_compute_nothing(starts, lens):
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    ctx = context(c)
    out = torch.full_like(c.q, 3.0)
    call(ctx, c, out, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == -4 and (out == 3).all()
    out, lse = run(c, ctx=ctx)                               # the context works as before
    check(c, out, lse)
    ctx.close()


@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_pages_outside_the_pool_read_as_zeros(bad):
    c = Cache(8, 2, chunk=[40, 1], lens=[100, 200], seed=1, poison=False)
    ctx = context(c)
    table = c.table.clone()
    table[0, 2] = bad
    out, lse = torch.empty_like(c.q), torch.empty(c.total_rows, 8, device="cuda")
    call(ctx, c, out, lse, table=table)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == -4
    spare = next(p for p in range(c.num_pages) if all(p not in r for r in c.rows))
    c.rows[0][2] = spare
    c.k[spare], c.v[spare] = 0, 0
    check(c, out, lse)
    ctx.close()


def test_as_many_branches_as_a_context_takes():
    g = torch.Generator().manual_seed(1)
    chunk = torch.randint(0, 4, (1024,), generator=g).tolist()
    lens = [x + int(torch.randint(0, 40, (1,), generator=g)) for x in chunk]
    c = Cache(8, 2, chunk=chunk, lens=lens, seed=5)
    check(c, *run(c))


def test_more_row_blocks_than_are_cut_into_pieces():
    c = Cache(128, 1, chunk=[10] * 500, lens=[10 + i % 30 for i in range(500)], seed=5)      # 2500 blocks of two tokens
    check(c, *run(c))


def test_partial_results_that_would_not_fit_make_larger_pieces():
    """142 tokens of 128 heads over 12 700 keys: cut as fine as the balance asks for, the partial results of the 256-row
    pieces would exceed the workspace."""
    c = Cache(128, 1, chunk=[142], lens=[12842], seed=6, poison=False)
    check(c, *run(c))


def test_output_over_its_own_queries_is_refused():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    ctx = context(c)
    with pytest.raises(tts.TtsError) as e:
        call(ctx, c, c.q)
    assert e.value.status == -1
    ctx.close()


def test_two_graphs_of_one_context():
    """Captured calls share the context's workspace: replayed one after the other, each gives its own result."""
    a = Cache(8, 1, chunk=[1, 90], lens=[9000, 5000], seed=1)
    b = Cache(8, 1, chunk=[70, 3], lens=[8000, 100], seed=2)
    width, pages = max(a.width, b.width), max(a.num_pages, b.num_pages)
    for c in (a, b):
        c.table = torch.nn.functional.pad(c.table, (0, width - c.width), value=-1)
        pad = lambda x: torch.cat([x, torch.zeros(pages - c.num_pages, *x.shape[1:], dtype=x.dtype, device="cuda")])
        c.k, c.v = pad(c.k), pad(c.v)
    ctx = tts.TtsContext(8, 1, 2, 1, width, pages)
    ctx.tts_chunk_reserve(200)
    graphs, outs = [], []
    side = torch.cuda.Stream()
    ctx.tts_set_stream(side)
    for c in (a, b):
        out, lse = torch.zeros_like(c.q), torch.zeros(c.total_rows, 8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(ctx, c, out, lse)
        graphs.append(graph), outs.append((out, lse))
    for order in ([0, 1], [1, 0, 0], [1, 1, 0]):
        for out, lse in outs:
            out.zero_(), lse.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        check(a, *outs[0])
        check(b, *outs[1])
    assert ctx.tts_last_status() == 0
    ctx.close()


def test_lse_over_queries_or_output_is_refused():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    ctx = context(c)
    buffer = torch.full((c.total_rows * 8 * 128 * 2 + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
    out = buffer[:c.total_rows * 8 * 128]
    last = out.data_ptr() + out.numel() * 2
    for lse in (out.data_ptr(), last - 4, c.q.data_ptr() + 64, out.data_ptr() - c.total_rows * 8 * 4 + 4):
        with pytest.raises(tts.TtsError) as e:
            call(ctx, c, out, lse)
        assert e.value.status == -1
    torch.cuda.synchronize()
    assert (buffer == 3).all()
    call(ctx, c, out, last)                                      # next to it is fine
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0 and not (out == 3).all()
    ctx.close()


def test_tables_that_32_bit_token_numbers_do_not_reach_are_refused():
    """2^26 blocks of 16 tokens are 2^30 tokens; nothing is read before the refusal."""
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    out, refs = torch.zeros_like(c.q), torch.zeros(c.num_pages + 16, dtype=torch.int32, device="cuda")
    ctx = tts.TtsContext(8, 2, 2, 1, (1 << 26) + 1, c.num_pages)
    ctx.tts_chunk_reserve(7)
    with pytest.raises(tts.TtsError) as e:
        call(ctx, c, out)
    assert e.value.status == -1
    for grow in (lambda: ctx.tts_kv_grow(c.table, 0, c.branch_lens, c.row_start, 2, refs), lambda: ctx.tts_kv_free(c.table, c.branch_lens, c.row_start, 2, refs)):
        with pytest.raises(tts.TtsError) as e:
            grow()
        assert e.value.status == -1
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_output_aligned_to_16_bytes_only(dtype):
    """The same values to the bit as in an array that starts on a larger boundary, and nothing beside it."""
    c = Cache(8, 2, chunk=[1, 70, 9], lens=[300, 400, 20], seed=5)
    ctx = context(c, out_dtype=tts.OUT_FP32 if dtype == torch.float32 else tts.OUT_BF16)
    pad = 16 // dtype.itemsize
    want, buffer = torch.zeros(c.total_rows, 8, 128, dtype=dtype, device="cuda"), torch.full((c.total_rows * 8 * 128 + 2 * pad,), 3.0, dtype=dtype, device="cuda")
    assert buffer.data_ptr() % 32 == 0
    call(ctx, c, want)
    call(ctx, c, buffer[pad:])
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0 and (want != 0).any()
    assert torch.equal(buffer[pad:-pad].view_as(want), want)
    assert (buffer[:pad] == 3).all() and (buffer[-pad:] == 3).all()
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq", [1, 3, 5, 31, 33])
def test_tiles_that_a_warp_shares_with_no_query(hq, dtype):
    """Warps some of whose threads have a row of the result and some none: whole, joined from both sides, and cut."""
    c = Cache(hq, 1, chunk=[1, 2, 3, 7, 1, 1], lens=[9, 300, 3, 40, 20000, 129], seed=hq)
    check(c, *run(c, dtype))


def test_results_over_what_is_read_are_refused():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1, poison=False)
    ctx = context(c)
    out, lse = torch.zeros_like(c.q), torch.zeros(c.total_rows, c.hq, device="cuda")
    read = [c.k, c.v, c.table, c.branch_lens, c.row_start]
    before = [x.clone() for x in read]
    for x in read:
        first, last = x.data_ptr() // 16 * 16, (x.data_ptr() + x.numel() * x.element_size() - 1) // 16 * 16
        for at in (first, last, first - out.numel() * 2 + 16):
            for o, l in ((at, None), (out, at), (at, lse)):
                if at == first - out.numel() * 2 + 16 and l is at:
                    l = first - lse.numel() * 4 + 4
                with pytest.raises(tts.TtsError) as e:
                    call(ctx, c, o, l)
                assert e.value.status == -1
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, read)) and not out.any() and not lse.any() and ctx.tts_last_status() == 0
    ctx.close()


@pytest.mark.parametrize("branch", [0, 50, 99])
@pytest.mark.parametrize("what", ["start", "end", "short", "long"])
def test_malformed_rows_or_lengths_among_many_branches_compute_nothing(branch, what):
    """More entries than the schedule inside the attention kernel takes: the plan kernel's own look at them."""
    c = Cache(8, 2, chunk=[3] * 100, lens=[30] * 100, seed=1)
    ctx = context(c)
    out, lse = torch.full_like(c.q, 3.0), torch.full((c.total_rows, 8), 3.0, device="cuda")
    starts, lens = c.row_start.clone(), c.branch_lens.clone()
    if what == "start":
        starts[branch] = starts[branch + 1] + 1
    elif what == "end":
        starts[branch + 1] = c.total_rows + 1
    else:
        lens[branch] = -1 if what == "short" else 16 * c.width + 1
    call(ctx, c, out, lse, row_start=starts, lens=lens)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == -4 and (out == 3).all() and (lse == 3).all()
    check(c, *run(c, ctx=ctx))                               # the context works as before
    ctx.close()


def test_capture_and_replay_with_a_plan_kernel():
    """Two dependent launches in one graph; the replay goes by the lengths and rows that the device holds then."""
    n = 100
    c = Cache(8, 2, chunk=[1 + 7 * (i % 13) for i in range(n)], lens=[200 + 31 * (i % 40) for i in range(n)], seed=2)
    ctx = context(c)
    out, lse = torch.full_like(c.q, 7.0), torch.full((c.total_rows, 8), 7.0, device="cuda")
    side = torch.cuda.Stream()
    ctx.tts_set_stream(side)
    before = ctx.tts_launch_count()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(ctx, c, out, lse)
    assert ctx.tts_launch_count() - before == 2
    for lens, chunk in ((c.lens, c.chunk), ([100 + 7 * (i % 9) for i in range(n)], c.chunk), ([90] * n, [0 if i % 5 else 60 for i in range(n)]), (c.lens, [1] * n)):
        d = c
        d.lens, d.chunk, d.starts = list(lens), list(chunk), [0]
        for x in chunk:
            d.starts.append(d.starts[-1] + x)
        c.branch_lens.copy_(torch.tensor(lens)), c.row_start.copy_(torch.tensor(d.starts))
        full = c.rows
        c.rows = [r[:-(-x // PAGE)] for r, x in zip(full, lens)]
        for _ in range(2):
            out.fill_(7), lse.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            check(c, out, lse)
        c.rows = full
    assert ctx.tts_last_status() == 0
    ctx.close()


def test_uneven_branches_beyond_what_is_cut_into_pieces():
    """4100 blocks of rows, whole: one branch with 9000 keys behind branches of a few."""
    n = 1024
    c = Cache(128, 1, chunk=[8] * (n - 1) + [40], lens=[8 + i % 30 for i in range(n - 1)] + [9000], seed=5)
    check(c, *run(c))


def test_a_row_sees_every_key_below_it_where_most_branches_are_empty():
    c = Cache(8, 1, chunk=[0] * 500 + [33] + [0] * 499 + [1], lens=[0] * 500 + [5000] + [16] * 499 + [1], seed=6)
    check(c, *run(c))
