"""Rotary positions on the way into the cache (tts_kv_append_rope) against a plain implementation in 64 bits.

Tolerance: a rotated element is a cos - b sin in fp32 from sines and cosines good to 2^-22, rounded once to bf16:
half a step of the result (2^-8 of it) and at most 2^-20 of |a| + |b|."""
import pytest
import torch

import paper_2505_19634_b200 as tts
from cache_plain import PAGE, Cache, rope_turn

pytestmark = pytest.mark.gpu


def inv_freq(n, base=1e6):
    return [base ** (-i / n) for i in range(n)]


def inputs(c: Cache, n_axes, seed=0, far=1 << 20):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.randn(c.total_rows, c.hkv, 128, generator=g, device="cuda").bfloat16()
    v = torch.randn(c.total_rows, c.hkv, 128, generator=g, device="cuda").bfloat16()
    pos = torch.randint(-far, far, (n_axes, c.total_rows), generator=g, device="cuda", dtype=torch.int32)
    return k, v, pos


def close(got, want, parts):
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -20 * parts
    assert ((got.double() - want).abs() <= bound).all(), ((got.double() - want).abs() - bound).max()


def magnitude(x, n, interleaved):
    """|a| + |b| of each dim's pair."""
    x = x.double().abs()
    out = x.clone()
    for i in range(n):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        out[..., lo] = out[..., hi] = x[..., lo] + x[..., hi]
    return out


def places(c: Cache, b):
    """(page, slot) of each row of branch b's chunk."""
    first = c.prefix + c.lens[b] - c.chunk[b]
    return [(c.rows[b][(first + i) // PAGE], (first + i) % PAGE) for i in range(c.chunk[b])]


def check(c, rope_args, k0, v0, k, v, pos, q_out, k_new, v_new, skip=()):
    axis, freq, inter = rope_args
    n = len(freq)
    rows = slice(c.starts[0], c.starts[-1])
    close(q_out[rows], rope_turn(c.q, pos, axis, freq, inter)[rows], magnitude(c.q, n, inter)[rows])
    assert torch.equal(q_out[rows][..., 2 * n:], c.q[rows][..., 2 * n:])
    turned, parts = rope_turn(k_new, pos, axis, freq, inter), magnitude(k_new, n, inter)
    want_k, want_v = k0.clone(), v0.clone()
    for b in range(c.n):
        if b in skip:
            continue
        for i, (page, slot) in enumerate(places(c, b)):
            r = c.starts[b] + i
            close(k[page, :, slot], turned[r], parts[r])
            assert torch.equal(v[page, :, slot], v_new[r])
            want_k[page, :, slot], want_v[page, :, slot] = k[page, :, slot], v_new[r]
    bits = lambda t: t.view(torch.int16)
    assert torch.equal(bits(k), bits(want_k)) and torch.equal(bits(v), bits(want_v))      # every other slot as it was


def run(c, axis, freq, inter, seed=0, inplace=False, fused=False, n_axes=None):
    k_new, v_new, pos = inputs(c, n_axes or max(axis) + 1, seed)
    ctx = tts.TtsContext(c.hq, c.hkv, c.n, 1, c.width, c.num_pages)
    k0, v0 = c.k.clone(), c.v.clone()
    q = c.q.clone()
    if fused:
        qkv = torch.cat([c.q[:c.total_rows], k_new, v_new], 1)
        q, kk, vv = qkv[:, :c.hq], qkv[:, c.hq:c.hq + c.hkv], qkv[:, c.hq + c.hkv:]
    else:
        kk, vv = k_new, v_new
    q_out = q if inplace else torch.full((c.total_rows, c.hq, 128), 7.0, device="cuda").bfloat16()
    ctx.tts_kv_append_rope(tts.TtsRope(axis, freq, inter), q, q.stride(0), kk, vv, kk.stride(0), pos, c.k, c.v, c.table, c.prefix,
                           c.branch_lens, c.row_start, c.n, c.total_rows, q_out)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    check(c, (axis, freq, inter), k0, v0, c.k, c.v, pos, q_out, k_new, v_new)
    ctx.close()
    return q_out


@pytest.mark.parametrize("pairs", [64, 32, 48, 20, 1, 63, 8])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (5, 1)])
def test_pairs_layouts_and_axes(pairs, inter, hq, hkv):
    c = Cache(hq, hkv, chunk=[1, 37, 0, 18], lens=[20, 37, 5, 333], prefix=32, seed=pairs)
    axis = [i % 3 for i in range(pairs)]
    run(c, axis, inv_freq(pairs), inter, n_axes=3)


def test_sections_of_contiguous_pairs_and_four_axes():
    c = Cache(16, 2, chunk=[50, 3], lens=[50, 100], seed=1)
    run(c, [0] * 16 + [1] * 24 + [2] * 12 + [3] * 12, inv_freq(64), False)


@pytest.mark.parametrize("pairs,inter", [(64, False), (20, False), (64, True)])
def test_in_place_and_fused_projection(pairs, inter):
    for kw in (dict(inplace=True), dict(fused=True)):
        c = Cache(40, 8, chunk=[4] * 5, lens=[4, 17, 33, 50, 64], prefix=16, seed=7)
        run(c, [0] * pairs, inv_freq(pairs), inter, **kw)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 65, 300, 1024])
def test_many_branches(n):
    g = torch.Generator().manual_seed(n)
    chunk = torch.randint(0, 4, (n,), generator=g).tolist()
    chunk[0] = 1
    c = Cache(4, 1, chunk=chunk, lens=[x + 9 for x in chunk], seed=n, poison=False)
    run(c, [0] * 64, inv_freq(64), False)


def test_rows_of_no_branch_stay():
    c = Cache(8, 2, chunk=[3, 9], lens=[30, 9], seed=3, first_row=5, rows_behind=11)
    q_out = run(c, [0] * 64, inv_freq(64), False)
    assert (q_out[:5] == 7).all() and (q_out[c.starts[-1]:] == 7).all()


def test_enough_rows_that_a_warp_walks_a_whole_row():
    c = Cache(6, 1, chunk=[9000, 800], lens=[9000, 1200], seed=3, poison=False)
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(6, 1, 2, 1, c.width, c.num_pages)
    q_out = torch.empty_like(c.q)
    ctx.tts_kv_append_rope(tts.TtsRope([0] * 64, inv_freq(64)), c.q, 6 * 128, k_new, v_new, 128, pos, c.k, c.v, c.table, 0, c.branch_lens,
                           c.row_start, 2, c.total_rows, q_out)
    torch.cuda.synchronize()
    close(q_out, rope_turn(c.q, pos, [0] * 64, inv_freq(64), False), magnitude(c.q, 64, False))
    turned, parts = rope_turn(k_new, pos, [0] * 64, inv_freq(64), False), magnitude(k_new, 64, False)
    for b in range(2):
        at = torch.tensor(places(c, b), device="cuda")
        rows = slice(c.starts[b], c.starts[b + 1])
        close(c.k[at[:, 0], :, at[:, 1]], turned[rows], parts[rows])
        assert torch.equal(c.v[at[:, 0], :, at[:, 1]], v_new[rows])
    ctx.close()


def test_pools_beyond_32_bit_offsets():
    pages = 70000                                            # x 8 heads x 4 KiB: 2.3 GB, byte offsets past 2^31
    c = Cache(8, 8, chunk=[20], lens=[40], seed=3, num_pages=2 * pages)
    c.k = torch.zeros(c.num_pages, 8, 16, 128, dtype=torch.bfloat16, device="cuda")
    c.v = torch.zeros_like(c.k)
    c.width = c.table.shape[1]
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(8, 8, 1, 1, c.width, c.num_pages)
    q_out = torch.empty_like(c.q)
    ctx.tts_kv_append_rope(tts.TtsRope([0] * 64, inv_freq(64)), c.q, 1024, k_new, v_new, 1024, pos, c.k, c.v, c.table, 0, c.branch_lens,
                           c.row_start, 1, 20, q_out)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    for i, (page, slot) in enumerate(places(c, 0)):
        assert page > pages and torch.equal(c.v[page, :, slot], v_new[i])
    ctx.close()


def test_refusals():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(8, 2, 2, 1, c.width, c.num_pages)
    q_out = torch.full_like(c.q, 3.0)
    k0 = c.k.clone()
    good = tts.TtsRope([0] * 64, inv_freq(64))

    def status(**kw):
        a = dict(rope=good, q=c.q, qs=1024, k=k_new, v=v_new, ks=256, pos=pos, kp=c.k, vp=c.v, table=c.table, prefix=0, lens=c.branch_lens,
                 starts=c.row_start, n=2, rows=7, out=q_out) | kw
        try:
            ctx.tts_kv_append_rope(a["rope"], a["q"], a["qs"], a["k"], a["v"], a["ks"], a["pos"], a["kp"], a["vp"], a["table"], a["prefix"],
                                   a["lens"], a["starts"], a["n"], a["rows"], a["out"])
        except tts.TtsError as e:
            return e.status
        return 0

    far_axis, nan_freq, no_pairs = (tts.TtsRope([0] * 64, inv_freq(64)) for _ in range(3))
    far_axis.axis[3] = 1
    nan_freq.inv_freq[3] = float("nan")
    no_pairs.n_pairs = 0
    for kw in [dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(kp=None), dict(vp=None), dict(table=None), dict(lens=None), dict(starts=None),
               dict(out=None), dict(qs=1016), dict(qs=1028), dict(ks=248), dict(ks=260), dict(prefix=8), dict(n=0), dict(n=3), dict(rows=-1),
               dict(rope=far_axis), dict(rope=nan_freq), dict(rope=no_pairs), dict(out=c.q.data_ptr() + 256), dict(q=c.q.data_ptr() + 2),
               dict(out=c.q, qs=2048)]:
        assert status(**kw) == -1, kw
    assert status(rows=0) == 0
    torch.cuda.synchronize()
    assert (q_out == 3).all() and torch.equal(c.k.view(torch.int16), k0.view(torch.int16)) and ctx.tts_last_status() == 0
    ctx.close()


def test_bad_places_write_no_key_and_are_reported():
    c = Cache(8, 2, chunk=[3, 4, 5], lens=[30, 40, 50], seed=1, poison=False)
    k_new, v_new, pos = inputs(c, 1)
    freq = inv_freq(64)
    for case in ("short", "page", "table"):
        ctx = tts.TtsContext(8, 2, 3, 1, c.width, c.num_pages)
        k, v, table, lens = c.k.clone(), c.v.clone(), c.table.clone(), c.branch_lens.clone()
        if case == "short":
            lens[1] = 3                                      # a chunk of 4
        elif case == "page":
            table[1, 2] = c.num_pages
        else:
            lens[1] = 16 * c.width + 4
        q_out = torch.empty_like(c.q)
        ctx.tts_kv_append_rope(tts.TtsRope([0] * 64, freq), c.q, 1024, k_new, v_new, 256, pos, k, v, table, 0, lens, c.row_start, 3, 12, q_out)
        torch.cuda.synchronize()
        assert ctx.tts_last_status() == -4
        check(c, ([0] * 64, freq, False), c.k, c.v, k, v, pos, q_out, k_new, v_new, skip=(1,))
        ctx.close()


def test_rotated_queries_over_the_new_keys_or_values_are_refused():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1)
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(8, 2, 2, 1, c.width, c.num_pages)
    rope, before = tts.TtsRope([0] * 64, inv_freq(64)), (k_new.clone(), v_new.clone())
    for out in (k_new.data_ptr(), v_new.data_ptr() + v_new.numel() * 2 - 16, k_new.data_ptr() - 7 * 1024 * 2 + 16):
        with pytest.raises(tts.TtsError) as e:
            ctx.tts_kv_append_rope(rope, c.q, 1024, k_new, v_new, 256, pos, c.k, c.v, c.table, 0, c.branch_lens, c.row_start, 2, 7, out)
        assert e.value.status == -1
    torch.cuda.synchronize()
    assert torch.equal(k_new, before[0]) and torch.equal(v_new, before[1])
    ctx.close()


@pytest.mark.parametrize("n", [4, 32, 33, 100])
@pytest.mark.parametrize("kind", ["swapped", "swapped_last", "negative", "behind"])
@pytest.mark.parametrize("pairs,inter", [(64, False), (20, False), (64, True)])
def test_malformed_rows_write_nothing(n, kind, pairs, inter):
    """Among them the starts 0, 9, 10, 1: row 3 would be found in the branch of rows 9 .. 9 and its key belong 6 tokens before
    that branch's first."""
    c = Cache(4, 1, chunk=[3] * n, lens=[3] * n, seed=n, spare=0, poison=False)
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(4, 1, n, 1, c.width, c.num_pages)
    starts = c.row_start.clone()
    if kind == "swapped":
        starts[:4] = torch.tensor([0, 9, 10, 1])
    elif kind == "swapped_last":
        starts[n - 1] = starts[n] + 1
    elif kind == "negative":
        starts[0] = -2 ** 31
    else:
        starts[n] = c.total_rows + 1
    k0, v0, q_out, rope = c.k.clone(), c.v.clone(), torch.full_like(c.q, 7.0), tts.TtsRope([0] * pairs, inv_freq(pairs), inter)
    ctx.tts_kv_append_rope(rope, c.q, 512, k_new, v_new, 128, pos, c.k, c.v, c.table, 0, c.branch_lens, starts, n, c.total_rows, q_out)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == -4
    assert (q_out == 7).all() and torch.equal(c.k, k0) and torch.equal(c.v, v0)
    ctx.tts_kv_append_rope(rope, c.q, 512, k_new, v_new, 128, pos, c.k, c.v, c.table, 0, c.branch_lens, c.row_start, n, c.total_rows, q_out)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    check(c, ([0] * pairs, inv_freq(pairs), inter), k0, v0, c.k, c.v, pos, q_out, k_new, v_new)
    ctx.close()


def test_what_is_written_over_what_is_read_is_refused():
    c = Cache(8, 2, chunk=[3, 4], lens=[30, 40], seed=1, poison=False)
    k_new, v_new, pos = inputs(c, 1)
    ctx = tts.TtsContext(8, 2, 2, 1, c.width, c.num_pages)
    a = dict(rope=tts.TtsRope([0] * 64, inv_freq(64)), q=c.q, qs=1024, k=k_new, v=v_new, ks=256, pos=pos, kp=c.k, vp=c.v, table=c.table, prefix=0,
             lens=c.branch_lens, starts=c.row_start, n=2, rows=7, out=torch.zeros_like(c.q))
    arrays = {k: x for k, x in a.items() if isinstance(x, torch.Tensor)}
    before = {k: x.clone() for k, x in arrays.items()}
    for w in ("out", "kp", "vp"):
        for other, x in arrays.items():
            if other == w:
                continue
            for at in (x.data_ptr() // 16 * 16, (x.data_ptr() + x.numel() * x.element_size() - 1) // 16 * 16):
                if (w, other) == ("out", "q") and at == x.data_ptr():
                    continue                                 # in place
                with pytest.raises(tts.TtsError) as e:
                    ctx.tts_kv_append_rope(*(a | {w: at}).values())
                assert e.value.status == -1, (w, other)
    torch.cuda.synchronize()
    assert all(torch.equal(before[k], x) for k, x in arrays.items()) and ctx.tts_last_status() == 0
    ctx.tts_kv_append_rope(*a.values())
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    ctx.close()
