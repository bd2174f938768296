"""Beam selection and reordering on the GPU, against plain implementations in 64 bits and whole numbers."""
import math
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pick(logits, scores, groups, beams, k, finished=None, pad=0, ctx=None, stride=None):
    vocab = logits.shape[1]
    own = ctx is None
    if own:
        ctx = tts.TtsContext(1, 1, groups * beams, 1, 1, 1)
        ctx.tts_beam_reserve(groups * beams, k)
    parents, tokens = (torch.full((groups, k), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    got = torch.full((groups, k), math.nan, device="cuda")
    ctx.tts_beam_select(logits, 0 if logits.dtype == torch.bfloat16 else 1, stride or logits.stride(0), vocab, scores, finished, pad, groups, beams, k,
                        parents, tokens, got)
    return parents, tokens, got


def check(logits, scores, groups, beams, k, finished=None, pad=0, **more):
    """Parents and tokens as the definition has them; scores within a rounding to fp32 and the exponentials' 2^-22.  Where two
    neighbours of the definition's order lie closer than that they may change places."""
    parents, tokens, got = pick(logits, scores, groups, beams, k, finished, pad, **more)
    want = k8.select(logits, scores, finished, pad, groups, beams, k)
    for g in range(groups):
        for i, (parent, token, score) in enumerate(want[g]):
            near = [w for w in want[g] if abs(w[2] - score) < 1e-6 and w[2] != score] if score > -math.inf else []
            if not near:
                assert (parents[g, i].item(), tokens[g, i].item()) == (parent, token), (g, i)
            if score == -math.inf:
                assert got[g, i].item() == -math.inf
            else:
                assert abs(got[g, i].item() - score) <= abs(score) * 2.0 ** -23 + 2.0 ** -21


def normal(rows, vocab, dtype, seed=0, scale=3.0):
    return (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def starts(rows, seed=1):
    return (-8 * torch.rand(rows, generator=torch.Generator().manual_seed(seed)) - 1).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("groups,beams,k,vocab", [(1, 1, 1, 1), (1, 4, 4, 1024), (3, 2, 5, 50257), (2, 5, 128, 300), (2, 16, 16, 32000), (1, 64, 64, 8192), (1, 1, 128, 9000),
                                                  (5, 3, 2, 7), (1, 2, 3, 151936), (40, 2, 2, 8200)])
def test_selection(dtype, groups, beams, k, vocab):
    rows = groups * beams
    check(normal(rows, vocab, dtype, vocab), starts(rows), groups, beams, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stride,offset", [(1003, 0), (1001, 3), (1008, 1), (1008, 8)])
def test_rows_of_any_alignment(dtype, stride, offset):
    x = normal(6, stride, dtype, 2)[:, offset:] if offset else normal(6, stride, dtype, 2)
    check(x[:, :999], starts(6), 2, 3, 7)


@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two values", "late peak", "equal but one"])
@pytest.mark.parametrize("k", [1, 16, 128])
def test_logits_in_awkward_orders(kind, k):
    """Ties go to the lowest beam, then the lowest token, in rows longer than a chunk of the kernel and cut between its CTAs."""
    vocab, rows = 40007, 4
    t = torch.arange(vocab, dtype=torch.float32)
    one = {"equal": torch.zeros(vocab), "rising": t / 4096, "falling": -t / 4096, "two values": (t % 97 == 5).float(),
           "late peak": torch.where(t >= vocab - 200, 3 + t / vocab, -1.0), "equal but one": torch.where(t == vocab - 1, 2.0, 0.0)}[kind]
    x = one.repeat(rows, 1).cuda()
    check(x, torch.full((rows,), -2.0, device="cuda"), 1, rows, k)         # equal rows too: equal scores across beams
    check(x, torch.tensor([-2.0, -1.0, -2.5, -1.0], device="cuda"), 2, 2, k)


@pytest.mark.parametrize("groups,beams,k,vocab", [(1, 64, 64, 40000), (2, 16, 64, 32768), (1, 64, 128, 33000)])
def test_questions_whose_parts_leave_thousands_of_candidates(groups, beams, k, vocab):
    check(normal(groups * beams, vocab, torch.float32, vocab + k), starts(groups * beams), groups, beams, k)


def test_more_candidates_than_a_block_compares_at_once_with_ties():
    """64 beams of 128 candidates, many scores equal: the last places go to the lowest beams and tokens."""
    x = torch.zeros(64, 500)
    x[:, 100:130] = 1.0
    check(x.cuda(), torch.full((64,), -3.0, device="cuda"), 1, 64, 128)
    check(x.cuda(), (torch.arange(64) % 4).neg().float().cuda(), 1, 64, 128)


def test_finished_and_dead_beams_and_too_few_candidates():
    x = normal(6, 5, torch.float32, 4)
    x[1, 1:] = -math.inf                                            # one candidate
    x[2] = -math.inf                                                # none
    x[4, 3] = math.nan
    scores = torch.tensor([-1.0, -2.0, -1.0, -math.inf, -1.0, -0.25], device="cuda")
    finished = ints([0, 0, 0, 1, 0, 7])
    check(x, scores, 2, 3, 12, finished, pad=4)
    parents, tokens, got = pick(x, scores, 2, 3, 12, finished, pad=4)
    assert parents[1].tolist() == [5] + [-1] * 11 and tokens[1, 0].item() == 4 and got[1, 0].item() == -0.25
    assert (parents[0] >= 0).sum() == 6
    x[4, 3] = math.inf
    assert pick(x, scores, 2, 3, 12, finished, pad=4)[0][1].tolist() == [5] + [-1] * 11
    every = torch.full((6,), math.nan, device="cuda")
    parents, tokens, got = pick(x, every, 2, 3, 4)
    assert (parents == -1).all() and (tokens == -1).all() and (got == -math.inf).all()


def test_first_step_of_a_search_and_large_values():
    """Only beam 0 is there at first; logits far from zero and far apart."""
    x = normal(8, 30000, torch.float32, 5, scale=300.0) + 1e4
    scores = torch.full((8,), -math.inf, device="cuda")
    scores[[0, 4]] = 0.0
    check(x, scores, 2, 4, 4)


def test_selection_repeats_itself_and_replays():
    ctx = tts.TtsContext(1, 1, 32, 1, 1, 1)
    ctx.tts_beam_reserve(32, 8)
    ctx.tts_beam_reserve(4, 2)                                      # less is there already
    x, scores = normal(32, 20000, torch.bfloat16, 6), starts(32)
    first = pick(x, scores, 4, 8, 8, ctx=ctx)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(first, pick(x, scores, 4, 8, 8, ctx=ctx)))
    stream = torch.cuda.Stream()
    ctx.tts_set_stream(stream)
    out = [torch.empty_like(t) for t in first]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ctx.tts_beam_select(x, 0, 20000, 20000, scores, None, 0, 4, 8, 8, *out)
    x.copy_(normal(32, 20000, torch.bfloat16, 7))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    ctx.tts_set_stream(None)
    assert all(torch.equal(a, b) for a, b in zip(out, pick(x, scores, 4, 8, 8, ctx=ctx)))


# ----------------------------------------------------------------------------------------------- reorder
@pytest.mark.parametrize("sizes", [[1], [16, 3, 4, 33000, 12, 7], [40000 * 16], [2048 * 4 + 4, 2049], list(range(1, 129))])
@pytest.mark.parametrize("n,children", [(1, 1), (5, 9), (16, 3)])
def test_reorder(sizes, n, children):
    gen = torch.Generator().manual_seed(len(sizes))
    src = [torch.randint(0, 256, (n, b), generator=gen, dtype=torch.uint8).cuda() for b in sizes]
    dst = [torch.randint(0, 256, (children, b), generator=gen, dtype=torch.uint8).cuda() for b in sizes]
    r = random.Random(n)
    parents = [r.randrange(-1, n) for _ in range(children)]
    parents[0] = n - 1
    want = [torch.stack([a[p] if p >= 0 else b[i] for i, p in enumerate(parents)]) for a, b in zip(src, dst)]
    ctx = tts.TtsContext(1, 1, 1, 1, 1, 1)
    ctx.tts_beam_reorder(tts.TtsStates(src, dst, sizes), ints(parents), n, children)
    assert all(torch.equal(a, b) for a, b in zip(dst, want)) and ctx.tts_last_status() == 0


@pytest.mark.parametrize("off", [1, 4, 8])
def test_reorder_of_rows_off_their_alignment(off):
    src, dst = torch.arange(16 * 7 + 16, dtype=torch.uint8, device="cuda"), torch.zeros(200, dtype=torch.uint8, device="cuda")
    ctx = tts.TtsContext(1, 1, 1, 1, 1, 1)
    ctx.tts_beam_reorder(tts.TtsStates([src.data_ptr() + off], [dst.data_ptr() + 16], [16]), ints([6, 0]), 7, 2)
    assert torch.equal(dst[16:48].view(2, 16), src[off:off + 112].view(7, 16)[[6, 0]]) and not dst[48:].any() and not dst[:16].any()


@pytest.mark.parametrize("bytes_", [1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 500, 32767, 32769, 65541])
def test_reorder_of_rows_at_every_shift(bytes_):
    """Rows of src and dst that start at all pairs of places within 16 bytes; nothing beside them changes."""
    gen = torch.Generator().manual_seed(bytes_)
    src, dst = [], []
    for shift in range(16):
        src.append(torch.randint(0, 256, (4 * bytes_ + 16,), generator=gen, dtype=torch.uint8).cuda())
        dst.append(torch.randint(0, 256, (3 * bytes_ + 32,), generator=gen, dtype=torch.uint8).cuda())
    parents, want = [3, 0, 2], [x.clone() for x in dst]
    for shift in range(16):
        for i, p in enumerate(parents):
            want[shift][(7 * shift) % 16 + i * bytes_:][:bytes_] = src[shift][shift + p * bytes_:][:bytes_]
    ctx = tts.TtsContext(1, 1, 1, 1, 1, 1)
    states = tts.TtsStates([x.data_ptr() + i for i, x in enumerate(src)], [x.data_ptr() + 7 * i % 16 for i, x in enumerate(dst)], [bytes_] * 16)
    ctx.tts_beam_reorder(states, ints(parents), 4, 3)
    assert all(torch.equal(a, b) for a, b in zip(dst, want)) and ctx.tts_last_status() == 0


def test_reorder_reports_parents_outside():
    src, dst = torch.ones(3, 32, dtype=torch.uint8, device="cuda"), torch.zeros(3, 32, dtype=torch.uint8, device="cuda")
    ctx = tts.TtsContext(1, 1, 1, 1, 1, 1)
    ctx.tts_beam_reorder(tts.TtsStates([src], [dst], [32]), ints([3, -2, 1]), 3, 3)
    assert ctx.tts_last_status() == -4 and not dst[:2].any() and dst[2].all()


def test_refusals():
    ctx = tts.TtsContext(1, 1, 8, 1, 1, 1)
    x, scores = normal(8, 64, torch.bfloat16), starts(8)
    parents, tokens, out = (torch.zeros(2, 4, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32))
    good = [x, 0, 64, 64, scores, None, 0, 2, 4, 4, parents, tokens, out]

    def refused(status, call, *args):
        with pytest.raises(tts.TtsError) as e:
            call(*args)
        assert e.value.status == status

    refused(-1, ctx.tts_beam_select, *good)                         # nothing reserved
    for rows, k, status in ((0, 1, -1), (9, 1, -1), (8, 0, -1), (8, 129, -2)):
        refused(status, ctx.tts_beam_reserve, rows, k)
    ctx.tts_beam_reserve(8, 4)
    refused(-1, ctx.tts_beam_reserve, 8, 5)
    ctx.tts_beam_select(*good)
    done = ints([0] * 8)
    for at, value, status in ((0, None, -1), (0, x.data_ptr() + 1, -1), (1, 2, -2), (2, 63, -1), (3, 0, -1), (3, 1 << 29, -2), (4, None, -1), (7, 0, -1), (7, 3, -1),
                              (8, 5, -1), (9, 5, -1), (9, 0, -1), (10, None, -1), (10, tokens, -1), (11, out, -1), (12, scores, -1), (12, x, -1)):
        args = [value if i == at else a for i, a in enumerate(good)]
        refused(status, ctx.tts_beam_select, *args)
    for pad in (-1, 64):
        refused(-1, ctx.tts_beam_select, *[done if i == 5 else pad if i == 6 else a for i, a in enumerate(good)])
    a, b = (torch.zeros(4, 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    order = ints([0, 1])
    call = lambda s, d, n, p=order, rows=4, children=2: ctx.tts_beam_reorder(tts.TtsStates(s, d, n), p, rows, children)  # noqa: E731
    call([a], [b], [32])
    call([a, a], [b, b.data_ptr() + 64], [32, 32])                  # one array read twice
    for args in (([a], [a], [32]), ([a], [a.data_ptr() + 96], [32]), ([a, a], [b, b.data_ptr() + 32], [32, 32]), ([a], [None], [32]), ([a], [b], [0]), ([], [], []),
                 ([a] * 129, [b.data_ptr() + i for i in range(129)], [1] * 129), ([a], [order], [4])):
        refused(-1, call, *args)
    refused(-1, call, [a], [b], [32], None)
    refused(-1, call, [a], [b], [32], order, 0)
    refused(-1, call, [a], [b], [32], order, 4, 0)
    assert ctx.tts_last_status() == 0
