"""What tts_last_status reports when several of the cache operators' calls went wrong, and that the context works
afterwards."""
import pytest
import torch

import paper_2505_19634_b200 as tts
from cache_plain import Cache
from test_gpu_chunk_attention import call, check, context

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("chunk,lens", [([1, 90, 700], [9000, 5000, 700]), ([3, 1, 40, 200] * 25, [700, 3000, 40, 900] * 25)])
def test_too_few_pages_do_not_hide_a_wait_that_ran_out(chunk, lens):
    """A call that gave up leaves the schedule's counters in disorder, and the next call's rows unwritten if nothing sets
    them right.  Both schedules: made inside the attention kernel, and by a kernel of its own."""
    c = Cache(8, 1, chunk=chunk, lens=lens, seed=1)
    ctx = context(c)
    table, count, refs = torch.full((1, c.width), -1, dtype=torch.int32, device="cuda"), i32([0]), torch.ones(c.num_pages, dtype=torch.int32, device="cuda")
    for order in ("timeout first", "pages first"):
        if order == "timeout first":
            ctx.tts_debug_wait_timeout(1_000_000)
        ctx.tts_kv_grow(table, 0, count, i32([16]), 1, refs)             # no page is free
        if order == "pages first":
            ctx.tts_debug_wait_timeout(1_000_000)
        assert [ctx.tts_last_status() for _ in range(3)] == [-5, -7, 0]
        out, lse = torch.zeros_like(c.q), torch.zeros(c.total_rows, c.hq, device="cuda")
        for _ in range(2):
            call(ctx, c, out, lse)
        torch.cuda.synchronize()
        assert ctx.tts_last_status() == 0
        check(c, out, lse)
    ctx.close()


def test_bad_values_and_too_few_pages_are_both_reported():
    ctx = tts.TtsContext(2, 1, 1, 1, 4, 8)
    table, refs = i32([[-1] * 4]), i32([1] * 8)
    ctx.tts_kv_grow(table, 0, i32([0]), i32([16]), 1, refs)
    ctx.tts_kv_grow(table, 0, i32([0]), i32([-1]), 1, refs)
    assert [ctx.tts_last_status() for _ in range(3)] == [-4, -7, 0]
    ctx.close()
