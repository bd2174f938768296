"""The memory of the attention over the 8-bit cache: that of the context's other attention calls, and there for a captured first call."""
import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from test_gpu_kv8 import attend, context

pytestmark = pytest.mark.gpu


def free():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("hq,hkv,branches,rows,most", [(8, 2, 4, 4, 34), (40, 8, 16, 60, 120)])
def test_contexts_hold_nothing_beside_the_verify_attentions_memory(hq, hkv, branches, rows, most):
    """MiB of a context: 32.6 and 110 of the verify attention's partial results and plans."""
    before = free()
    contexts = [context(hq, hkv, branches, rows, 64, 256) for _ in range(16)]
    assert (before - free()) / 16 <= most << 20
    for ctx in contexts:
        ctx.close()


@pytest.mark.parametrize("rows", [4, 14])
def test_both_attentions_of_one_context_in_turn(rows):
    """Long branches, cut into parts by either: what one leaves in the shared memory is nothing to the other, eager and replayed."""
    c = k8.Cache8(k8.E4M3, 2, [5000, 1200 + rows], prefix=64, seed=7, poison=False)
    k, v = (torch.zeros(c.num_pages, 2, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    every = torch.arange(c.num_pages, dtype=torch.int32, device="cuda")
    contexts = [context(8, 2, 2, rows, c.width, c.num_pages) for _ in range(3)]
    contexts[0].tts_kv8_read(c.fmt, c.pool, every, every, c.num_pages, k, v, c.num_pages)
    q = torch.randn(2 * rows, 8, 128, generator=torch.Generator().manual_seed(8)).bfloat16().cuda()

    def bf16(ctx, out):
        ctx.tts_verify_attn(q, k, v, c.table, c.prefix, c.branch_lens, 2, rows - 1, tts.MASK_CAUSAL, out)

    def kv8(ctx, out):
        ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, c.prefix, c.branch_lens, None, 2, rows, out, None)

    want, got = (torch.zeros(2, *q.shape, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    bf16(contexts[0], want[0])
    kv8(contexts[1], want[1])
    ctx = contexts[2]
    for _ in range(3):
        got.zero_()
        bf16(ctx, got[0])
        kv8(ctx, got[1])
        assert torch.equal(got, want)
    stream = torch.cuda.Stream()
    ctx.tts_set_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(2):
            kv8(ctx, got[1])
            bf16(ctx, got[0])
    for _ in range(3):
        got.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    assert all(x.tts_last_status() == 0 for x in contexts)


@pytest.mark.parametrize("rows", [4, 20])
@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_the_first_call_may_be_a_captured_one(rows, mode):
    c = k8.Cache8(k8.INT8, 2, [900, 70], prefix=16, seed=3)
    q, want, want_lse = attend(c, 8, rows, seed=4)
    ctx = context(8, 2, 2, rows, c.width, c.num_pages)
    stream = torch.cuda.Stream()
    ctx.tts_set_stream(stream)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream, capture_error_mode=mode):
        ctx.tts_kv8_attn(c.fmt, q, q.stride(0), c.pool, c.table, c.prefix, c.branch_lens, None, 2, rows, out, lse)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert ctx.tts_last_status() == 0
