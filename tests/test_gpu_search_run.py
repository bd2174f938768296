"""A beam search on the 8-bit cache as it is used: prompts, forks by the selection's parents, single tokens, drafted chains cut back, draft
trees, finished beams, the pool closed up, on a stream of its own.  After every step the attention over the cache is compared with
attention in 64 bits over each branch's own list of tokens, which knows nothing of pages, and the selection with its definition."""
import random

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts

pytestmark = pytest.mark.gpu

HQ, HKV, WIDTH, PAGES, QUESTIONS, BEAMS, LAYERS, VOCAB, STEPS = 8, 1, 12, 90, 2, 3, 2, 1003, 24
N = QUESTIONS * BEAMS


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Branches:
    """One layer's branches as lists of (K, V) values, with what k8.attention asks of a cache."""

    def __init__(self):
        self.n, self.prefix, self.hkv, self.tokens = N, 0, HKV, [[] for _ in range(N)]

    @property
    def lens(self):
        return [len(x) for x in self.tokens]

    def kv(self, b):
        return tuple(torch.stack([t[j] for t in self.tokens[b]], 1) for j in range(2))


class Search:
    def __init__(self, fmt):
        self.fmt, self.gen, self.r = fmt, torch.Generator(device="cuda").manual_seed(fmt), random.Random(fmt)
        self.ctx = tts.TtsContext(HQ, HKV, N, 16, WIDTH, PAGES)
        self.ctx.tts_set_stream(torch.cuda.current_stream())
        self.ctx.tts_beam_reserve(N, BEAMS)
        self.records = [torch.full((PAGES, HKV, k8.RECORD), 127, dtype=torch.uint8, device="cuda") for _ in range(LAYERS)]
        self.pools = tts.TtsKv8Pools(self.records)
        self.table, self.lens, self.refs = i32([[-1] * WIDTH] * N), i32([0] * N), i32([0] * PAGES)
        self.books = [Branches() for _ in range(LAYERS)]
        self.scores, self.finished = torch.zeros(N, device="cuda"), i32([0] * N)
        self.history, self.hidden = i32([[-1] * STEPS] * N), torch.zeros(N, 5, device="cuda", dtype=torch.bfloat16)
        self.texts = [[] for _ in range(N)]

    def append(self, chunk):
        starts = [0]
        for c in chunk:
            starts.append(starts[-1] + c)
        self.ctx.tts_kv_grow(self.table, 0, self.lens, i32(chunk), N, self.refs)
        for records, book in zip(self.records, self.books):
            kv = torch.randn(starts[-1], 2, HKV, 128, generator=self.gen, device="cuda").bfloat16()
            self.ctx.tts_kv8_append(self.fmt, None, None, 0, kv[:, 0], kv[:, 1], kv.stride(0), None, records, self.table, 0, self.lens, i32(starts), N,
                                    starts[-1], None)
            scale = k8.scales(kv.float(), self.fmt)
            value = k8.table(self.fmt, "cuda")[k8.codes(kv.float(), scale, self.fmt).long()] * scale.double()[..., None]
            for b, c in enumerate(chunk):
                book.tokens[b] += [(value[starts[b] + i, 0], value[starts[b] + i, 1]) for i in range(c)]

    def attend(self, rows, parents=None):
        for records, book in zip(self.records, self.books):
            q = torch.randn(N * rows, HQ, 128, generator=self.gen, device="cuda").bfloat16()
            out, lse = torch.empty_like(q), torch.empty(N * rows, HQ, device="cuda")
            self.ctx.tts_kv8_attn(self.fmt, q, HQ * 128, records, self.table, 0, self.lens, None if parents is None else i32(parents), N, rows, out, lse)
            k8.assert_attention(book, q, rows, out, lse, parents=parents)
        self.hidden = out[::rows, 0, :5].contiguous()

    def fork(self, parents, device_parents=None):
        table, lens, refs = torch.empty_like(self.table), torch.empty_like(self.lens), torch.empty_like(self.refs)
        self.ctx.tts_kv8_fork(self.pools, self.table, 0, self.lens, N, i32(parents) if device_parents is None else device_parents, N, self.refs, table, lens, refs)
        self.table, self.lens, self.refs = table, lens, refs
        for book in self.books:
            book.tokens = [list(book.tokens[p]) for p in parents]
        assert self.lens.tolist() == self.books[0].lens

    def select(self, step):
        logits = torch.randn(N, VOCAB, generator=self.gen, device="cuda") * 3
        parents, tokens, scores = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")
        self.ctx.tts_beam_select(logits, 1, VOCAB, VOCAB, self.scores, self.finished, VOCAB - 1, QUESTIONS, BEAMS, BEAMS, parents, tokens, scores)
        want = [w for g in k8.select(logits, self.scores, self.finished, VOCAB - 1, QUESTIONS, BEAMS, BEAMS) for w in g]
        assert parents.tolist() == [w[0] for w in want] and tokens.tolist() == [w[1] for w in want]
        assert all(abs(s - w[2]) <= abs(w[2]) * 2.0 ** -23 + 2.0 ** -21 for s, w in zip(scores.tolist(), want))
        self.fork(parents.tolist(), parents)
        history, hidden, finished = torch.empty_like(self.history), torch.empty_like(self.hidden), torch.empty_like(self.finished)
        states = tts.TtsStates([self.history, self.hidden, self.finished], [history, hidden, finished], [4 * STEPS, 10, 4])
        self.ctx.tts_beam_reorder(states, parents, N, N)
        before = self.hidden
        self.history, self.hidden, self.finished, self.scores = history, hidden, finished, scores
        self.history[:, step] = tokens
        self.texts = [self.texts[w[0]] + [w[1]] for w in want]
        assert torch.equal(self.hidden, before[parents.long()]) and self.history[:, :step + 1].tolist() == self.texts

    def compact(self):
        used = i32([0])
        self.ctx.tts_kv8_compact(self.pools, self.table, N, self.refs, self.table, self.refs, torch.empty_like(self.refs), used)
        assert used.item() == len({e for row in self.table.tolist() for e in row if e >= 0})

    def read(self):
        """All pages back in bf16, where each branch's tokens stand as their values, rounded once."""
        live = sorted({e for row in self.table.tolist() for e in row if e >= 0})
        for records, book in zip(self.records, self.books):
            k, v = (torch.zeros(len(live), HKV, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            self.ctx.tts_kv8_read(self.fmt, records, i32(live), i32(list(range(len(live)))), len(live), k, v, len(live))
            for b, row in enumerate(self.table.tolist()):
                at = [live.index(e) for e in row if e >= 0]
                for got, want in zip((k, v), book.kv(b)):
                    assert torch.equal(got[at].transpose(0, 1).flatten(1, 2)[:, :book.lens[b]], want.float().bfloat16())


@pytest.mark.parametrize("fmt", [k8.E4M3, k8.INT8])
def test_a_beam_search_from_prompt_to_answer(fmt):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s = Search(fmt)
        s.append([37, 0, 0, 16, 0, 0])                  # two questions' prompts
        s.fork([0] * BEAMS + [BEAMS] * BEAMS)
        s.scores = torch.tensor([0.0, float("-inf"), float("-inf")] * QUESTIONS, device="cuda")      # so that the first step takes different tokens
        step = 0
        for _ in range(5):                              # single tokens
            s.append([int(not f) for f in s.finished.tolist()])
            s.attend(1)
            s.select(step)
            step += 1
        s.finished[s.r.randrange(N)] = 1
        for _ in range(4):
            s.append([int(not f) for f in s.finished.tolist()])
            s.attend(1)
            s.select(step)
            step += 1
        s.compact()
        s.append([4] * N)                               # drafted chains, cut back
        s.attend(4)
        accepted = [s.r.randrange(5) for _ in range(N)]
        s.ctx.tts_kv_rollback(s.lens, i32(accepted), N, 4)
        for book in s.books:
            for b, a in enumerate(accepted):
                del book.tokens[b][len(book.tokens[b]) - (4 - a):]
        assert s.lens.tolist() == s.books[0].lens
        s.append([10] * N)                              # draft trees: 80 rows to the KV head
        s.attend(10, [[s.r.randrange(-1, i) if i else -1 for i in range(10)] for _ in range(N)])
        s.select(step)
        s.append([1] * N)
        s.attend(16)                                    # and chains of as many rows as the context allows
        s.compact()
        s.attend(1)
        s.read()
        assert s.ctx.tts_last_status() == 0
    stream.synchronize()


def test_a_captured_step_is_the_eager_one():
    """Grow, append, attention, selection, fork and reordering, captured once and replayed for several steps, against the same
    calls made one by one on another context."""
    def make(stream):
        ctx = tts.TtsContext(HQ, HKV, N, 8, WIDTH, PAGES)
        ctx.tts_set_stream(stream)
        ctx.tts_beam_reserve(N, BEAMS)
        t = {"records": torch.zeros(PAGES, HKV, k8.RECORD, dtype=torch.uint8, device="cuda"), "table": i32([[-1] * WIDTH] * N), "lens": i32([0] * N),
             "refs": i32([0] * PAGES), "scores": -torch.arange(N, device="cuda").float(), "tokens": i32([0] * N), "parents": i32([0] * N),
             "q": torch.zeros(N, HQ, 128, device="cuda", dtype=torch.bfloat16), "kv": torch.zeros(N, 2, HKV, 128, device="cuda", dtype=torch.bfloat16),
             "logits": torch.zeros(N, VOCAB, device="cuda"), "out": torch.zeros(N, HQ, 128, device="cuda", dtype=torch.bfloat16),
             "wide_q": torch.zeros(8 * N, HQ, 128, device="cuda", dtype=torch.bfloat16), "wide_out": torch.zeros(8 * N, HQ, 128, device="cuda", dtype=torch.bfloat16),
             "hidden": torch.zeros(N, HQ * 128, device="cuda", dtype=torch.bfloat16), "table2": i32([[-1] * WIDTH] * N), "lens2": i32([0] * N),
             "refs2": i32([0] * PAGES), "scores2": torch.zeros(N, device="cuda"), "ones": i32([1] * N), "starts": i32(list(range(N + 1)))}
        return ctx, t, tts.TtsKv8Pools([t["records"]]), tts.TtsStates([t["out"]], [t["hidden"]], [HQ * 256])

    def step(ctx, t, pools, states):
        ctx.tts_kv_grow(t["table"], 0, t["lens"], t["ones"], N, t["refs"])
        ctx.tts_kv8_append(k8.INT8, None, None, 0, t["kv"][:, 0], t["kv"][:, 1], 2 * HKV * 128, None, t["records"], t["table"], 0, t["lens"], t["starts"], N, N, None)
        ctx.tts_kv8_attn(k8.INT8, t["q"], HQ * 128, t["records"], t["table"], 0, t["lens"], None, N, 1, t["out"], None)
        ctx.tts_kv8_attn(k8.INT8, t["wide_q"], HQ * 128, t["records"], t["table"], 0, t["lens"], None, N, 8, t["wide_out"], None)
        ctx.tts_beam_select(t["logits"], 1, VOCAB, VOCAB, t["scores"], None, 0, QUESTIONS, BEAMS, BEAMS, t["parents"], t["tokens"], t["scores2"])
        ctx.tts_kv8_fork(pools, t["table"], 0, t["lens"], N, t["parents"], N, t["refs"], t["table2"], t["lens2"], t["refs2"])
        ctx.tts_beam_reorder(states, t["parents"], N, N)
        for name in ("table", "lens", "refs", "scores"):
            t[name].copy_(t[name + "2"])

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        eager, captured = make(stream), make(stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(*captured)
        gen = torch.Generator(device="cuda").manual_seed(3)
        for _ in range(40):
            for name in ("q", "kv", "logits", "wide_q"):
                captured[1][name].normal_(generator=gen)
                eager[1][name].copy_(captured[1][name])
            step(*eager)
            graph.replay()
            for name in eager[1]:
                assert torch.equal(eager[1][name], captured[1][name]), name
        assert eager[0].tts_last_status() == 0 and captured[0].tts_last_status() == 0
        assert eager[1]["lens"].tolist() == [40] * N
    del graph
