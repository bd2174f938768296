"""The cache operators as they are used together: prompts enter the cache in pieces, branches are forked, grow, decode a
speculative step, are cut back, some finish, the pool is closed up.  After every step the attention over the cache is
compared with dense attention, in 64 bits, over each branch's own list of tokens, which knows nothing of pages.

Tolerance: keys and queries are rotated and rounded to bf16 by the library and not by the reference.  A rounded element is
off by 2^-8 of itself at most, so a score by 2 x 2^-8 x scale x sum |q k|, and that sum by Cauchy and Schwarz is at most
|q| |k| (about 11.3 each for N(0, 1) vectors, below 14.5 here), 1.6 in all; every weight is off by at most e^1.6 in the
worst case but by 2^-8 x 1.6 = 0.0064 for errors that do not conspire (128 independent ones: x sqrt(1/128) x 4 sigma).
The checks are the relative RMS error of all elements, 1.5e-2, and 0.15 of the softmax mean of |V| for each element."""
import math
import random

import pytest
import torch

import paper_2505_19634_b200 as tts
from cache_plain import rope_turn

pytestmark = pytest.mark.gpu

HQ, HKV, WIDTH, PAGES, N, LAYERS = 10, 2, 40, 160, 6, 2
FREQ = [1e4 ** (-i / 64) for i in range(64)]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Server:
    def __init__(self):
        self.gen = torch.Generator(device="cuda").manual_seed(0)
        self.ctx = tts.TtsContext(HQ, HKV, N, 4, WIDTH, PAGES, debug_bounds=True)
        self.ctx.tts_chunk_reserve(1000)
        self.k = torch.full((LAYERS, PAGES, HKV, 16, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
        self.v = self.k.clone()
        self.pools = tts.TtsPools(list(self.k), list(self.v))
        self.table = torch.full((N, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.lens, self.refs = i32([0] * N), i32([0] * PAGES)
        self.rope = tts.TtsRope([0] * 64, FREQ)
        self.tokens = [[[] for _ in range(N)] for _ in range(LAYERS)]      # (key, value) of every token, per layer and branch

    def rows(self, chunk):
        """New tokens for the branches: grows them, rotates and appends, attends; returns the rows' queries per layer."""
        starts = [0]
        for c in chunk:
            starts.append(starts[-1] + c)
        total = starts[-1]
        self.ctx.tts_kv_grow(self.table, 0, self.lens, i32(chunk), N, self.refs)
        position = torch.cat([torch.arange(len(self.tokens[0][b]), len(self.tokens[0][b]) + c, device="cuda") for b, c in enumerate(chunk)])
        position = position.to(torch.int32)[None].contiguous()
        queries = []
        for layer in range(LAYERS):
            qkv = torch.randn(total, HQ + 2 * HKV, 128, generator=self.gen, device="cuda").bfloat16()
            q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
            q_out = torch.empty(total, HQ, 128, device="cuda", dtype=torch.bfloat16)
            self.ctx.tts_kv_append_rope(self.rope, q, q.stride(0), k, v, k.stride(0), position, self.k[layer], self.v[layer], self.table, 0,
                                        self.lens, i32(starts), N, total, q_out)
            turned = rope_turn(k, position, [0] * 64, FREQ, False)
            for b, c in enumerate(chunk):
                for i in range(c):
                    self.tokens[layer][b].append((turned[starts[b] + i], v[starts[b] + i].double()))
            queries.append((rope_turn(q, position, [0] * 64, FREQ, False), q_out))
        self.check(chunk, starts, queries)
        return starts, queries

    def check(self, chunk, starts, queries, out_of=None):
        for layer in range(LAYERS):
            q64, q = queries[layer]
            if out_of is None:
                out = torch.empty_like(q)
                self.ctx.tts_chunk_attn(q, HQ * 128, self.k[layer], self.v[layer], self.table, 0, self.lens, i32(starts), N, q.shape[0], out)
            else:
                out = out_of(layer, q)
            torch.cuda.synchronize()
            assert self.ctx.tts_last_status() == 0
            square = total = 0.0
            for b, c in enumerate(chunk):
                if c == 0:
                    continue
                k = torch.stack([t[0] for t in self.tokens[layer][b]]).repeat_interleave(HQ // HKV, 1)
                v = torch.stack([t[1] for t in self.tokens[layer][b]]).repeat_interleave(HQ // HKV, 1)
                n = len(k)
                s = torch.einsum("rhd,thd->hrt", q64[starts[b]:starts[b] + c], k) / math.sqrt(128)
                s = s.masked_fill(torch.arange(n, device="cuda")[None] > torch.arange(n - c, n, device="cuda")[:, None], -math.inf)
                p = s.softmax(-1)
                want = torch.einsum("hrt,thd->rhd", p, v)
                off = (out[starts[b]:starts[b] + c].double() - want).abs()
                assert (off <= 0.15 * torch.einsum("hrt,thd->rhd", p, v.abs())).all()
                square += off.square().sum().item()
                total += want.square().sum().item()
            assert math.sqrt(square / total) <= 1.5e-2

    def fork(self, parents):
        table, lens, refs = torch.empty_like(self.table), torch.empty_like(self.lens), torch.empty_like(self.refs)
        self.ctx.tts_kv_fork(self.pools, self.table, 0, self.lens, N, i32(parents), N, self.refs, table, lens, refs)
        self.table, self.lens, self.refs = table, lens, refs
        self.tokens = [[list(t[p]) if p >= 0 else [] for p in parents] for t in self.tokens]

    def cut(self, gamma, accepted):
        self.ctx.tts_kv_rollback(self.lens, i32(accepted), N, gamma)
        for t in self.tokens:
            for b, a in enumerate(accepted):
                if gamma - a:
                    del t[b][len(t[b]) - (gamma - a):]


def test_a_search_from_prompt_to_answer():
    r = random.Random(4)
    s = Server()
    s.rows([33, 0, 0, 100, 0, 0])                        # two questions: the first pieces of their prompts
    s.rows([17, 0, 0, 64, 0, 0])                         # and the rest
    s.fork([0, 0, 0, 3, 3, 3])                           # three branches each
    for step in range(3):
        # a speculative step: the last token and three drafts of every branch, through the chunk attention and, on the
        # same rows, through the verify attention
        starts, queries = s.rows([4] * N)

        def verify(layer, q):
            out = torch.empty_like(q)
            s.ctx.tts_verify_attn(q, s.k[layer], s.v[layer], s.table, 0, s.lens, N, 3, tts.MASK_CAUSAL, out)
            return out

        s.check([4] * N, starts, queries, verify)
        s.cut(3, [r.randrange(4) for _ in range(N)])
        s.fork([r.choice([0, 1, 2]) for _ in range(3)] + [r.choice([3, 4, 5]) for _ in range(3)])
    # two branches finish, the pool is closed up, the others go on with one token each
    s.ctx.tts_kv_free(s.table, s.lens, i32([0, 1, 0, 0, 0, 1]), N, s.refs)
    for t in s.tokens:
        t[1], t[5] = [], []
    page_map, used = torch.empty_like(s.refs), i32([0])
    s.ctx.tts_kv_compact(s.pools, s.table, N, s.refs, s.table, s.refs, page_map, used)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    held = s.table[s.table >= 0]
    assert used.item() == held.unique().numel() == int(held.max()) + 1
    assert torch.equal(s.refs, torch.bincount(held.long(), minlength=PAGES).to(torch.int32))
    s.rows([1, 0, 1, 1, 1, 0])
    s.rows([1, 60, 1, 1, 30, 0])                         # a freed branch takes a new prompt
    s.ctx.close()
