"""Plain implementations, in 64 bits or in whole numbers, of the cache operators, and cases for them.  Nothing
here calls the library.  Works on CPU and GPU tensors alike."""
from __future__ import annotations

import math
import random

import torch

PAGE, DIM = 16, 128


class Cache:
    """A paged cache with ragged chunks of new tokens: page tables, pools, lengths."""

    def __init__(self, hq, hkv, chunk, lens, prefix=0, seed=0, device="cuda", spare=3, extra_blocks=0, first_row=0, rows_behind=0,
                 q_scale=1.0, poison=True, num_pages=None):
        r = random.Random(seed)
        gen = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.prefix, self.chunk, self.lens = hq, hkv, prefix, list(chunk), list(lens)
        self.n = len(chunk)
        shared = prefix // PAGE
        need = [-(-x // PAGE) for x in lens]
        total = shared + sum(need) + spare
        self.num_pages = num_pages or total
        ids = r.sample(range(self.num_pages), total) if num_pages is None or num_pages < 100000 else \
            [self.num_pages - 1 - i for i in range(total)]
        at, self.rows = shared, []
        for n in need:
            self.rows.append(ids[:shared] + ids[at:at + n])
            at += n
        self.width = max(1, max(len(x) for x in self.rows)) + extra_blocks
        self.table = torch.tensor([x + [-1] * (self.width - len(x)) for x in self.rows], dtype=torch.int32, device=device)
        starts = [first_row]
        for c in chunk:
            starts.append(starts[-1] + c)
        self.starts, self.total_rows = starts, starts[-1] + rows_behind
        self.row_start = torch.tensor(starts, dtype=torch.int32, device=device)
        self.branch_lens = torch.tensor(lens, dtype=torch.int32, device=device)
        if num_pages is None or num_pages < 100000:
            self.k = torch.randn(self.num_pages, hkv, PAGE, DIM, generator=gen).bfloat16()
            self.v = torch.randn(self.num_pages, hkv, PAGE, DIM, generator=gen).bfloat16()
            if poison:
                self._poison()
            self.k, self.v = self.k.to(device), self.v.to(device)
        self.q = (torch.randn(max(1, self.total_rows), hq, DIM, generator=gen) * q_scale).bfloat16().to(device)

    def _poison(self):
        """NaN in every slot that holds no token."""
        used = torch.zeros(self.num_pages, PAGE, dtype=torch.bool)
        for b, row in enumerate(self.rows):
            for i, page in enumerate(row):
                filled = min(PAGE, self.prefix + self.lens[b] - i * PAGE)
                used[page, :max(0, filled)] = True
        for x in (self.k, self.v):
            x.permute(0, 2, 1, 3)[~used] = float("nan")


def chunk_attention(c: Cache, scale=None):
    """(out, lse, mean) in 64 bits for the rows that belong to a branch; `mean`: the same mean of |V|, which the
    rounding of the probabilities is relative to.  Rows of no branch are zeros."""
    scale = scale or 1 / math.sqrt(DIM)
    dev = c.q.device
    out = torch.zeros(c.total_rows, c.hq, DIM, dtype=torch.float64, device=dev)
    mean = torch.zeros_like(out)
    lse = torch.zeros(c.total_rows, c.hq, dtype=torch.float64, device=dev)
    group = c.hq // c.hkv
    for b in range(c.n):
        n, total = c.chunk[b], c.prefix + c.lens[b]
        if n == 0:
            continue
        rows = slice(c.starts[b], c.starts[b] + n)
        pages = torch.tensor(c.rows[b], dtype=torch.long, device=dev)
        k = c.k[pages].permute(1, 0, 2, 3).reshape(c.hkv, -1, DIM)[:, :total].double().repeat_interleave(group, 0)
        v = c.v[pages].permute(1, 0, 2, 3).reshape(c.hkv, -1, DIM)[:, :total].double().repeat_interleave(group, 0)
        s = torch.einsum("rhd,htd->hrt", c.q[rows].double(), k) * scale
        place = torch.arange(n, device=dev) + total - n
        s = s.masked_fill(torch.arange(total, device=dev)[None, :] > place[:, None], -math.inf)
        if total == 0:
            lse[rows] = -math.inf
            continue
        l = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(l == -math.inf, 0.0, l)[..., None])
        out[rows] = torch.einsum("hrt,htd->rhd", p, v)
        mean[rows] = torch.einsum("hrt,htd->rhd", p, v.abs())
        lse[rows] = l.T
    return out, lse, mean


def rope_turn(x, positions, axis, inv_freq, interleaved):
    """x [rows][heads][128] turned in 64 bits, pair by pair."""
    x = x.double().clone()
    n = len(inv_freq)
    for i in range(n):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = (positions[axis[i]].double() * inv_freq[i])[:, None]
        a, b = x[..., lo].clone(), x[..., hi].clone()
        x[..., lo] = a * angle.cos() - b * angle.sin()
        x[..., hi] = a * angle.sin() + b * angle.cos()
    return x


# ---------------------------------------------------------------------------- pages: lists and whole numbers
class Book:
    """Tables, lengths and reference counts as Python lists."""

    def __init__(self, table, prefix, lens, num_pages):
        self.table, self.prefix, self.lens, self.num_pages = [list(x) for x in table], prefix, list(lens), num_pages

    def refs(self):
        n = [0] * self.num_pages
        for row in self.table:
            for e in row:
                if e >= 0:
                    n[e] += 1
        return n

    def fork(self, parents, refs):
        """(children's Book, [(source, target)]) with free pages taken lowest first; None when they do not suffice."""
        free = [p for p, n in enumerate(refs) if n == 0]
        width, seen, copies, table, lens = len(self.table[0]), set(), [], [], []
        for p in parents:
            if p < 0:
                table.append([-1] * width)
                lens.append(0)
                continue
            full, rest = divmod(self.prefix + self.lens[p], PAGE)
            if p not in seen:
                row = list(self.table[p])
            else:
                row = self.table[p][:full] + [-1] * (width - full)
                if rest:
                    if not free:
                        return None
                    row[full] = free.pop(0)
                    copies.append((self.table[p][full], row[full]))
            seen.add(p)
            table.append(row)
            lens.append(self.lens[p])
        return Book(table, self.prefix, lens, self.num_pages), copies

    def grow(self, n_new, refs):
        free = [p for p, n in enumerate(refs) if n == 0]
        table = [list(x) for x in self.table]
        for b, more in enumerate(n_new):
            if more == 0:
                continue
            for i in range(-(-(self.prefix + self.lens[b]) // PAGE), -(-(self.prefix + self.lens[b] + more) // PAGE)):
                if table[b][i] < 0:
                    if not free:
                        return None
                    table[b][i] = free.pop(0)
        return Book(table, self.prefix, [x + m for x, m in zip(self.lens, n_new)], self.num_pages)

    def compact(self, refs):
        used = [p for p, n in enumerate(refs) if n]
        moved = [p for p in used if p >= len(used)]
        to = dict(zip(moved, [p for p in range(len(used)) if not refs[p]]))
        page_map = [to.get(p, p) if refs[p] else -1 for p in range(self.num_pages)]
        table = [[page_map[e] if e >= 0 else -1 for e in row] for row in self.table]
        return Book(table, self.prefix, self.lens, self.num_pages), page_map, len(used)
