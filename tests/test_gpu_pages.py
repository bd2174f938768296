"""Upkeep of the cache's pages (tts_kv_fork, _grow, _free, _compact, _copy_pages) against lists and whole numbers:
every table entry, length, count and byte of the pools has to be equal."""
import random

import pytest
import torch

import paper_2505_19634_b200 as tts
from cache_plain import PAGE, Book

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Setup:
    def __init__(self, seed, n, prefix, lens, layers=3, hkv=2, spare=20, width=None, max_branches=None, held_back=()):
        r = random.Random(seed)
        shared = prefix // PAGE
        need = [-(-x // PAGE) for x in lens]
        num_pages = shared + sum(need) + spare
        ids = r.sample(range(num_pages), num_pages)
        width = width or shared + max(need) + 6
        at, table = shared, []
        for k in need:
            table.append(ids[:shared] + ids[at:at + k] + [-1] * (width - shared - k))
            at += k
        for b, more in held_back:                             # pages a branch holds beyond its length
            for j in range(more):
                table[b][shared + need[b] + j] = ids[at]
                at += 1
        self.book = Book(table, prefix, lens, num_pages)
        self.n, self.prefix, self.width, self.pages, self.hkv = n, prefix, width, num_pages, hkv
        self.table, self.lens, self.refs = i32(table), i32(lens), i32(self.book.refs())
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k = torch.randn(layers, num_pages, hkv, PAGE, 128, generator=g, device="cuda").bfloat16()
        self.v = torch.randn(layers, num_pages, hkv, PAGE, 128, generator=g, device="cuda").bfloat16()
        self.pools = tts.TtsPools(list(self.k), list(self.v))
        self.ctx = tts.TtsContext(2 * hkv, hkv, max_branches or max(n, 64), 1, width, num_pages)

    def fork(self, parents, alias=False, **kw):
        m = len(parents)
        self.new_table, self.new_lens = torch.full((m, self.width), 77, dtype=torch.int32, device="cuda"), torch.full((m,), 77, dtype=torch.int32, device="cuda")
        self.new_refs = self.refs if alias else torch.full_like(self.refs, 77)
        self.ctx.tts_kv_fork(self.pools, kw.get("table", self.table), self.prefix, kw.get("lens", self.lens), self.n, i32(parents), m, self.refs,
                             self.new_table, self.new_lens, self.new_refs)
        torch.cuda.synchronize()
        return self.ctx.tts_last_status()


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("parents", [[0], [0, 0, 0, 0], [2, 1, 0, 3], [3, 3, 1, 3, 1, 3], [-1, 2, -1, 2], [-1], [0] * 20])
def test_fork(parents, alias):
    s = Setup(1, 4, 32, [5, 16, 37, 160], spare=25, held_back=[(2, 2)])
    k0, v0 = s.k.clone(), s.v.clone()
    want, copies = s.book.fork(parents, s.book.refs())
    assert s.fork(parents, alias) == 0
    assert s.new_table.tolist() == want.table and s.new_lens.tolist() == want.lens and s.new_refs.tolist() == want.refs()
    for a, b in copies:
        k0[:, b], v0[:, b] = k0[:, a], v0[:, a]
    assert torch.equal(s.k, k0) and torch.equal(s.v, v0)
    s.ctx.close()


def test_fork_generations_keep_the_books():
    """Forks, growth and frees in a row: after each, the counts are those of the table, and every branch reads the
    tokens that its line of ancestors wrote."""
    s = Setup(2, 8, 16, [20] * 8, spare=400, width=40)
    r = random.Random(0)
    tokens = torch.zeros(s.pages, PAGE, dtype=torch.long)                 # what is written in layer 0, head 0, dim 0
    stamp = 1
    table, lens, refs = s.table, s.lens, s.refs
    lines = [[-1] * 36 for _ in range(8)]
    for b in range(8):
        for t in range(36):
            page = s.book.table[b][t // PAGE]
            v = 0 if t < 16 else stamp
            lines[b][t] = v
            s.k[0, page, 0, t % PAGE, 0] = v
            stamp += t >= 16
    for step in range(6):
        parents = [r.randrange(-1, 8) if r.random() < 0.3 else r.randrange(8) for _ in range(8)]
        parents = [p if p >= 0 and len(lines[p]) else -1 for p in parents]
        nt, nl, nr = torch.empty_like(table), torch.empty_like(lens), torch.empty_like(refs)
        s.ctx.tts_kv_fork(s.pools, table, 16, lens, 8, i32(parents), 8, refs, nt, nl, nr)
        lines = [list(lines[p]) if p >= 0 else [] for p in parents]
        more = [r.randrange(0, 23) if lines[b] else 0 for b in range(8)]
        s.ctx.tts_kv_grow(nt, 16, nl, i32(more), 8, nr)
        torch.cuda.synchronize()
        assert s.ctx.tts_last_status() == 0
        book = Book(nt.tolist(), 16, nl.tolist(), s.pages)
        assert nr.tolist() == book.refs()
        for b in range(8):
            for _ in range(more[b]):
                t = len(lines[b])
                s.k[0, book.table[b][t // PAGE], 0, t % PAGE, 0] = stamp % 256
                lines[b].append(stamp % 256)
                stamp += 1
            assert book.lens[b] == (len(lines[b]) - 16 if lines[b] else 0)
            got = [int(s.k[0, book.table[b][t // PAGE], 0, t % PAGE, 0]) for t in range(len(lines[b]))]
            assert got == [int(torch.tensor(float(x)).bfloat16()) for x in lines[b]]
        table, lens, refs = nt, nl, nr
    s.ctx.close()


def test_fork_without_enough_pages_changes_nothing():
    s = Setup(1, 4, 32, [5, 16, 37, 160], spare=2)
    k0 = s.k.clone()
    assert s.fork([0, 0, 0, 2, 2]) == -7                                  # three copies, two free pages
    assert (s.new_table == 77).all() and (s.new_lens == 77).all() and torch.equal(s.new_refs, s.refs) and torch.equal(s.k, k0)
    assert s.fork([0, 0, 2, 2]) == 0                                      # two copies
    s.ctx.close()


def test_fork_bad_values_are_reported():
    s = Setup(1, 4, 32, [5, 16, 37, 160])
    assert s.fork([0, 4, -2, 1]) == -4                                    # no such parents: empty rows
    want, _ = s.book.fork([0, -1, -1, 1], s.book.refs())
    assert s.new_table.tolist() == want.table and s.new_refs.tolist() == want.refs()
    assert s.fork([3, 0], lens=i32([5, 16, 37, 16 * s.width])) == -4      # longer than the table row
    assert s.new_table[0].tolist() == [-1] * s.width
    bad = s.table.clone()
    bad[0, 2] = s.pages + 3                                               # the part-filled page of branch 0
    assert s.fork([0, 0], table=bad) == -4
    assert s.new_table[1, 2] == -1 and s.new_table[0, 2] == -1
    s.ctx.close()


@pytest.mark.parametrize("n_new", [[0, 0, 0, 0], [1, 1, 1, 1], [11, 0, 12, 30], [80, 0, 0, 0], [16, 16, 16, 16]])
def test_grow(n_new):
    s = Setup(3, 4, 32, [5, 16, 37, 160], held_back=[(2, 1)])
    refs = s.book.refs()
    want = s.book.grow(n_new, refs)
    s.ctx.tts_kv_grow(s.table, 32, s.lens, i32(n_new), 4, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    assert s.table.tolist() == want.table and s.lens.tolist() == want.lens and s.refs.tolist() == want.refs()
    s.ctx.close()


@pytest.mark.parametrize("n_new,status", [([-1, 1, 1, 1], -4), ([1, 1, 1, 200], -4), ([1, 1, 1, 2 ** 31 - 1], -4), ([90, 90, 90, 0], -7)])
def test_grow_is_all_or_nothing(n_new, status):
    s = Setup(3, 4, 32, [5, 16, 37, 160], spare=9)
    before = s.table.clone(), s.lens.clone(), s.refs.clone()
    s.ctx.tts_kv_grow(s.table, 32, s.lens, i32(n_new), 4, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == status
    assert all(torch.equal(a, b) for a, b in zip(before, (s.table, s.lens, s.refs)))
    s.ctx.close()


def test_grow_many_branches_and_pages_past_one_step_of_the_scan():
    lens = [random.Random(i).randrange(1, 300) for i in range(1000)]
    s = Setup(3, 1000, 0, lens, layers=1, hkv=1, spare=40000, width=40, max_branches=1000)
    n_new = [random.Random(i).randrange(0, 300) for i in range(1000)]
    want = s.book.grow(n_new, s.book.refs())
    s.ctx.tts_kv_grow(s.table, 0, s.lens, i32(n_new), 1000, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    assert s.table.tolist() == want.table and s.lens.tolist() == want.lens and s.refs.tolist() == want.refs()
    s.ctx.close()


def test_free():
    s = Setup(4, 5, 32, [5, 16, 37, 160, 90], held_back=[(1, 3)])
    freed = [0, 1, 0, 7, 0]
    s.ctx.tts_kv_free(s.table, s.lens, i32(freed), 5, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    rows = [[-1] * s.width if f else row for f, row in zip(freed, s.book.table)]
    want = Book(rows, 32, [0 if f else n for f, n in zip(freed, s.book.lens)], s.pages)
    assert s.table.tolist() == rows and s.lens.tolist() == want.lens and s.refs.tolist() == want.refs()
    s.ctx.tts_kv_free(s.table, s.lens, i32(freed), 5, s.refs)             # freeing empty rows again does nothing
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0 and s.refs.tolist() == want.refs()
    s.table[0, 0] = s.pages                                               # a page that does not exist
    s.ctx.tts_kv_free(s.table, s.lens, i32([1, 0, 0, 0, 0]), 5, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4
    s.ctx.close()


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("n,kept,spare,hkv,layers", [(6, 3, 20, 2, 3), (6, 6, 0, 1, 1), (6, 0, 5, 2, 2), (200, 77, 33000, 1, 2), (40, 1, 100, 8, 2)])
def test_compact(n, kept, spare, hkv, layers, alias):
    r = random.Random(n)
    s = Setup(5, n, 48, [r.randrange(1, 200) for _ in range(n)], layers=layers, hkv=hkv, spare=spare, max_branches=n)
    gone = set(range(n)) - set(r.sample(range(n), kept))
    book = Book([[-1] * s.width if b in gone else row for b, row in enumerate(s.book.table)], 48, s.book.lens, s.pages)
    table, refs = i32(book.table), i32(book.refs())
    want, page_map, used = book.compact(book.refs())
    k0, v0 = s.k.clone(), s.v.clone()
    new_table, new_refs = (table, refs) if alias else (torch.full_like(table, 77), torch.full_like(refs, 77))
    got_map, got_used = torch.full_like(refs, 77), i32([77])
    s.ctx.tts_kv_compact(s.pools, table, n, refs, new_table, new_refs, got_map, got_used)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    assert new_table.tolist() == want.table and new_refs.tolist() == want.refs() and got_map.tolist() == page_map and got_used.item() == used
    assert all(x > 0 for x in new_refs.tolist()[:used]) and not any(new_refs.tolist()[used:])
    for old, new in enumerate(page_map):
        if new >= 0 and new != old:
            k0[:, new], v0[:, new] = k0[:, old], v0[:, old]
    assert torch.equal(s.k, k0) and torch.equal(s.v, v0)
    s.ctx.close()


def test_compact_reports_entries_that_the_counts_do_not_know():
    s = Setup(5, 4, 0, [40, 50, 60, 70])
    free = s.book.refs().index(0)
    s.table[1, 1] = free
    out, refs, page_map, used = torch.empty_like(s.table), torch.empty_like(s.refs), torch.empty_like(s.refs), i32([0])
    s.ctx.tts_kv_compact(s.pools, s.table, 4, s.refs, out, refs, page_map, used)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4 and out[1, 1] == -1
    s.ctx.close()


def test_copy_pages():
    s = Setup(6, 2, 0, [100, 200], layers=5, hkv=8)
    src, dst = [3, 0, -1, 7, 2], [10, 11, 12, -1, 2]
    k0, v0 = s.k.clone(), s.v.clone()
    s.ctx.tts_kv_copy_pages(s.pools, i32(src), i32(dst), 5)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    for a, b in zip(src, dst):
        if a >= 0 and b >= 0:
            k0[:, b], v0[:, b] = k0[:, a], v0[:, a]
    assert torch.equal(s.k, k0) and torch.equal(s.v, v0)
    s.ctx.tts_kv_copy_pages(s.pools, i32([1, s.pages]), i32([s.pages, 1]), 2)
    s.ctx.tts_kv_copy_pages(s.pools, i32([1]), i32([2]), 0)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4 and torch.equal(s.k, k0)
    s.ctx.close()


def test_copies_beyond_32_bit_offsets():
    pages = 140000                                            # x 8 heads x 4 KiB = 4.6 GB per pool
    k = torch.zeros(pages, 8, PAGE, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[5], v[5] = 1.5, 2.5
    ctx = tts.TtsContext(8, 8, 2, 1, 4, pages)
    ctx.tts_kv_copy_pages(tts.TtsPools([k], [v]), i32([5]), i32([pages - 1]), 1)
    table = i32([[pages - 1, 7, -1, -1], [-1] * 4])
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[pages - 1] = refs[7] = 1
    page_map, used = torch.empty_like(refs), i32([0])
    ctx.tts_kv_compact(tts.TtsPools([k], [v]), table, 2, refs, table, refs, page_map, used)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0 and used.item() == 2
    assert table[0].tolist() == [1, 0, -1, -1] and page_map[pages - 1] == 1 and page_map[7] == 0
    assert (k[pages - 1] == 1.5).all() and (k[1] == 1.5).all() and (v[1] == 2.5).all() and k.double().abs().sum() == 1.5 * 3 * 8 * PAGE * 128
    ctx.close()


def test_captured_fork_and_grow():
    s = Setup(7, 4, 32, [5, 16, 37, 160], spare=60)
    parents, more = i32([1, 1, 2, 2]), i32([9, 9, 9, 9])
    nt, nl, nr = torch.empty_like(s.table), torch.empty_like(s.lens), torch.empty_like(s.refs)
    side = torch.cuda.Stream()
    s.ctx.tts_set_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.ctx.tts_kv_fork(s.pools, s.table, 32, s.lens, 4, parents, 4, s.refs, nt, nl, nr)
        s.ctx.tts_kv_grow(nt, 32, nl, more, 4, nr)
    for p in ([1, 1, 2, 2], [3, 3, 3, 0], [0, 1, 2, 3]):
        parents.copy_(i32(p))
        graph.replay()
        torch.cuda.synchronize()
        want, _ = s.book.fork(p, s.book.refs())
        want = want.grow([9] * 4, want.refs())
        assert nt.tolist() == want.table and nl.tolist() == want.lens and nr.tolist() == want.refs()
    assert s.ctx.tts_last_status() == 0
    s.ctx.close()


def test_refusals():
    s = Setup(8, 4, 32, [5, 16, 37, 160])
    p, m = i32([0, 0]), i32([1, 1, 1, 1])
    nt, nl, nr = torch.empty(2, s.width, dtype=torch.int32, device="cuda"), i32([0, 0]), torch.empty_like(s.refs)
    full, pm, nu = torch.empty_like(s.table), torch.empty_like(s.refs), i32([0])
    none = tts.TtsPools([], [])
    many = tts.TtsPools([s.k[0]] * 129, [s.v[0]] * 129)
    odd = tts.TtsPools([s.k.data_ptr() + 2], [s.v.data_ptr()])
    lost = tts.TtsPools([s.k[0]], [None])

    def refused(fn, *a):
        with pytest.raises(tts.TtsError) as e:
            fn(*a)
        assert e.value.status == -1, a

    fork = [s.pools, s.table, 32, s.lens, 4, p, 2, s.refs, nt, nl, nr]
    for i, bad in [(0, none), (0, many), (0, odd), (0, lost), (1, None), (2, 8), (2, -16), (3, None), (4, 0), (4, 65), (5, None), (6, 0), (6, 65), (7, None), (8, None),
                   (8, s.table), (9, s.lens), (9, None), (10, None), (10, s.refs.data_ptr() + 16), (7, s.refs.data_ptr() + 4)]:
        refused(s.ctx.tts_kv_fork, *fork[:i], bad, *fork[i + 1:])
    grow = [s.table, 32, s.lens, m, 4, s.refs]
    for i, bad in [(0, None), (1, 7), (2, None), (3, None), (4, 0), (4, 65), (5, None)]:
        refused(s.ctx.tts_kv_grow, *grow[:i], bad, *grow[i + 1:])
    free = [s.table, s.lens, m, 4, s.refs]
    for i, bad in [(0, None), (1, None), (2, None), (3, 0), (4, None)]:
        refused(s.ctx.tts_kv_free, *free[:i], bad, *free[i + 1:])
    compact = [s.pools, s.table, 4, s.refs, full, nr, pm, nu]
    for i, bad in [(0, none), (1, None), (2, 0), (3, None), (4, None), (4, s.table.data_ptr() + 4), (5, s.refs.data_ptr() + 16), (6, None), (7, None)]:
        refused(s.ctx.tts_kv_compact, *compact[:i], bad, *compact[i + 1:])
    copy = [s.pools, p, p, 2]
    for i, bad in [(0, none), (1, None), (2, None), (3, -1)]:
        refused(s.ctx.tts_kv_copy_pages, *copy[:i], bad, *copy[i + 1:])
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0
    s.ctx.close()


def test_grow_that_lacks_more_pages_than_32_bits_count():
    """32 rows of the largest table, 2^26 entries each and none with a page, lack 2^31 of them together."""
    n, width, pages = 32, 1 << 26, 64
    ctx = tts.TtsContext(2, 2, n, 1, width, pages)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    lens, refs = i32([0] * n), i32([0] * pages)
    ctx.tts_kv_grow(table, 0, lens, i32([16 * width] * n), n, refs)
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == -7
    assert not lens.any() and not refs.any() and int(table.max()) == -1
    ctx.tts_kv_grow(table, 0, lens, i32([16] * n), n, refs)               # one page each
    torch.cuda.synchronize()
    assert ctx.tts_last_status() == 0
    assert table[:, 0].tolist() == list(range(n)) and int(table[:, 1:].max()) == -1 and lens.tolist() == [16] * n
    assert refs.tolist() == [1] * n + [0] * (pages - n)
    ctx.close()


@pytest.mark.parametrize("emptied_by", ["free", "fork"])
@pytest.mark.parametrize("prefix", [16, 48])
def test_a_row_without_its_prefix_does_not_grow(emptied_by, prefix):
    s = Setup(9, 4, prefix, [5, 16, 37, 160], spare=30)
    if emptied_by == "free":
        s.ctx.tts_kv_free(s.table, s.lens, i32([0, 1, 0, 0]), 4, s.refs)
    else:
        assert s.fork([0, -1, 2, 3]) == 0
        s.table, s.lens, s.refs = s.new_table, s.new_lens, s.new_refs
    before = s.table.clone(), s.lens.clone(), s.refs.clone()
    s.ctx.tts_kv_grow(s.table, prefix, s.lens, i32([1, 20, 1, 1]), 4, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4
    assert all(torch.equal(a, b) for a, b in zip(before, (s.table, s.lens, s.refs)))
    book = Book(s.table.tolist(), prefix, s.lens.tolist(), s.pages)
    s.ctx.tts_kv_grow(s.table, prefix, s.lens, i32([12, 0, 1, 0]), 4, s.refs)           # the others grow beside it
    torch.cuda.synchronize()
    want = book.grow([12, 0, 1, 0], book.refs())
    assert s.ctx.tts_last_status() == 0
    assert s.table.tolist() == want.table and s.lens.tolist() == want.lens and s.refs.tolist() == want.refs()
    shared = prefix // PAGE                                   # the caller gives the row its prefix back
    s.table[1, :shared] = s.table[0, :shared]
    s.refs[s.table[0, :shared].long()] += 1
    book = Book(s.table.tolist(), prefix, s.lens.tolist(), s.pages)
    s.ctx.tts_kv_grow(s.table, prefix, s.lens, i32([0, 20, 0, 0]), 4, s.refs)
    torch.cuda.synchronize()
    want = book.grow([0, 20, 0, 0], book.refs())
    assert s.ctx.tts_last_status() == 0
    assert s.table.tolist() == want.table and s.lens.tolist() == want.lens and s.refs.tolist() == want.refs()
    s.ctx.close()


@pytest.mark.parametrize("branch,entry,page", [(0, 0, -1), (3, 1, -1), (3, 7, -1), (3, 7, "pool"), (3, 12, "free"), (3, 12, "pool"), (3, 12, 2 ** 31 - 1)])
def test_grow_looks_at_the_pages_that_a_row_holds(branch, entry, page):
    """Branch 3 has 32 + 160 tokens, entries 0 .. 11, and an entry behind them that its new tokens would use."""
    s = Setup(9, 4, 32, [5, 16, 37, 160], spare=30, held_back=[(3, 1)])
    s.table[branch, entry] = {"pool": s.pages, "free": s.book.refs().index(0)}.get(page, page)
    before = s.table.clone(), s.lens.clone(), s.refs.clone()
    s.ctx.tts_kv_grow(s.table, 32, s.lens, i32([1, 1, 1, 1]), 4, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4
    assert all(torch.equal(a, b) for a, b in zip(before, (s.table, s.lens, s.refs)))
    more = [0 if b == branch else 1 for b in range(4)]
    s.ctx.tts_kv_grow(s.table, 32, s.lens, i32(more), 4, s.refs)                        # a row that does not grow is not looked at
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == 0 and s.lens.tolist() == [n + m for n, m in zip([5, 16, 37, 160], more)]
    s.ctx.close()


@pytest.mark.parametrize("alias", [False, True])
def test_fork_does_not_give_away_the_pages_of_a_parent_of_a_bad_length(alias):
    for length in (-1, 16 * 100, 2 ** 31 - 1):
        s = Setup(1, 4, 32, [5, 16, 37, 160])
        assert s.fork([3, 0, 3], alias, lens=i32([5, 16, 37, length])) == -4
        want = Book([[-1] * s.width, s.book.table[0], [-1] * s.width], 32, [0, 5, 0], s.pages)
        assert s.new_table.tolist() == want.table and s.new_lens.tolist() == want.lens
        assert s.new_refs.tolist() == Book(want.table + [s.book.table[3]], 32, [0] * 4, s.pages).refs()
        s.ctx.close()


@pytest.mark.parametrize("branch,entry", [(0, 1), (1, 1), (2, 4)])
@pytest.mark.parametrize("page", ["pool", "free", 2 ** 31 - 1])
def test_fork_reports_bad_entries_of_every_row(branch, entry, page):
    """Branch 0 has two children, branch 1 one, branch 2 none.  A bad entry counts as none: the children's are -1."""
    s = Setup(1, 4, 32, [5, 16, 37, 160])
    free = max(p for p, n in enumerate(s.book.refs()) if n == 0)
    table = s.table.clone()
    table[branch, entry] = {"pool": s.pages, "free": free}.get(page, page)
    refs = Book([[-1 if (b, i) == (branch, entry) else e for i, e in enumerate(row)] for b, row in enumerate(s.book.table)], 32, s.book.lens, s.pages)
    s.refs.copy_(i32(refs.refs()))
    want, _ = refs.fork([0, 1, 0, 3], refs.refs())
    assert s.fork([0, 1, 0, 3], table=table) == -4
    assert s.new_table.tolist() == want.table and s.new_refs.tolist() == want.refs()
    s.ctx.close()


@pytest.mark.parametrize("page", ["pool", "free"])
def test_free_of_an_entry_that_nothing_counts_leaves_the_counts(page):
    s = Setup(4, 3, 32, [5, 16, 37])
    s.table[1, 6] = {"pool": s.pages, "free": s.book.refs().index(0)}[page]
    s.ctx.tts_kv_free(s.table, s.lens, i32([0, 1, 0]), 3, s.refs)
    torch.cuda.synchronize()
    assert s.ctx.tts_last_status() == -4
    assert s.refs.tolist() == Book([s.book.table[0], s.book.table[2]], 32, [5, 37], s.pages).refs() and s.table[1].tolist() == [-1] * s.width
    s.ctx.close()


def test_overlaps_are_refused():
    """Whatever a call writes shares no memory with anything else it is given, but for what the header names."""
    s = Setup(8, 4, 32, [5, 16, 37, 160])
    p, m = i32([0, 0, 1, 3]), i32([1, 1, 1, 1])
    nt, nl, nr, pm, nu = torch.empty_like(s.table), i32([0] * 4), torch.empty_like(s.refs), torch.empty_like(s.refs), i32([0])
    calls = {
        "fork": (s.ctx.tts_kv_fork, dict(pools=s.pools, table=s.table, prefix=32, lens=s.lens, n=4, parents=p, m=4, refs=s.refs, new_table=nt, new_lens=nl, new_refs=nr)),
        "grow": (s.ctx.tts_kv_grow, dict(table=s.table, prefix=32, lens=s.lens, more=m, n=4, refs=s.refs)),
        "free": (s.ctx.tts_kv_free, dict(table=s.table, lens=s.lens, freed=m, n=4, refs=s.refs)),
        "compact": (s.ctx.tts_kv_compact, dict(pools=s.pools, table=s.table, n=4, refs=s.refs, new_table=nt, new_refs=nr, page_map=pm, n_used=nu)),
        "copy": (s.ctx.tts_kv_copy_pages, dict(pools=s.pools, src=p, dst=m, n=4)),
    }
    written = {"fork": ["new_table", "new_lens", "new_refs"], "grow": ["table", "lens", "refs"], "free": ["table", "lens", "refs"],
               "compact": ["new_table", "new_refs", "page_map", "n_used"], "copy": []}
    same = {("fork", "new_refs", "refs"), ("compact", "new_table", "table"), ("compact", "new_refs", "refs")}
    before = [x.clone() for x in (s.table, s.lens, s.refs, p, m, nt, nl, nr, pm, nu, s.k, s.v)]

    def refused(name, **kw):
        fn, args = calls[name]
        with pytest.raises(tts.TtsError) as e:
            fn(*(args | kw).values())
        assert e.value.status == -1, (name, kw)

    bytes_of = lambda t: t.numel() * t.element_size()
    for name, (_, args) in calls.items():
        arrays = {k: v for k, v in args.items() if isinstance(v, torch.Tensor)}
        for w in written[name]:
            for other, t in arrays.items():
                if other == w:
                    continue
                wide = 16 if {w, other} & {"refs", "new_refs", "page_map"} else 4
                end = t.data_ptr() + (bytes_of(t) - 1) // wide * wide       # the last place that the alignment allows
                for at in (t.data_ptr(), end):
                    if (name, w, other) in same and at == t.data_ptr():
                        continue
                    refused(name, **{w: at})
        if "pools" in args:
            size = bytes_of(s.k[0])
            for w, t in arrays.items():
                for at in (s.k.data_ptr(), s.k[1].data_ptr() + size - 16, s.v[2].data_ptr() + size - 16):
                    refused(name, **{w: at})
            shifted = s.k[0].data_ptr() + 4096
            refused(name, pools=tts.TtsPools([s.k[0], shifted], [s.v[0], s.v[1]]))
            refused(name, pools=tts.TtsPools([s.v[2], s.v[0]], [s.k[0], s.v[2].data_ptr() - 4096]))
    torch.cuda.synchronize()
    bits = lambda x: x.view(torch.int16) if x.dtype == torch.bfloat16 else x
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(before, (s.table, s.lens, s.refs, p, m, nt, nl, nr, pm, nu, s.k, s.v)))
    assert s.ctx.tts_last_status() == 0
    # the same pool twice, and arrays and pools that touch, are fine
    k0, v0 = s.k.clone(), s.v.clone()
    s.ctx.tts_kv_copy_pages(tts.TtsPools([s.k[2], s.k[0], s.k[2]], [s.v[1], s.v[1], s.v[0]]), i32([3]), i32([4]), 1)
    both = torch.empty(2, 4, s.width, dtype=torch.int32, device="cuda")
    both[0] = s.table
    s.ctx.tts_kv_fork(s.pools, both[0], 32, s.lens, 4, p, 4, s.refs, both[1], nl, nr)
    torch.cuda.synchronize()
    want, copies = s.book.fork(p.tolist(), s.book.refs())
    assert s.ctx.tts_last_status() == 0 and both[1].tolist() == want.table and nr.tolist() == want.refs()
    for layer in (0, 2):
        k0[layer, 4] = k0[layer, 3]
    for layer in (0, 1):
        v0[layer, 4] = v0[layer, 3]
    for a, b in copies:
        k0[:, b], v0[:, b] = k0[:, a], v0[:, a]
    assert torch.equal(s.k, k0) and torch.equal(s.v, v0)
    s.ctx.close()


def test_fork_of_as_many_branches_as_a_context_takes():
    r = random.Random(5)
    lens = [r.randrange(0, 100) for _ in range(1024)]
    s = Setup(11, 1024, 16, lens, layers=1, hkv=1, spare=1100)
    parents = [r.randrange(-1, 1024) for _ in range(1024)]
    want, copies = s.book.fork(parents, s.book.refs())
    k0 = s.k.clone()
    assert s.fork(parents) == 0
    assert s.new_table.tolist() == want.table and s.new_lens.tolist() == want.lens and s.new_refs.tolist() == want.refs()
    for a, b in copies:
        k0[:, b] = k0[:, a]
    assert torch.equal(s.k, k0)
    s.ctx.close()
