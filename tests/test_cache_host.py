"""CPU checks of the cache operators: what the library and its binding refuse without a GPU, the layout of the
rotary struct, and the plain implementations that the GPU tests compare with, pinned on cases small enough to
work out another way."""
import ctypes
import math
import random
import re
from pathlib import Path

import pytest
import torch

import cache_plain
import paper_2505_19634_b200 as tts
from paper_2505_19634_b200.binding import TtsPools, TtsRope
from paper_2505_19634_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def test_null_contexts_are_refused():
    lib, z = tts.load_library(), ctypes.c_void_p(0)
    assert lib.tts_chunk_reserve(z, 16) == -1
    assert lib.tts_chunk_attn(z, z, 1024, z, z, z, 16, z, z, 1, 1, z, z) == -1
    assert lib.tts_kv_append_rope(z, z, z, 1024, z, z, 256, z, z, z, z, 16, z, z, 1, 1, z) == -1
    assert lib.tts_kv_copy_pages(z, 1, z, z, z, z, 1) == -1
    assert lib.tts_kv_fork(z, 1, z, z, z, 16, z, 1, z, 1, z, z, z, z) == -1
    assert lib.tts_kv_grow(z, z, 16, z, z, 1, z) == -1
    assert lib.tts_kv_free(z, z, z, z, 1, z) == -1
    assert lib.tts_kv_compact(z, 1, z, z, z, 1, z, z, z, z, z) == -1


def test_the_status_of_too_few_pages_has_words():
    assert "page" in tts.tts_strerror(-7) and tts.tts_strerror(-7) != tts.tts_strerror(-4)


def test_rotary_struct():
    rope = TtsRope([0, 1, 2, 1], [1.0, 0.5, 0.25, 0.125], interleaved=True)
    assert ctypes.sizeof(rope) == 592 and TtsRope.axis.offset == 12 and TtsRope.inv_freq.offset == 80      # as a C compiler lays it out
    assert (rope.n_axes, rope.n_pairs, rope.interleaved) == (3, 4, 1)
    assert list(rope.axis[:4]) == [0, 1, 2, 1] and list(rope.inv_freq[:4]) == [1.0, 0.5, 0.25, 0.125]


@pytest.mark.parametrize("axis,freq", [([], []), ([0] * 65, [1.0] * 65), ([0, 0], [1.0]), ([-1], [1.0]), ([8], [1.0])])
def test_rotary_struct_refuses(axis, freq):
    with pytest.raises(ValueError):
        TtsRope(axis, freq)


def test_pools_come_in_pairs():
    a, b = torch.zeros(4), torch.zeros(4)
    pools = TtsPools([a, b], [b, a])
    assert pools.n_layers == 2 and pools.k[0] == a.data_ptr() == pools.v[1]
    with pytest.raises(ValueError):
        TtsPools([a, b], [a])


@pytest.mark.parametrize("hq,hkv,chunk,lens,prefix", [(2, 1, [3, 1, 0], [5, 17, 2], 16), (4, 2, [4], [3], 0), (1, 1, [2, 2], [40, 2], 0)])
def test_plain_attention_against_one_row_at_a_time(hq, hkv, chunk, lens, prefix):
    c = cache_plain.Cache(hq, hkv, chunk, lens, prefix=prefix, seed=3, device="cpu", first_row=1, rows_behind=2)
    out, lse, mean = cache_plain.chunk_attention(c)
    for row in range(c.total_rows):
        b = next((b for b in range(c.n) if c.starts[b] <= row < c.starts[b + 1]), None)
        for h in range(hq):
            if b is None:
                assert not out[row, h].any()
                continue
            seen = prefix + lens[b] - chunk[b] + (row - c.starts[b]) + 1
            weights, values = [], []
            for t in range(max(0, seen)):
                page, at = c.rows[b][t // 16], t % 16
                weights.append(math.exp(float(c.q[row, h].double() @ c.k[page, h * hkv // hq, at].double()) / math.sqrt(128)))
                values.append(c.v[page, h * hkv // hq, at].double())
            if not weights:
                assert not out[row, h].any() and lse[row, h] == -math.inf
                continue
            total = sum(weights)
            want = sum(w * v for w, v in zip(weights, values)) / total
            torch.testing.assert_close(out[row, h], want, rtol=1e-12, atol=1e-12)
            torch.testing.assert_close(mean[row, h], sum(w * v.abs() for w, v in zip(weights, values)) / total, rtol=1e-12, atol=1e-12)
            assert abs(float(lse[row, h]) - math.log(total)) < 1e-12


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs", [64, 20, 1])
def test_plain_rotation_is_one_of_the_plane(interleaved, pairs):
    """Every pair is a complex number times exp(i angle); lengths stay, dims behind the pairs too, and the product of a
    query and a key depends on the difference of their positions alone."""
    gen = torch.Generator().manual_seed(1)
    x, y = torch.randn(5, 2, 128, generator=gen), torch.randn(5, 2, 128, generator=gen)
    r = random.Random(2)
    axis, freq = [r.randrange(3) for _ in range(pairs)], [r.uniform(0, 1) for _ in range(pairs)]
    pos = torch.randint(0, 1000, (3, 5), generator=gen)
    got = cache_plain.rope_turn(x, pos, axis, freq, interleaved)
    lo = torch.tensor([2 * i if interleaved else i for i in range(pairs)])
    hi = lo + (1 if interleaved else pairs)
    angle = torch.stack([pos[axis[i]].double() * freq[i] for i in range(pairs)], -1)[:, None]
    want = torch.complex(x[..., lo].double(), x[..., hi].double()) * torch.polar(torch.ones_like(angle), angle)
    torch.testing.assert_close(torch.complex(got[..., lo], got[..., hi]), want, rtol=1e-12, atol=1e-12)
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:].double())
    dots = [(cache_plain.rope_turn(x, pos + d, axis, freq, interleaved) * cache_plain.rope_turn(y, pos + 7 + d, axis, freq, interleaved)).sum(-1) for d in (0, 431)]
    torch.testing.assert_close(dots[0], dots[1], rtol=1e-9, atol=1e-9)


def test_plain_fork():
    """Branch 0: 16 shared + 20 own tokens (pages 0, 3, 5); branch 1: 16 + 16 (pages 0, 4); branch 2 is dropped."""
    book = cache_plain.Book([[0, 3, 5, -1], [0, 4, -1, -1], [0, 7, -1, -1]], 16, [20, 16, 9], 10)
    refs = book.refs()
    assert refs == [3, 0, 0, 1, 1, 1, 0, 1, 0, 0]
    children, copies = book.fork([1, 0, 0, 1, -1, 0], refs)
    assert children.table == [[0, 4, -1, -1], [0, 3, 5, -1], [0, 3, 1, -1], [0, 4, -1, -1], [-1] * 4, [0, 3, 2, -1]]
    assert children.lens == [16, 20, 20, 16, 0, 20] and copies == [(5, 1), (5, 2)]
    assert children.refs() == [5, 1, 1, 3, 2, 1, 0, 0, 0, 0]
    assert book.fork([0] * 8, refs) is None                     # seven copies, five free pages


def test_every_wait_of_the_chunk_attention_is_bounded():
    """A warp may leave the kernel's loop on its own when a wait somewhere has run out, so no other may be waiting for it at
    a barrier without a limit; the two block-wide ones are where all warps begin and where all end."""
    source = (Path(tts.library_path()).parent / "csrc" / "chunk_attn.cu").read_text()
    code = "\n".join(line.split("//")[0] for line in source.splitlines())
    assert "barrier.cta" not in code and "bar.sync" not in code and "bar.red" not in code
    assert code.count("__syncthreads") == 2
    assert "try_wait" not in code                               # mbar_wait alone, which has the limit


def test_the_chunk_attention_waits_for_what_it_has_in_flight_when_it_gives_up():
    """Each warp that starts copies or products waits for them with a word of its own: a wait given up in one of them must
    not cut another's short."""
    source = (Path(tts.library_path()).parent / "csrc" / "chunk_attn.cu").read_text()
    words = re.findall(r"Abort(?: quiet)?\{(misc \+ [^,]*),", source)
    assert sorted(words) == ["misc + 2 + is_v", "misc + 6", "misc + 7"]
    assert source.index("umma_commit(bar(DRAINED))") < source.index("tcgen05.dealloc")


@pytest.mark.parametrize("name", ["chunk_attn.cu", "chunk_plan.cu", "rope_append.cu", "kv_pages.cu"])
def test_kernels_that_start_early_read_coherently(name):
    """Blocks of a programmatic dependent are resident while the kernel before it writes: the read-only path, which const and
    __restrict__ together or __ldg allow, is for data that nothing writes meanwhile."""
    source = (Path(tts.library_path()).parent / "csrc" / name).read_text()
    assert "launch_dependent(" in source and not re.search(r"__restrict__|__ldg\(|ld\.global\.nc", source)
