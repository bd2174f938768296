"""CPU checks of the search operators: what the library and its binding refuse without a GPU, and the plain implementations
that the GPU tests compare with, pinned another way."""
import ctypes
import math
import re
from pathlib import Path

import pytest
import torch

import kv8_plain as k8
import paper_2505_19634_b200 as tts
from paper_2505_19634_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def test_null_contexts_are_refused():
    lib, z = tts.load_library(), ctypes.c_void_p(0)
    none = ctypes.POINTER(ctypes.c_void_p)()
    assert lib.tts_kv8_append(z, 0, z, z, 0, z, z, 256, z, z, z, 0, z, z, 1, 1, z) == -1
    assert lib.tts_kv8_read(z, 0, z, z, z, 1, z, z, 1) == -1
    assert lib.tts_kv8_attn(z, 0, z, 1024, z, z, 0, z, z, 1, 1, z, z) == -1
    assert lib.tts_kv8_copy_pages(z, 1, none, z, z, 1) == -1
    assert lib.tts_kv8_fork(z, 1, none, z, 0, z, 1, z, 1, z, z, z, z) == -1
    assert lib.tts_kv8_compact(z, 1, none, z, 1, z, z, z, z, z) == -1
    assert lib.tts_beam_reserve(z, 1, 1) == -1
    assert lib.tts_beam_select(z, z, 0, 8, 8, z, z, 0, 1, 1, 1, z, z, z) == -1
    assert lib.tts_beam_reorder(z, 1, none, none, ctypes.POINTER(ctypes.c_int64)(), z, 1, 1) == -1


def test_lists_of_arrays():
    a, b = torch.zeros(4), torch.zeros(4)
    assert tts.TtsKv8Pools([a, b]).p[1] == b.data_ptr()
    states = tts.TtsStates([a], [b], [16])
    assert (states.n, states.src[0], states.dst[0], states.row_bytes[0]) == (1, a.data_ptr(), b.data_ptr(), 16)
    with pytest.raises(ValueError):
        tts.TtsStates([a], [b], [16, 16])


def test_the_record_is_what_the_header_says():
    header = (Path(tts.library_path()).parent.parent / "include" / "tts.h").read_text()
    assert int(re.search(r"#define TTS_KV8_RECORD (\d+)", header)[1]) == tts.KV8_RECORD == k8.RECORD == 2 * 16 * 128 + 2 * 16 * 4


def test_plain_codes_are_torchs():
    """The table of e4m3, and rounding to nearest with ties to even, against torch's own conversion of values in range."""
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    torch.testing.assert_close(k8.table(k8.E4M3), every.view(torch.float8_e4m3fn).double(), rtol=0, atol=0, equal_nan=True)
    assert torch.equal(k8.table(k8.INT8), every.view(torch.int8).double())
    gen = torch.Generator().manual_seed(1)
    x = torch.cat((torch.randn(40, 128, generator=gen) * torch.exp(3 * torch.randn(40, 1, generator=gen)),
                   torch.arange(-448, 448, 7.).view(1, 128), torch.arange(-64, 64).view(1, 128) / 2.0 ** 10, torch.zeros(1, 128)))
    one = torch.ones(x.shape[0])
    assert torch.equal(k8.codes(x.clamp(-448, 448), one, k8.E4M3), x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    assert torch.equal(k8.codes(x.clamp(-127, 127), one, k8.INT8), x.clamp(-127, 127).round().to(torch.int8).view(torch.uint8))


@pytest.mark.parametrize("fmt", [k8.E4M3, k8.INT8])
def test_plain_records_are_a_rearrangement(fmt):
    gen = torch.Generator().manual_seed(2)
    code = torch.randint(0, 256, (3, 2, 2, 16, 128), generator=gen, dtype=torch.uint8)
    scale = torch.rand(3, 2, 2, 16, generator=gen)
    rec = k8.pack(code[..., 0, :, :], code[..., 1, :, :], scale[..., 0, :], scale[..., 1, :])
    back, s = k8.unpack(rec)
    assert torch.equal(back, code) and torch.equal(s, scale)
    # every token's codes are one line of 128 bytes, and no chunk's place is taken twice
    for t in range(16):
        assert sorted(k8.place(t, c) for c in range(8)) == list(range(8))
        assert sorted(rec[0, 0, 128 * t:128 * t + 128].tolist()) == sorted(code[0, 0, 0, t].tolist())
    del fmt


@pytest.mark.parametrize("fmt,worst", [(k8.E4M3, 2.0 ** -4), (k8.INT8, 0.5 / 127)])
def test_quantisation_error_is_half_a_step(fmt, worst):
    """e4m3: 2^-4 of the value or half its smallest step, 2^-10 of the scale; int8: half a scale."""
    x = torch.randn(200, 128, generator=torch.Generator().manual_seed(3))
    s = k8.scales(x, fmt)
    off = (k8.table(fmt)[k8.codes(x, s, fmt).long()] * s.double()[:, None] - x.double()).abs()
    limit = torch.maximum(x.double().abs() * worst, s.double()[:, None] * 2.0 ** -10) if fmt == k8.E4M3 else s.double()[:, None] * 0.5
    assert (off <= limit * (1 + 1e-6)).all()


def test_plain_visibility():
    assert k8.sees(3, 5).int().tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 1, 1]]
    assert k8.sees(3, 2).int().tolist() == [[0, 0], [1, 0], [1, 1]]
    assert k8.sees(4, 5, [-1, 0, 0, 2]).int().tolist() == [[1, 1, 0, 0, 0], [1, 1, 1, 0, 0], [1, 1, 0, 1, 0], [1, 1, 0, 1, 1]]


def test_plain_attention_one_row_at_a_time():
    c = k8.Cache8(k8.INT8, 2, [20, 3], prefix=16, seed=4, device="cpu")
    q = torch.randn(4, 4, 128, generator=torch.Generator().manual_seed(5)).bfloat16()
    out, lse, bound, _ = k8.attention(c, q, 2)
    for b in range(2):
        for i in range(2):
            for h in range(4):
                k, v = (x[h // 2] for x in c.kv(b))
                seen = c.prefix + c.lens[b] - 1 + i
                w = [math.exp(float(q[2 * b + i, h].double() @ k[t]) / math.sqrt(128)) for t in range(seen)]
                torch.testing.assert_close(out[2 * b + i, h], sum(x * v[t] for t, x in enumerate(w)) / sum(w), rtol=1e-12, atol=1e-12)
                assert abs(float(lse[2 * b + i, h]) - math.log(sum(w))) < 1e-12
    assert (bound > 0).all()


def test_plain_selection_by_brute_force():
    gen = torch.Generator().manual_seed(6)
    logits = torch.randint(-3, 3, (6, 5), generator=gen).float()
    logits[1, 2] = -math.inf
    logits[4] = -math.inf
    scores, finished = torch.tensor([-1.0, -2.0, -math.inf, -1.0, -3.0, -0.5]), torch.tensor([0, 0, 0, 0, 0, 1])
    got = k8.select(logits, scores, finished, 3, 2, 3, 12)
    p = torch.log_softmax(logits.double(), -1)
    for g in range(2):
        every = []
        for r in range(3 * g, 3 * g + 3):
            if r == 5:
                every.append((0.5, r, 3))
            elif r not in (2, 4):
                every += [(-float(scores[r] + p[r, t]), r, t) for t in range(5) if logits[r, t] > -math.inf]
        every.sort(key=lambda e: (round(e[0], 12), e[1], e[2]))
        assert [(r, t) for r, t, _ in got[g] if r >= 0] == [(r, t) for _, r, t in every[:12]]
        assert all(x == (-1, -1, -math.inf) for x in got[g][len(every):])


@pytest.mark.parametrize("name", ["kv8_attn.cu", "kv8_read.cu", "beam.cu"])
def test_kernels_that_start_early_read_coherently(name):
    """Blocks of a programmatic dependent are resident while the kernel before it writes: no read-only loads."""
    source = (Path(tts.library_path()).parent / "csrc" / name).read_text()
    assert "launch_dependent(" in source and not re.search(r"__restrict__|__ldg\(|ld\.global\.nc", source)


def test_every_wait_of_the_attention_over_the_8bit_cache_is_bounded():
    """A warp waits for its own copies alone, through mbar_wait, which has the limit; a warp that gave up works on to the block's barriers, and
    waits in the end for what it has in flight with a word of its own."""
    source = (Path(tts.library_path()).parent / "csrc" / "kv8_attn.cu").read_text()
    code = "\n".join(line.split("//")[0] for line in source.splitlines())
    assert code.count("mbar_wait(") == 2 and not re.search(r"try_wait|test_wait|barrier\.cta|bar\.sync", code)
    assert re.findall(r"Abort quiet\{(flags \+ [^,]*),", code) == ["flags + 1 + warp"]
    assert "break" not in code[code.index("for (bool more_items"):code.index("if (!alive)")].replace("if (r >= kRows) break", "")
