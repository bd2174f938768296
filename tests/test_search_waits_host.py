"""CPU checks of the sources of the search operators' kernels: every wait has its limit, a kernel that gives up waits for what it has in flight,
and kernels that start early read coherently."""
import re
from pathlib import Path

import pytest

import paper_2505_19634_b200 as tts


def source(name):
    text = (Path(tts.library_path()).parent / "csrc" / name).read_text()
    return "\n".join(line.split("//")[0] for line in text.splitlines())


@pytest.mark.parametrize("name", ["kv8_attn_wide.cu", "rope_append.cu", "kv_pages.cu"])
def test_kernels_that_start_early_read_coherently(name):
    code = source(name)
    assert "launch_dependent(" in code and not re.search(r"__restrict__|__ldg\(|ld\.global\.nc", code)


def roles():
    """The kernel for many rows, cut into its roles."""
    code = source("kv8_attn_wide.cu")
    code = code[code.index("kv8_attn_wide_kernel(const"):]
    cuts = [code.index(x) for x in ("if (warp >= kSoftmaxWarps && warp < kMmaWarp)", "else if (warp == kLoadWarp)", "else if (warp == kMmaWarp)",
                                    "else if (warp < kSoftmaxWarps)", "tcgen05.dealloc")]
    return {name: code[a:b] for name, a, b in zip(("convert", "load", "mma", "softmax"), cuts, cuts[1:])}


def test_every_wait_of_the_kernel_for_many_rows_is_bounded():
    """Through mbar_wait, which has the limit, or in the load warp's one loop, which has it too and looks at the flag."""
    code = source("kv8_attn_wide.cu")
    assert len(re.findall(r"try_wait|test_wait", code)) == 1 and code.count("mbar_test(") == 2
    part = roles()
    # (a wait's first argument, and who is told that it ran out)
    assert re.findall(r"mbar_wait\((.*), (ab|quiet|Abort\{.*?\})\)", code) == [
        ("bar(i), parity", "ab"), ("bar(full0 + i % ring), i / ring & 1", "quiet"), ("bar(i), parity", "ab"), ("bar(DRAINED), 0", "Abort{misc + 4, p.status}"),
        ("bar(i), parity", "ab"), ("bar(PART_DONE), parts_left & 1", "ab")]
    loop = part["load"][part["load"].index("for (int spin"):part["load"].index("Abort quiet")]
    assert "mbar_test(" in loop and "now - since > kWaitLimitNs" in loop and "*ab.flag = 1" in loop and "*ab.flag != 0)) break" in loop
    for name in ("convert", "load", "mma"):                         # no barrier that a warp that left would be missed at
        assert not re.search(r"bar_sync_id|bar_red_or|__syncthreads", part[name])


def test_the_warps_of_a_row_meet_however_a_wait_ends():
    """The softmax warps meet at barriers, so that none leaves its loops early: no return, and no break but behind the last row of a join."""
    part = roles()["softmax"]
    assert "return" not in re.sub(r"auto place = .*", "", part)
    assert re.findall(r"if \([^\n]*\) break", part) == ["if (warp * 16 + g + i >= rows) break"] and part.count("break") == 1
    assert re.findall(r"continue", part) == ["continue"] * 2 and "if (idle) { warp_arrive(bar(P_FULL + st), lane); continue; }" in part and "if (!valid) continue;" in part
    # a pair of warps is idle or not as a whole, and only those that are not meet
    assert part.count("bool idle = (warp & 3) * 32 >= rows") == 1


def test_what_is_in_flight_is_waited_for_at_the_end_of_every_run():
    """Copies and products, with words of their own and not only where a wait has run out already: a warp may give up after these have ended
    their loops."""
    part = roles()
    end = part["load"][part["load"].index("for (int spin"):]
    end = end[end.index("\n        }\n"):]
    assert re.sub(r"\s+", " ", end).startswith(" } const Abort quiet{misc + 3, p.status}; for (int i = max(0, n - ring); i < n; ++i) { misc[3] = 0; mbar_wait(")
    end = part["mma"][part["mma"].index("for (bool more_items"):]
    end = end[end.index("\n        }\n"):]
    assert re.sub(r"\s+", " ", end).startswith(" } if (elect_one()) { misc[4] = 0; umma_commit(bar(DRAINED)); } __syncwarp(); mbar_wait(bar(DRAINED), 0,")
