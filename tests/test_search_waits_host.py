"""CPU checks of the sources of the search operators' kernels: every wait has its limit, a kernel that gives up waits for what it has in flight,
and kernels that start early read coherently."""
import re
from pathlib import Path

import paper_2505_19634_b200 as tts


def source(name):
    text = (Path(tts.library_path()).parent / "csrc" / name).read_text()
    return "\n".join(line.split("//")[0] for line in text.splitlines())


def roles():
    """The kernel for many rows, cut into its roles."""
    code = source("kv8_attn_wide.cu")
    code = code[code.index("kv8_attn_wide_kernel(const"):]
    cuts = [code.index(x) for x in ("if (warp >= kSoftmaxWarps && warp < kMmaWarp)", "else if (warp == kLoadWarp)", "else if (warp == kMmaWarp)",
                                    "else if (warp < kSoftmaxWarps)", "tcgen05.dealloc")]
    return {name: code[a:b] for name, a, b in zip(("convert", "load", "mma", "softmax"), cuts, cuts[1:])}


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
