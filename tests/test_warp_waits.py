"""A warp that gives up a bounded wait gives it up together.  Reads of tensor memory, shuffles and __syncwarp name all 32 lanes of a warp: lanes
that wait one by one, or read the abort flag one by one, may part when a wait runs out, and the others then wait for them for good.
That cannot be tried without risking just that, so the sources are read: a wait of a single thread stands only in code that one lane
runs, and a loop of a whole warp asks the abort flag for all its lanes at once."""
import os
import re

import pytest

from paper_2603_06626_b200.build import CSRC

SOURCES = ["gemm.cu", "fp8_gemm.cu", "fp8_small.cu", "linear_small.cu", "route.cu"]
ONE_LANE = re.compile(r"\b(lane|threadIdx\.x) == 0\b")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", lambda m: re.sub(r"[^\n]", " ", m.group()), text, flags=re.S)


def _headers(text, at):
    """What stands before each brace that is open at this place, innermost first."""
    depth, found = 0, []
    for i in range(at - 1, -1, -1):
        if text[i] == "}":
            depth += 1
        elif text[i] == "{":
            if depth == 0:
                start = max(text.rfind(c, 0, i) for c in "{};")
                if text[:i].rstrip().endswith(")"):                # a for loop's header holds semicolons
                    n, j = 0, len(text[:i].rstrip()) - 1
                    while j >= 0:
                        n += {")": 1, "(": -1}.get(text[j], 0)
                        if n == 0:
                            break
                        j -= 1
                    start = max(text.rfind(c, 0, j) for c in "{};")
                found.append(text[start + 1:i])
            else:
                depth -= 1
    return found


def _by_one_lane(text, at):
    return any(ONE_LANE.search(h) and "else" not in h.split("(")[0] for h in _headers(text, at))


def faults(text):
    bad = []
    for m in re.finditer(r"\bmbar_wait_bounded\(", text):
        if not _by_one_lane(text, m.start()):
            bad.append((text.count("\n", 0, m.start()) + 1, "a wait of single lanes"))
    for m in re.finditer(r"\b(for|while) \(", text):
        n, end = 1, m.end()
        while n:
            n += {"(": 1, ")": -1}.get(text[end], 0)
            end += 1
        header = text[m.start():end]
        if "abort_flag" in header and not re.search(r"__any_sync\(0xffffffffu, \*abort_flag\)", header) and not _by_one_lane(text, m.start()):
            bad.append((text.count("\n", 0, m.start()) + 1, "a loop whose lanes ask for themselves"))
    return bad


@pytest.mark.parametrize("name", SOURCES)
def test_warps_give_up_together(name):
    text = _code(name)
    kernel_of_one_thread = text.find("wait_selftest_kernel(")          # one thread, nothing to part from
    found = faults(text if kernel_of_one_thread < 0 else text[:kernel_of_one_thread])
    assert not found, found


def test_every_source_that_reads_tensor_memory_is_looked_at():
    assert sorted(SOURCES) == sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "tmem_ld_wait" in _code(f))


def test_the_reading_tells_the_forms_apart():
    one = "if (lane == 0) {\n for (int i = 0; i < n && !*abort_flag; ++i) { if (!ptx::mbar_wait_bounded(b)) break; } }"
    assert not faults(one)
    assert not faults("for (; pick() && !__any_sync(0xffffffffu, *abort_flag); ++n) { ptx::mbar_wait_bounded_warp(b); }")
    assert [k for _, k in faults("for (; t < n && !*abort_flag; ++t) {\n ptx::mbar_wait_bounded(b); }")] == [
        "a wait of single lanes", "a loop whose lanes ask for themselves"]
    assert faults("if (lane == 0) { f(); } else { ptx::mbar_wait_bounded(b); }")
