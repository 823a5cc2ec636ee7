"""Waits that run out, read in the microscaled kernels' source (no GPU run makes one end early): a warp that runs instructions of the whole
warp behind a wait comes to one answer in all lanes, or goes on whatever the answer is. Where lanes were told different things and some
left a loop for it, the others would wait in such an instruction for them."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_03298_b200", "csrc")
WHOLE_WARP = r"_sync\(|warp_arrive\(|tmem_load|take_sum|bar\.sync|cluster\(\)|meet\(|\.aligned"

# the part of the warps that issue matrix instructions: (file, where it begins, where it ends)
ISSUING = [("enec_micro_many.cu", "} else if (warp < kFirstX) {", "} else if (warp < kFirstW) {"),
           ("enec_micro_both.cu", "} else if (warp == 1) {", "} else {"),
           ("enec_micro_pieces.cuh", "} else if (warp == 1) {", "    } else {\n        uint32_t group")]


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _parts(name, begin, end):
    text = _source(name)
    a = text.index(begin)
    b = text.index(end, a + len(begin))
    return text[a:b], text[:a] + text[b:]


def test_the_wait_of_a_warp_has_one_answer():
    text = _source("enec_micro_mma.cuh")
    assert re.search(r"bool warp_wait\(.*?return __all_sync\(0xFFFFFFFFu, suspended_wait\(", text, re.S)
    assert re.search(r"bool warp_failed\(.*?return __any_sync\(0xFFFFFFFFu, \*flag\)", text, re.S)
    # a wait lane by lane sets the flag and gives no answer
    assert re.search(r"void wait_or_fail\([^{}]*{\s*if \(!mbar_try_wait\(bar, parity\) && !suspended_wait\(bar, parity, flag\)\) \*flag = 1;\s*}", text)
    assert text.count("suspended_wait(") == 2


def test_every_file_with_waits_is_looked_at():
    with_waits = {f for f in os.listdir(CSRC) if f.startswith("enec_micro") and re.search(r"(suspended_wait|warp_wait|wait_or_fail|mbar_wait_bounded)\(", _source(f))}
    assert with_waits == {name for name, _, _ in ISSUING} | {"enec_micro_mma.cuh"}


@pytest.mark.parametrize("name, begin, end", ISSUING)
def test_only_issuing_warps_leave_lane_by_lane(name, begin, end):
    issuing, others = _parts(name, begin, end)
    assert "mma_" in issuing and "tcgen05_commit" in issuing and "suspended_wait(" in issuing
    assert "suspended_wait(" not in others and "warp_wait(" in others
    # in the issuing part instructions of the whole warp stand behind a __syncwarp() only, and the part ends with one
    assert issuing.rstrip().endswith("__syncwarp();")
    rest = re.sub(r"__syncwarp\(\);\s*if \(lockstep\) meet\(i\);", "", issuing)
    assert not re.search(WHOLE_WARP, rest), re.search(WHOLE_WARP, rest).group(0)


@pytest.mark.parametrize("name, begin, end", ISSUING)
def test_the_flag_divides_no_warp(name, begin, end):
    """Outside the issuing part the flag of a CTA that gives up is set, reported by a thread, or read by a whole warp; where a thread reads
    it for itself, stores depend on it and nothing else: those places are listed."""
    _, others = _parts(name, begin, end)
    alone = {"enec_micro_many.cu": ["if (failed) report(", "if (threadIdx.x < 512 && good && !failed && row < job.s.rows) {"],
             "enec_micro_both.cu": ["if (failed && threadIdx.x == 0) report("], "enec_micro_pieces.cuh": ["const bool ok = !sh.failed;"]}[name]
    for line in others.split("\n"):
        line = re.sub(r"(sh\.)?failed = [01];|&(sh\.)?failed|warp_failed|volatile int failed;|wait_or_fail", "", line)
        assert not re.search(r"\bfailed\b", line) or any(a in line for a in alone), line


@pytest.mark.parametrize("name", ["enec_micro_few.cu", "enec_micro_moe.cu"])
def test_what_a_task_says_lane_by_lane_guards_stores_only(name):
    """`ok` of a task's sums: in `take` a condition of a store; in `after` a way out, behind which stands no instruction of the whole warp."""
    text = _source(name)
    for found in re.finditer(r"\bok\b", text):
        line = text[text.rindex("\n", 0, found.start()) + 1:text.index("\n", found.start())]
        if "bool ok" in line or re.fullmatch(r"\s*(} else )?if \([^()]*(\([^()]*\))*[^()]*\bok && row < [\w.]+\)( {)?", line):
            continue
        assert line.strip() == "if (!last || !good || !ok) return;"
        assert not re.search(WHOLE_WARP, text[found.end():text.index("false, [](uint32_t) {});", found.end())])
