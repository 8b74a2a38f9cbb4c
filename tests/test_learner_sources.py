"""Rules of the learner-side kernels that hold by how they are written: checked on their source, no GPU needed."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1509_04210_b200", "csrc")


def _code(name):
    """A source file without its comments."""
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _started_early():
    """Files with kernels that are set up while the kernel before them still writes."""
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "launch_after(" in _code(f))


def test_kernels_that_start_early_are_known():
    assert _started_early() == ["act8.cu", "act8_weight_grad.cu", "mx4.cu", "mx4_matmul.cu", "mx4_matmul_pair.cu"]


@pytest.mark.parametrize("name", _started_early() + ["blocks.cuh", "tensor.cuh"])
def test_what_the_kernel_before_writes_is_not_read_as_read_only(name):
    # Such a load promises that nobody writes there while the kernel runs, and may be moved above the wait for the
    # kernel before, which still writes; so may an assembler load that is not volatile.
    code = _code(name)
    assert not re.findall(r"__ldg\b|__ldcs\b|__ldcg\b|__ldca\b|__restrict__|ld\.global\.nc", code)
    for asm in re.findall(r"asm[^;]*?\"[^;]*?ld\.global.*?;\s*(?=\n)", code, flags=re.S):
        assert "volatile" in asm[:20] and '"memory"' in asm, asm


def test_waits_are_those_of_whole_warps():
    # the one wait in use asks all lanes; nothing else tries a barrier
    assert all("barrier_try(" not in _code(f) for f in _started_early())
    body = _code("tensor.cuh").split("bool barrier_wait(")[1].split("\n}")[0]
    assert body.count("barrier_try(") == body.count("all_lanes(barrier_try(") == 2


@pytest.mark.parametrize("name,loaders", [("mx4_matmul.cu", 1), ("mx4_matmul_pair.cu", 1), ("act8_weight_grad.cu", 2)])
def test_loading_warps_end_with_their_copies_landed(name, loaders):
    # whichever warp gives up, and also where the loading warp itself came to its end: its last copies are waited for
    # before the block may end, under no condition but that of a pair, whose first block waits for both
    code = _code(name)
    ends = re.findall(r"[^\n]*\bawait_copies\(", code)
    assert len(ends) == loaders and code.count("barrier_expect(") == loaders
    for line in ends:
        assert re.fullmatch(r"\s*(if \((!PAIR \|\| )?rank == 0\) )?await_copies\(", line), line
