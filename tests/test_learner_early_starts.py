"""Rules of all kernels that are set up while the kernel before them still writes, under whichever of its two names they are launched, and of
every header that they read memory through; no GPU needed."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1509_04210_b200", "csrc")


def _code(name):
    """A source file without its comments."""
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _early():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and re.search(r"\blaunch_(after|overlapped)\(", _code(f)))


def _headers():
    """What those files include of this folder, and what that includes."""
    found, todo = set(), _early()
    while todo:
        for name in re.findall(r'#include "([\w.]+)"', _code(todo.pop())):
            if name not in found and os.path.exists(os.path.join(CSRC, name)):
                found.add(name)
                todo.append(name)
    return sorted(found)


def test_the_attribute_is_asked_for_in_one_place():
    users = [f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h", ".cpp")) and "ProgrammaticStreamSerialization" in _code(f)]
    assert users == ["launch.cuh"] and _code("launch.cuh").count("cudaLaunchKernelEx(") == 1
    assert _early() == ["act8.cu", "act8_weight_grad.cu", "fp8.cu", "fp8_matmul.cu", "fp8_matmul_pair.cu", "grad_clip.cu", "mx4.cu", "mx4_matmul.cu", "mx4_matmul_pair.cu", "rms_norm.cu"]
    assert {"blocks.cuh", "fp8.cuh", "launch.cuh", "pairs.cuh", "tensor.cuh", "vec.cuh"} <= set(_headers())


def test_the_servers_loads_stay_with_the_server():
    # vec.cuh has loads for kernels that are launched the ordinary way
    assert all(not re.search(r"(GradUnit|F8|ld8)\b", _code(f)) for f in _early() + _headers() if f != "vec.cuh")


@pytest.mark.parametrize("name", _early())
def test_every_kernel_waits_for_the_one_before(name):
    code = _code(name)
    kernels = len(re.findall(r"__global__", code))
    assert kernels and kernels == code.count("await_previous_kernel();") == code.count("admit_next_kernel();") and "<<<" not in code


@pytest.mark.parametrize("name", _early() + [f for f in _headers() if f != "vec.cuh"])
def test_what_the_kernel_before_writes_is_not_read_as_read_only(name):
    # neither by such a load, which may be moved above the wait, nor by an assembler load that may be
    code = _code(name)
    assert not re.findall(r"__ldg\b|__ldcs\b|__ldcg\b|__ldca\b|__restrict__|ld\.global\.nc", code)
    for asm in re.findall(r"asm[^;]*?\"[^;]*?ld\.global.*?;\s*(?=\n)", code, flags=re.S):
        assert "volatile" in asm[:20] and '"memory"' in asm, asm
