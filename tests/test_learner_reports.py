"""Who is told of kernels that gave up a wait: the host's part, no GPU needed."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1509_04210_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "reports.h"

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
  rudra::Reports r;
  CHECK(!r.fresh(0, 7, {0, 0, 0}));
  // one kernel gave up: every stream of the device is told, each once, in whatever order they ask
  CHECK(r.fresh(0, 7, {0, 1, 0}));
  CHECK(!r.fresh(0, 7, {0, 1, 0}));
  CHECK(r.fresh(0, 8, {0, 1, 0}));
  CHECK(!r.fresh(0, 8, {0, 1, 0}) && !r.fresh(0, 7, {0, 1, 0}));
  // a stream that asks for the first time too; another device's streams are not
  CHECK(r.fresh(0, 9, {0, 1, 0}));
  CHECK(!r.fresh(1, 7, {0, 0, 0}));
  // one more, in another file, between two streams' asking
  CHECK(r.fresh(0, 8, {1, 1, 0}) && r.fresh(0, 7, {1, 1, 0}) && !r.fresh(0, 8, {1, 1, 0}));
  // counts that run over are still other counts
  CHECK(r.fresh(0, 7, {0, 1, 0}));
  return 0;
}
"""


def test_no_stream_takes_anothers_report(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "t")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", CSRC, str(tmp_path / "t.cpp"), "-o", exe, "-pthread"])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout


def test_counts_are_never_set_back():
    for name in ("mx4_matmul.cu", "mx4_matmul_pair.cu", "act8_weight_grad.cu", "tensor.cuh", "learner.cu"):
        text = open(os.path.join(CSRC, name)).read()
        assert "cudaMemcpyToSymbol" not in text and "g_wait_failed =" not in text, name


def test_a_sync_waits_before_it_copies():
    # on a stream that is being captured the wait is refused, so no copy to this call's memory gets into the graph
    text = open(os.path.join(CSRC, "learner.cu")).read()
    body = text[text.index("int rudra_learner_sync("):]
    assert body.index("cudaStreamSynchronize(") < body.index("mx4_matmul_gave_up(")
