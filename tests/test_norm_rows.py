"""How the norm's kernels give rows to blocks: the rules themselves, on the host, no GPU needed."""
import os
import subprocess

import pytest

from test_gpu_norm_rings import RINGS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1509_04210_b200", "csrc")

# backward, matrices, rows, columns, padded columns -> parts, warps, groups, slots, bytes of a slot, threads; backward 2: of blocks that
# load rows themselves, matrices != 0: bf16 rows that lie anyhow, and forward 3, padded columns, matrices != 0: rows that lie anyhow -> parts, warps, groups, blocks, floats of a part, threads
PROGRAM = r"""
#include <cinttypes>
#include <cstdio>
#include "norm_rows.h"

int main() {
  int back;
  unsigned matrices;
  uint64_t rows, cols, padded;
  while (std::scanf("%d %u %" SCNu64 " %" SCNu64 " %" SCNu64, &back, &matrices, &rows, &cols, &padded) == 5) {
    if (back >= 2) {
      const rudra::Split s = back == 2 ? rudra::backward_split(rows, cols, matrices != 0) : rudra::forward_split(rows, padded, matrices != 0);
      std::printf("%u %u %u %u %u %u\n", s.parts, s.warps, s.threads / 32 / s.warps, s.blocks, s.length(), s.threads);
      continue;
    }
    const rudra::Staged s(rows, cols, 2, matrices, padded, back != 0);
    if (!s.parts) std::printf("0 0 0 0 0 0\n");
    else std::printf("%u %u %u %u %u %u\n", s.parts, s.warps, s.ring.groups, s.ring.slots, s.ring.slot(), s.threads());
  }
}
"""


@pytest.fixture(scope="module")
def rings(tmp_path_factory):
    """Of (backward, matrices, rows, columns, padded columns): (parts, warps, groups, slots, bytes of a slot, threads)."""
    at = tmp_path_factory.mktemp("rows")
    (at / "t.cpp").write_text(PROGRAM)
    exe = str(at / "t")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I", CSRC, "-isystem", os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), str(at / "t.cpp"), "-o", exe])

    def ask(queries):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, map(int, q))) for q in queries), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return ask


WAYS = [(False, 1), (False, 2), (True, 2), (True, 3)]       # pass, and the matrices it reads


def test_the_rings_that_are_run_on_the_gpu_are_all_that_there_are(rings):
    for back, matrices in WAYS:
        all_ = {s[:3] for s in rings([(back, matrices, 1 << 20, c, c) for c in range(8, 16_385, 8)])}
        run = {s[:3] for s in rings([(back, matrices, t, c, c) for t, c in RINGS])}
        assert all_ == run, (back, matrices, sorted(all_ ^ run))


def test_rings_fit_their_block(rings):
    for back, matrices in WAYS:
        queries = [(back, matrices, t, c, p) for t in (444, 1_000, 10_656, 1 << 30) for c in range(8, 16_385, 8) for p in {c, -(-c // 128) * 128}]
        for (_, _, t, c, padded), (parts, warps, groups, slots, slot, threads) in zip(queries, rings(queries)):
            if not parts:
                continue
            assert parts * warps * 512 >= padded and groups * matrices * -(-2 * c // 128) * 128 == slot
            assert 2 <= slots <= 8 and slots * slot <= 216 * 1024 and t >= 444 * groups
            assert groups <= (15 if warps > 1 else 32) and threads == 32 * (groups * warps + 1)      # named barriers; a lane each
            # what the kernels are built for: 16 warps that work with 32 values to a thread, backward 24 with 16
            assert groups * warps <= (24 if back and parts == 1 else 16)
            assert groups * matrices * 2 * c < 1 << 20                # bytes that a barrier counts


def test_few_rows_and_rows_that_bulk_copies_do_not_read_go_without(rings):
    assert all(s[0] == 0 for s in rings([(back, m, t, c, c) for back, m in WAYS for t, c in ((443, 16_384), (2_000, 500), (1 << 20, 12), (1 << 20, 4_111), (1 << 20, 4_100), (100, 4_096))]))
    assert all(s[0] == 0 for s in rings([(False, 2, 1 << 20, 40_000, 40_000), (True, 3, 1 << 20, 20_000, 20_000)]))


def test_blocks_of_the_backward_pass(rings):
    for halves in (0, 1):
        queries = [(2, halves, t, c, 0) for t in (1, 7, 40, 149, 1_000, 4_000, 1 << 30) for c in list(range(1, 16_385, 13)) + [512, 4096, 4097, 5120, 5121, 8192, 8193, 16_384]]
        for (_, _, t, c, _), (parts, warps, groups, blocks, part, threads) in zip(queries, rings(queries)):
            assert parts * warps * 512 == part >= c and threads == groups * warps * 32
            assert threads <= (640 if halves and parts == 1 and 4096 < c <= 5120 else 512)
            # a part of the weight's gradient to every block, in a workspace that does not know how rows lie
            assert blocks <= 148 and part <= -(-c // 1024) * 1024
            assert groups <= (15 if warps > 1 else 32)
    # bf16 rows of nine or ten warps that lie anyhow: two to a block, as 20 warps hold them
    assert [s[2] for s in rings([(2, 1, 4_000, c, 0) for c in (4_111, 4_999, 5_120)] + [(2, 0, 4_000, 4_111, 0), (2, 1, 4_000, 4_001, 0), (2, 1, 4_000, 5_121, 0)])] == [2, 2, 2, 1, 2, 1]


def test_blocks_of_the_forward_pass(rings):
    for anyhow in (0, 1):
        queries = [(3, anyhow, t, c, p) for t in (1, 149, 4_000, 1 << 30) for c in list(range(1, 16_385, 13)) + [4096, 8192, 12_288, 12_289, 16_384] for p in {c, -(-c // 128) * 128}]
        for (_, _, t, _, padded), (parts, warps, groups, _, _, threads) in zip(queries, rings(queries)):
            assert parts * warps * 512 >= padded and threads == groups * warps * 32 and groups <= (15 if warps > 1 else 32)
            assert threads <= (1024 if anyhow else 512 if parts == 2 else 768) and not (anyhow and parts == 2)


def test_no_kernel_is_built_that_no_call_reaches():
    code = open(os.path.join(CSRC, "rms_norm.cu")).read()
    assert "norm_kernel<G, W, kSpread, 2>" not in code
    from paper_1509_04210_b200 import binding as rb
    # rows of more than 16 384 values: a token's statistics and nothing else, for the weight's gradient is written at once
    assert rb.lib().rudra_rms_norm_backward_workspace(5, 20_000) == 40 and rb.lib().rudra_rms_norm_backward_workspace(1, 2**31 - 128) == 8
