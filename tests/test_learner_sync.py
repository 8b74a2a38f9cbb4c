"""What rudra_learner_sync costs and shares between calls at the same time."""
import os
import re
import subprocess
import threading

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1509_04210_b200", "csrc")

PROGRAM = r"""
#include <atomic>
#include <cstdio>
#include <thread>
#include <vector>
#include "reports.h"

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
  rudra::Places places;
  {
    std::vector<int> all;
    for (int i = 0; i < rudra::Places::kMost; ++i) all.push_back(places.take());
    for (int i = 0; i < rudra::Places::kMost; ++i) CHECK(all[i] == i);
    const rudra::Places::Place none(places);
    CHECK(none.number == -1 && places.take() == -1);
    places.give(17);
    const rudra::Places::Place one(places);
    CHECK(one.number == 17 && places.take() == -1);
    for (int i : all) if (i != 17) places.give(i);
  }
  // what a call has nobody else has
  std::atomic<int> users[rudra::Places::kMost] = {};
  std::atomic<int> twice{0}, without{0};
  std::vector<std::thread> threads;
  for (int t = 0; t < 80; ++t)
    threads.emplace_back([&] {
      for (int i = 0; i < 2000; ++i) {
        const rudra::Places::Place mine(places);
        if (mine.number < 0) { ++without; continue; }
        if (users[mine.number]++) ++twice;
        --users[mine.number];
      }
    });
  for (auto& t : threads) t.join();
  CHECK(twice == 0);
  for (int i = 0; i < rudra::Places::kMost; ++i) CHECK(places.take() == i);
  return 0;
}
"""


def test_places_are_one_calls_at_a_time(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "t")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC, str(tmp_path / "t.cpp"), "-o", exe, "-pthread"])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout


def test_one_copy_brings_all_counts():
    # to ordinary memory of the host every copy waits for itself
    text = open(os.path.join(CSRC, "learner.cu")).read()
    body = text[text.index("cudaError_t gather("):text.index('extern "C"')]
    files = [f for f in os.listdir(CSRC) if f.endswith(".cu") and "__device__ uint32_t g_gave_up;" in open(os.path.join(CSRC, f)).read()]
    assert len(re.findall(r"_count\(&at\.of\[\d\]\)", body)) == len(files) and body.count("cudaMemcpyFromSymbolAsync(") == 1


@pytest.mark.gpu
def test_calls_at_the_same_time():
    import torch
    from paper_1509_04210_b200 import learner as L

    L.sync()
    failed = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                x = torch.ones(64, 64 + i, device="cuda")
                for _ in range(50):
                    q = L.fp8_quantize(x)
                    L.sync()
                    if not bool((L.fp8_dequantize(q, torch.float32) == 1).all()):
                        failed.append(i)
        except Exception as exc:      # noqa: BLE001
            failed.append(exc)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(70)]      # more than there are places
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
