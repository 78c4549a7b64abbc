"""A kernel's limit of dynamic shared memory under calls from several threads, with a function of the test's own in place of the device's (no GPU)."""
import subprocess

from paper_2503_01840_b200 import build

PROGRAM = r"""
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "common.cuh"
int main() {
  int lost = 0, sets = 0, refused = 0;
  for (int round = 0; round < 200; round++) {
    spec::SmemLimit limit;
    std::atomic<int> attribute{0}, calls{0}, short_of{0}, ready{0};
    auto set = [&](int size) {                  // as the device's: the last one counts; slow, so that others come in between
      calls++;
      std::this_thread::sleep_for(std::chrono::microseconds(50 + size % 7 * 20));
      if (size > 200000) return false;
      attribute = size;
      return true;
    };
    std::vector<std::thread> threads;
    for (int t = 0; t < 8; t++)
      threads.emplace_back([&, t] {
        ready++;
        while (ready < 8) std::this_thread::yield();
        for (int i = 0; i < 4; i++) {
          const int size = 50000 + (t * 37 + i * 11 + round) % 8 * 10000;
          if (!limit.raise(0, size, set) || attribute < size) short_of++;      // the launch that follows would fail
        }
        if (limit.raise(0, 300000, set)) short_of++;
      });
    for (auto &t : threads) t.join();
    lost += short_of;
    const int before = calls;
    if (!limit.raise(0, 50000, set) || calls != before) lost++;                // what has been set is not set again
    if (!limit.raise(1, 50000, set) || calls != before + 1) lost++;            // another device
    if (!limit.raise(64, 50000, set) || !limit.raise(64, 50000, set) || calls != before + 3) lost++;      // one that is not remembered
    sets += calls, refused += limit.raise(0, 300000, set) ? 1 : 0;
  }
  printf("%d %d", lost, refused);
}
"""


def test_threads_with_different_sizes_never_lower_the_limit(tmp_path):
    src, exe = tmp_path / "limits.cu", tmp_path / "limits"
    src.write_text(PROGRAM)
    subprocess.run([build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, timeout=120).stdout == b"0 0"
