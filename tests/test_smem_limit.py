"""The bookkeeping behind calls that raise a kernel's shared-memory limit: two host threads whose first calls
need different sizes, with a stand-in for the CUDA call that makes them meet inside it."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_08252_b200", "csrc")

PROGRAM = r"""
#include <chrono>
#include <thread>
#include <stdio.h>
#include "smem_limit.h"
using namespace std::chrono;

int main() {
  int bad = 0;
  for (int round = 0; round < 6; ++round) {
    rest::SmemLimits<2, 3> limits;
    std::atomic<size_t> limit{0};            // what the kernel allows
    std::atomic<int> inside{0}, calls{0};
    auto call = [&](size_t bytes, int wait_ms) {
      const int e = limits.ensure(1, 2, bytes, [&]() -> int {
        ++calls;
        ++inside;
        // give the other thread time to come in as well, then let the larger size be set first
        for (int i = 0; i < 50 && inside < 2; ++i) std::this_thread::sleep_for(milliseconds(1));
        std::this_thread::sleep_for(milliseconds(wait_ms));
        limit = bytes;
        return 0;
      });
      if (e != 0 || limit < bytes) ++bad;    // a launch with `bytes` would fail
    };
    std::thread large([&] { call(200, 0); });
    std::thread small([&] { call(60, 40); });
    large.join();
    small.join();
    call(200, 0);
    call(60, 0);
    if (calls > 2) ++bad;                    // remembered, whichever came first
  }
  rest::SmemLimits<2, 3> limits;             // an error is passed on and nothing is remembered
  int calls = 0;
  if (limits.ensure(0, 0, 10, [&] { ++calls; return 7; }) != 7) ++bad;
  if (limits.ensure(0, 0, 10, [&] { ++calls; return 0; }) != 0 || calls != 2) ++bad;
  if (limits.ensure(5, 0, 10, [&] { ++calls; return 3; }) != 3 || calls != 3) ++bad;      // a device that has no place
  printf("%d\n", bad);
  return bad != 0;
}
"""


def test_two_threads_that_need_different_sizes(tmp_path):
    src, exe = tmp_path / "limits.cpp", tmp_path / "limits"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert got.returncode == 0, got.stdout
