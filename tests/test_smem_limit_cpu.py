"""How a kernel's limit of dynamic shared memory is raised (ensure_dynamic_smem in csrc/common.cuh) where two host threads do so at once:
compiled for the host, with the runtime's call replaced by one that holds the threads where they can undo each other's work."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>

#include "common.cuh"

namespace {
std::mutex m;
std::condition_variable cv;
int limit = 0, calls = 0;           // the kernel's limit, calls that set it
bool wide_set = false, narrow_set = false;
constexpr int kWide = 160 * 1024, kNarrow = 60 * 1024, kBetween = 100 * 1024;
}  // namespace

// The wide thread sets its limit, and comes back only when the narrow one has set its own, or after a while.
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  std::unique_lock<std::mutex> hold(m);
  limit = bytes, ++calls;
  if (bytes == kWide) {
    wide_set = true, cv.notify_all();
    cv.wait_for(hold, std::chrono::milliseconds(500), [] { return narrow_set; });
  } else if (bytes == kNarrow) {
    narrow_set = true, cv.notify_all();
  }
  return cudaSuccess;
}

int main() {
  struct Tag {};
  const void* kernel = nullptr;
  int seen = 0;
  std::thread wide([&] { if (approxifer::ensure_dynamic_smem<Tag>(kernel, 0, kWide) != cudaSuccess) seen = -1; });
  std::thread narrow([&] {
    {
      std::unique_lock<std::mutex> hold(m);
      cv.wait(hold, [] { return wide_set; });
    }
    if (approxifer::ensure_dynamic_smem<Tag>(kernel, 0, kNarrow) != cudaSuccess) seen = -1;
  });
  wide.join(), narrow.join();
  const int both = limit;
  if (approxifer::ensure_dynamic_smem<Tag>(kernel, 0, kBetween) != cudaSuccess) seen = -1;
  std::printf("%d %d %d %d\n", both, limit, calls, seen);
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_two_threads_never_lower_a_kernels_limit(tmp_path):
    from paper_2109_09868_b200 import build

    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc()))), "include")
    source, program = tmp_path / "limit.cpp", tmp_path / "limit"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-pthread", "-I", build.CSRC, "-I", build.INCLUDE, "-isystem", cuda, str(source), "-o", str(program)], check=True, timeout=300)
    both, after, calls, seen = map(int, subprocess.run([str(program)], check=True, capture_output=True, text=True, timeout=60).stdout.split())
    assert seen == 0
    assert both == 160 * 1024 and after == both  # what the wide call needs, and what any later call up to it does
    assert calls == 1
