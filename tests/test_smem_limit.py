"""The shared-memory limit of a kernel, set by threads that launch it at different sizes.

The host code is compiled against a stand-in for the CUDA runtime whose attribute calls the test
can hold up, so no GPU takes part."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNTIME = r"""
#pragma once
#include <stddef.h>
typedef int cudaError_t;
typedef void* cudaStream_t;
enum { cudaSuccess = 0, cudaErrorInvalidDevice = 101 };
enum cudaFuncAttribute { cudaFuncAttributeMaxDynamicSharedMemorySize = 8 };
cudaError_t cudaGetDevice(int* dev);
cudaError_t cudaFuncSetAttribute(void (*kern)(), cudaFuncAttribute attr, int value);
"""

PROGRAM = r"""
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>

#include "internal.h"

static std::atomic<int> limit{0}, inside{0}, second_done{0};
static bool hold = false;
cudaError_t cudaGetDevice(int* dev) { *dev = 0; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(void (*)(), cudaFuncAttribute, int value) {
  if (hold && value == 100) {  // the first thread's call takes effect late
    inside = 1;
    for (int i = 0; i < 300 && !second_done; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
  }
  limit = value;
  return cudaSuccess;
}
static void kernel() {}
static size_t set_one[wm::kSmemOptDevices], set_many[wm::kSmemOptDevices];

int main() {
  hold = true;
  std::thread a([] { wm::opt_in_smem(kernel, 100, set_one); });
  while (!inside) std::this_thread::yield();
  std::thread b([] { wm::opt_in_smem(kernel, 200, set_one); second_done = 1; });
  a.join();
  b.join();
  std::printf("two: limit %d recorded %zu\n", limit.load(), set_one[0]);
  if (limit < 200 || set_one[0] != (size_t)limit.load()) return 1;
  if (wm::opt_in_smem(kernel, 150, set_one) != cudaSuccess || limit < 200) return 2;

  hold = false;
  limit = 0;
  std::atomic<int> below{0};
  std::vector<std::thread> all;
  for (int t = 0; t < 8; ++t)
    all.emplace_back([t, &below] {
      unsigned x = 12345u + t;
      for (int i = 0; i < 20000; ++i) {
        x = x * 1664525u + 1013904223u;
        const int want = 1000 + i + (int)(x >> 24);
        if (wm::opt_in_smem(kernel, want, set_many) != cudaSuccess || limit < want) ++below;
      }
    });
  for (auto& t : all) t.join();
  std::printf("many: %d launches would have been under their size\n", below.load());
  return below == 0 ? 0 : 3;
}
"""


def test_the_limit_is_never_below_a_size_that_a_thread_was_granted(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    (tmp_path / "cuda_runtime.h").write_text(RUNTIME)
    (tmp_path / "main.cc").write_text(PROGRAM)
    exe = tmp_path / "limit"
    subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", f"-I{tmp_path}", f"-I{ROOT}/include",
                    f"-I{ROOT}/paper_2608_18486_gb300/csrc", str(tmp_path / "main.cc"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
