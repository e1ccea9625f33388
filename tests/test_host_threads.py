"""Host code that several threads may be in at once, against a fake of the CUDA calls it makes.  No GPU."""
import os
import subprocess

from paper_2609_25405_b200 import build

# A thread that enables a small size is held inside the call until one that wants a large size has had time to make its own.
PROGRAM = r"""
#include "hb_internal.h"
#include <chrono>
#include <cstdio>
#include <thread>

static std::atomic<int> enabled{0}, inside{0}, calls{0};
extern "C" cudaError_t cudaGetDevice(int* dev) { *dev = 3; return cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  ++calls;
  inside = 1;
  if (bytes < 100000) std::this_thread::sleep_for(std::chrono::milliseconds(300));
  if (bytes > 200000) return cudaErrorInvalidValue;
  enabled = bytes;
  return cudaSuccess;
}
int main() {
  static DynSmemState st;
  int rc[2] = {-9, -9};
  std::thread small([&] { rc[0] = hb_ensure_dyn_smem(nullptr, st, 60000); });
  while (!inside) std::this_thread::yield();
  std::thread large([&] { rc[1] = hb_ensure_dyn_smem(nullptr, st, 150000); });
  small.join();
  large.join();
  const int n = calls;
  const int again = hb_ensure_dyn_smem(nullptr, st, 140000);   // what a launch in between needs
  const int refused = hb_ensure_dyn_smem(nullptr, st, 250000), kept = hb_ensure_dyn_smem(nullptr, st, 150000);
  std::printf("%d %d %d %d %d %d %d", rc[0], rc[1], again, enabled.load(), calls.load() - n, refused, kept);
}
"""


def test_a_smaller_launch_does_not_take_back_what_a_larger_one_enabled(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-w", "-I", os.path.join(cuda, "include"), "-I", build.CSRC, str(src), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.split()
    # the size that is enabled is the larger one; 140000 needed no call, 250000 one that failed and changed nothing
    assert out == ["0", "0", "0", "150000", "1", "-2", "0"]
