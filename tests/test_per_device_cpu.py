"""What the library keeps about a device is kept for that device: the host code is
compiled against a stand-in of the runtime's current device."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "internal.h"

static int current = 0, failing = 0;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = current; return failing ? cudaErrorInvalidDevice : cudaSuccess; }

int main() {
  static normpre::PerDevice known;
  int asked = 0, refuse = 0;
  auto get = [&](int device) {
    int v = -1;
    current = device;
    const cudaError_t e = known.get(&v, [&](int* n) {
      ++asked;
      if (refuse) return cudaErrorUnknown;
      *n = 10 * device;
      return cudaSuccess;
    });
    std::printf("%d:%d:%d ", static_cast<int>(e != cudaSuccess), v, asked);
  };
  refuse = 1; get(1);                        // an error is not kept
  refuse = 0; get(1); get(0); get(1); get(0);   // zero is a value like others
  get(64); get(64); get(1000);               // beyond the table: asked each time
  failing = 1; get(1);
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++") or not os.path.exists("/usr/local/cuda/include/cuda_runtime.h"),
                    reason="needs g++ and the CUDA headers")
def test_values_are_kept_per_device(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I/usr/local/cuda/include",
                    "-I" + os.path.join(ROOT, "paper_2609_36692_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["1:-1:1", "0:10:2", "0:0:3", "0:10:3", "0:0:3", "0:640:4", "0:640:5", "0:10000:6", "1:-1:6"]
