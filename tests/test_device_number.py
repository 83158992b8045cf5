"""What the runtime says about a device is kept for that device, and not when the
question failed. The library's helper, compiled against a stand-in of the runtime."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_34867_gb300 import build as B

PROGRAM = r"""
#include "p4q_smem_limit.h"
#include <cassert>
#include <thread>
#include <vector>

static thread_local int device = 0;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }

int main() {
  p4q::DeviceNumber one;
  int asked = 0, n = -1;
  cudaError_t answer = cudaErrorInvalidValue;
  auto ask = [&](int* number) {
    ++asked;
    if (answer == cudaSuccess) *number = 10 * device;
    return answer;
  };
  for (int i = 0; i < 3; ++i) assert(one.get(&n, ask) == cudaErrorInvalidValue);  // reported and not kept
  assert(asked == 3);
  answer = cudaSuccess;
  asked = 0;
  for (int i = 0; i < 3; ++i) assert(one.get(&n, ask) == cudaSuccess && n == 0);  // (0 is an answer)
  assert(asked == 1);
  device = 1;  // another device of the process
  for (int i = 0; i < 3; ++i) assert(one.get(&n, ask) == cudaSuccess && n == 10);
  assert(asked == 2);
  device = 70;  // past the devices it keeps: asked each time
  for (int i = 0; i < 3; ++i) assert(one.get(&n, ask) == cudaSuccess && n == 700);
  assert(asked == 5);
  device = 0;
  assert(one.get(&n, ask) == cudaSuccess && n == 0 && asked == 5);
  p4q::DeviceNumber many;
  std::vector<std::thread> ts;
  for (int t = 0; t < 16; ++t)
    ts.emplace_back([&, t] {
      device = t % 4;
      for (int i = 0; i < 1000; ++i) {
        int m = -1;
        assert(many.get(&m, [](int* number) { *number = 3 + device; return cudaSuccess; }) == cudaSuccess && m == 3 + t % 4);
      }
    });
  for (auto& t : ts) t.join();
  return 0;
}
"""


def test_number_per_device_and_thread(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "number.cpp", tmp_path / "number"
    src.write_text(PROGRAM)
    inc = os.path.join(os.path.dirname(os.path.dirname(B.nvcc())), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-UNDEBUG", "-pthread", "-I", B.CSRC, "-isystem", inc, str(src), "-o",
                    str(exe)], check=True)
    subprocess.run([str(exe)], check=True, timeout=60)


def test_every_occupancy_question_is_kept_by_the_helper():
    """None is kept for the process, with what only its first device was told."""
    asks = 0
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*.cu"))):
        code = re.sub(r"//[^\n]*", "", open(path).read())
        assert "static std::atomic" not in code, path
        for m in re.finditer(r"cudaOccupancy\w+\(", code):
            before = code[:m.start()]
            # inside the lambda that a DeviceNumber is given
            assert re.search(r"\.get\(&\w+, \[[^\]]*\]\(int\* \w+\) \{[^}]*$", before), path
            asks += 1
    assert asks == 1
