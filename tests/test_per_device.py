"""What a launch remembers of a device (how many clusters it holds) is remembered for that device alone.  The
helper runs on the host, against a cudaGetDevice of the test's own."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2605_28396_b200" / "csrc"

PROGRAM = r"""
#include "adwin_internal.h"
#include <cstdio>

static int current = 0, asked = 0;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = current; return current < 0 ? cudaErrorNoDevice : cudaSuccess; }

int main() {
  static std::atomic<int> table[adwin::kKnownDevices];
  auto get = [&](int dev, int answer, cudaError_t rc) {
    current = dev;
    int v = -1;
    const cudaError_t e = adwin::per_device(table, v, [&](int& x) { ++asked; x = answer; return rc; });
    return e == cudaSuccess ? v : -(int)e;
  };
  bool ok = get(0, 70, cudaSuccess) == 70 && asked == 1;
  ok = ok && get(1, 60, cudaSuccess) == 60 && asked == 2;         // another device is asked for itself
  ok = ok && get(0, 5, cudaSuccess) == 70 && get(1, 5, cudaSuccess) == 60 && asked == 2;
  ok = ok && get(2, 9, cudaErrorInvalidConfiguration) == -(int)cudaErrorInvalidConfiguration && asked == 3;
  ok = ok && get(2, 8, cudaSuccess) == 8 && asked == 4;           // a failure is not remembered
  ok = ok && get(200, 3, cudaSuccess) == 3 && get(200, 4, cudaSuccess) == 4 && asked == 6;
  ok = ok && get(-1, 7, cudaSuccess) == -(int)cudaErrorNoDevice && asked == 6;
  std::puts(ok ? "ok" : "wrong");
  return ok ? 0 : 1;
}
"""


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="no nvcc")
def test_an_answer_is_kept_for_the_device_that_gave_it(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    # (without the CUDA runtime library: nothing else of it is called)
    subprocess.run(["nvcc", "-std=c++17", "--cudart=none", f"-I{CSRC}", str(tmp_path / "t.cpp"), "-o",
                    str(tmp_path / "t")], check=True, capture_output=True, text=True)
    assert subprocess.run([str(tmp_path / "t")], capture_output=True, text=True).stdout == "ok\n"
