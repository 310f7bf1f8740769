"""A kernel's attributes belong to a device: what sets them runs on each device, and again where it has failed (csrc/once.h)."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include <cstdio>
#include "once.h"

enum Error { kSuccess = 0, kFailed = 2 };

int main() {
  cdsl::OncePerDevice once, other;             // of two kernels
  int calls[70] = {};
  auto step = [&](cdsl::OncePerDevice& o, int device, Error e) {
    return o(device, [&] { ++calls[device]; return e; });
  };
  bool ok = step(once, 0, kFailed) == kFailed && calls[0] == 1;            // a failure is told
  ok = ok && step(once, 0, kSuccess) == kSuccess && calls[0] == 2;         // and not kept
  ok = ok && step(once, 0, kFailed) == kSuccess && calls[0] == 2;          // done
  ok = ok && step(once, 1, kSuccess) == kSuccess && calls[1] == 1;         // another device
  ok = ok && step(once, 63, kSuccess) == kSuccess && step(once, 63, kFailed) == kSuccess && calls[63] == 1;
  ok = ok && step(other, 0, kSuccess) == kSuccess && calls[0] == 3;        // another kernel
  for (int i = 0; i < 2; ++i) ok = ok && step(once, 64 + 4, kSuccess) == kSuccess;
  ok = ok && calls[68] == 2;
  std::puts(ok ? "ok" : "wrong");
}
"""


def test_once_per_device(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no g++")
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2412_10418_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "ok\n"


def test_no_attribute_is_set_once_in_a_process():
    """Results of CUDA calls in function-local statics are of the device that was current at the first call."""
    src = os.path.join(ROOT, "paper_2412_10418_gb300", "csrc")
    for name in sorted(os.listdir(src)):
        with open(os.path.join(src, name)) as f:
            assert "static const cudaError_t" not in f.read(), name
