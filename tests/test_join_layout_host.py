"""What the residual join's host code lays out, without a GPU: workspaces, the pieces that its rings copy."""
import os
import subprocess

import pytest

from paper_2503_12450_gb300 import build
from paper_2503_12450_gb300 import lazymar as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return lm.lib()


def _host_program(tmp_path, source):
    """Compiles C++ that includes the library's host headers and returns what it prints."""
    src, exe = tmp_path / "host.cpp", tmp_path / "host"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2503_12450_gb300", "csrc"),
                    str(src), "-o", str(exe)], check=True, timeout=120)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=120).stdout


def test_gradient_sums_lie_on_their_boundary_in_any_workspace(lib, tmp_path):
    """Vectors of eight floats need boundaries of 32 bytes; a workspace may start on any of 16, and its size has room for
    the step between them (152 CTAs' four sums of a column with one modulation for all rows or for each)."""
    for group in (0, 1):
        for D in (8, 777, 1280):
            assert lm.lazymar_join_grad_workspace(40960, D, group) >= 4 * 152 * D * 4 + 16
    text = _host_program(tmp_path, r"""
#include <cstdio>
#include <initializer_list>
#include "join_host.h"
int main() {
  bool good = true;
  for (uintptr_t at = 4096; at < 4096 + 256; at += 16)
    for (size_t floats : {size_t(4), size_t(4 * 152 * 777), size_t(1) << 33}) {
      const uintptr_t from = reinterpret_cast<uintptr_t>(lm::join_sums_at(reinterpret_cast<void*>(at)));
      good = good && from % 32 == 0 && from >= at && from + 4 * floats <= at + lm::join_sums_bytes(floats);
    }
  std::printf("%d", good);
}
""")
    assert text == "1"
    source = open(os.path.join(ROOT, "paper_2503_12450_gb300", "csrc", "train_api.cu")).read()
    assert "p.ws = join_sums_at(a->workspace)" in source
