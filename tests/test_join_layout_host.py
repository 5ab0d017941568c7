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


def test_no_piece_of_a_row_is_copied_from_outside_its_tensor(tmp_path):
    """Pieces of 256 columns, rounded to 16-byte units, at all alignments: those that would reach outside the tensor's bytes
    are told apart, the last row's one but last among them, where the last has fewer bytes than fill the unit (257 to 262
    columns of two bytes, 257 and 258 of four); and no others are."""
    text = _host_program(tmp_path, r"""
#include <cstdio>
#include <initializer_list>
#include "join_host.h"
int main() {
  int wrong = 0, inner = 0;
  for (int e : {1, 2, 4})
    for (int D : {1, 3, 8, 255, 256, 257, 258, 259, 262, 263, 264, 511, 513, 777, 1281})
      for (int pad : {0, 1, 3, 8})
        for (int offset = 0; offset < 16; offset += e)
          for (int M : {1, 2, 306}) {
            const uintptr_t base = 4096 + offset;
            const size_t pitch = (size_t)(D + pad) * e;
            const uintptr_t end = lm::rows_end(base, M - 1, pitch, D, e);
            for (int row : {0, 1, M / 2, M - 2, M - 1})
              for (int c0 = 0; c0 < D && row >= 0 && row < M; c0 += 256) {
                const int n = (D - c0 < 256 ? D - c0 : 256) * e;
                const uintptr_t p = base + row * pitch + (size_t)c0 * e;
                const uintptr_t from = p / 16 * 16, to = (p + n + 15) / 16 * 16;
                const bool out = from < base || to > base + (M - 1) * pitch + (size_t)D * e;
                wrong += out != lm::piece_reaches_out(p, n, base, end);
                inner += out && c0 + 256 < D;
              }
          }
  std::printf("%d %d", wrong, inner > 0);
}
""")
    assert text == "0 1"
    source = open(os.path.join(ROOT, "paper_2503_12450_gb300", "csrc", "join_rows.cuh")).read()
    assert "piece_reaches_out(p, bytes, lowest, tensor_end)" in source
    assert "tensor_end = rows_end(lowest, stream_row(magic, shift, M - 1), pitch, D, t.e)" in source


def test_rings_wait_for_their_copies_before_a_kernel_leaves_them():
    """A warp whose wait has run out leaves the loop over its rows with copies under way; each kernel with a ring waits for
    them, with a limit, before it returns or uses the rings' memory for sums. (What follows a wait that ran out is
    not run on a GPU: nothing makes one run out without a fault.)"""
    csrc = os.path.join(ROOT, "paper_2503_12450_gb300", "csrc")
    for name, after in (("join_ring.cuh", "template <int WPR, bool PLAIN, bool STREAMED>\ncudaError_t join_ring_run"),
                        ("join_grad.cuh", "float* const mem = reinterpret_cast<float*>(rings);")):
        source = open(os.path.join(csrc, name)).read()
        assert source.count("ring.wait(") == 1
        at = source.index("if (dead) drain_ring(plan, bars);")
        assert source.index("ring.wait(") < at < source.index(after)
        loop = source[source.index("ring.wait("):at]
        assert "return;" not in loop and "break;" not in loop
    rows = open(os.path.join(csrc, "join_rows.cuh")).read()
    assert "for (int i = 0; i < 500 && !mbar_try_wait(&bars[s], now); ++i) {}" in rows
