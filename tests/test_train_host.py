"""The training operators without a GPU: the oracle's pins (format, gradients
against differences), exports, and the argument checks that need no device."""
import ctypes
import importlib.util
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import build
from paper_2503_12450_gb300 import lazymar as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return lm.lib()


# --------------------------------------------------------------------------
# Oracle
# --------------------------------------------------------------------------

def test_e4m3_every_byte_decodes_and_encodes_to_itself():
    q = np.arange(256, dtype=np.uint8)
    v = T.e4m3_decode(q)
    assert v[0x7E] == 448.0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1.0
    keep = ~np.isnan(v)
    assert (T.e4m3_encode(v[keep]) == q[keep]).all()


def test_e4m3_rounds_to_the_nearest_ties_to_even():
    v = np.sort(T.e4m3_decode(np.arange(0, 0x7F, dtype=np.uint8)))
    mid = (v[1:] + v[:-1]) / 2
    q = T.e4m3_encode(mid)
    assert (q % 2 == 0).all()  # the neighbour with the even mantissa
    assert (T.e4m3_decode(T.e4m3_encode(mid * (1 + 1e-9))) == v[1:]).all()
    assert (T.e4m3_decode(T.e4m3_encode(mid * (1 - 1e-9))) == v[:-1]).all()


def test_exponent_is_the_smallest_that_holds_the_maximum():
    for a in [448.0, 448.0000001, 1.0, 3.5, 1.75, 1.7500001, 3.4e38, 1e-30, 2.0 ** -118]:
        e = int(T.exponent(a))
        assert a <= 448.0 * 2.0 ** e and (e == -126 or a > 448.0 * 2.0 ** (e - 1))
    assert int(T.exponent(0.0)) == -126 and int(T.exponent(1e-45)) == -126


def test_pack_error_is_that_of_three_mantissa_bits():
    x = np.random.default_rng(0).standard_normal((7, 300)) * np.exp2(np.arange(7) * 9.0 - 30)[:, None]
    q, s = T.pack(x)
    v = T.unpack(q, s)
    big = np.abs(x) >= np.exp2(s.astype(float) - 127 - 6)[np.arange(300) // 128].T
    assert (np.abs(v - x)[big] <= np.abs(x)[big] / 16).all()
    assert (v.astype(np.float32).view(np.uint32) & 0xFFFF == 0).all()  # exact in bf16


def _difference(f, x, h):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        d[i] = (f(a) - f(b)) / (2 * h)
    return d


def test_layernorm_gradient_against_differences():
    r = np.random.default_rng(1)
    x, dy, g, b = r.standard_normal((3, 9)), r.standard_normal((3, 9)), r.standard_normal(9), r.standard_normal(9)
    f = lambda x, g, b: float((T.layernorm(x, g, b, 1e-6)[0] * dy).sum())  # noqa: E731
    _, mean, rstd = T.layernorm(x, g, b, 1e-6)
    dx, dg, db = T.layernorm_grad(dy, x, mean, rstd, g)
    # central differences of step h: error O(h^2) + rounding 1e-16 / h
    np.testing.assert_allclose(dx, _difference(lambda v: f(v, g, b), x, 1e-5), atol=1e-8)
    np.testing.assert_allclose(dg, _difference(lambda v: f(x, v, b), g, 1e-5), atol=1e-8)
    np.testing.assert_allclose(db, _difference(lambda v: f(x, g, v), b, 1e-5), atol=1e-8)


def test_gelu_gradient_against_differences():
    x = np.linspace(-8, 8, 161)
    np.testing.assert_allclose(T.gelu_grad(x), (T.gelu(x + 1e-5) - T.gelu(x - 1e-5)) / 2e-5, atol=1e-9)


def test_gelu_polynomial_of_degree_six_within_its_bound():
    """The constants compiled into the 8-bit product's GELU, in the kernels' order of fp32 operations."""
    special = pytest.importorskip("scipy.special")
    csrc = os.path.join(ROOT, "paper_2503_12450_gb300", "csrc")
    found = dict(re.findall(r"constexpr float kGelu6P(\d) = ([-+0-9.eE]+)f;", open(os.path.join(csrc, "block8.cuh")).read()))
    c = np.array([np.float32(found[str(k)]) for k in range(7)])
    spec = importlib.util.spec_from_file_location("gen_gelu_poly", os.path.join(csrc, "gen_gelu_poly.py"))
    gen = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(gen)
    x = np.linspace(-12, 12, 200001).astype(np.float32)
    ref = 0.5 * x.astype(np.float64) * (1.0 + special.erf(x.astype(np.float64) / np.sqrt(2.0)))
    assert (np.abs(gen.gelu_fp32(x, c) - ref) <= 1.1e-7 * np.maximum(1.0, np.abs(x))).all()


# --------------------------------------------------------------------------
# Library
# --------------------------------------------------------------------------

def test_exports_every_declared_training_symbol(lib):
    text = open(os.path.join(ROOT, "include", "lazymar.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = [n for n in set(re.findall(r"\b(lazymar_[a-z0-9_]+)\s*\(", text)) if "block8" in n or "_forward" in n
             or "_backward" in n]
    assert len(names) == 11
    raw = ctypes.CDLL(lm.LIB_PATH)
    assert not [n for n in names if not hasattr(raw, n) or not hasattr(lm, n)]


def _b8(q=0, scale=0, ldq=128, lds=4):
    d = lm.lazymar_block8_desc(q or None, scale or None, ldq, lds)
    d.addr = ctypes.addressof(d)
    return d


@pytest.mark.parametrize("call,status,word", [
    (lambda L, q: L.lazymar_layernorm_forward(0, None, 8, None, None, 0, None, 8, None, None, None, None, 4, 8, 1e-6,
                                              None), 1, "no output"),
    (lambda L, q: L.lazymar_layernorm_forward(0, None, 8, None, None, 0, 16, 8, None, None, None, None, -1, 8, 1e-6,
                                              None), 1, "M >= 0"),
    (lambda L, q: L.lazymar_layernorm_forward(0, None, 8, None, None, 0, 16, 8, None, None, None, None, 4, 0, 1e-6,
                                              None), 1, "D >= 1"),
    (lambda L, q: L.lazymar_layernorm_forward(0, None, 8, None, None, 0, 16, 8, None, None, None, None, 4, 8, 0.0,
                                              None), 1, "eps"),
    (lambda L, q: L.lazymar_layernorm_forward(0, None, 9000, None, None, 0, 16, 9000, None, None, None, None, 4, 8193,
                                              1e-6, None), 6, "8192"),
    (lambda L, q: L.lazymar_layernorm_forward(2, 16, 8, None, None, 0, 16, 8, None, None, None, None, 4, 8, 1e-6,
                                              None), 1, "x:"),
    (lambda L, q: L.lazymar_layernorm_forward(0, 16, 7, None, None, 0, 16, 8, None, None, None, None, 4, 8, 1e-6,
                                              None), 1, "ldx"),
    (lambda L, q: L.lazymar_layernorm_backward(0, 16, 8, 0, None, 0, None, 16, 16, None, None, 0, 0, 16, 8, None, None,
                                               0, 4, 8, None, 0, None), 1, "exactly one"),
    (lambda L, q: L.lazymar_layernorm_backward(0, 16, 8, 0, 16, 8, q.addr, 16, 16, None, None, 0, 0, 16, 8, None, None,
                                               0, 4, 8, None, 0, None), 1, "exactly one"),
    (lambda L, q: L.lazymar_layernorm_backward(0, 16, 8, 0, 16, 8, None, 16, 16, None, None, 0, 0, 16, 8, 16, None, 0,
                                               4, 8, None, 0, None), 1, "both or neither"),
    (lambda L, q: L.lazymar_block8_pack(0, 16, 8, None, 4, 8, None), 1, "q required"),
    (lambda L, q: L.lazymar_block8_pack(0, 16, 8, q.addr, 4, 0, None), 1, "cols >= 1"),
    (lambda L, q: L.lazymar_block8_unpack(q.addr, 0, 16, 8, -1, 8, None), 1, "rows >= 0"),
    (lambda L, q: L.lazymar_block8_unpack(q.addr, 0, 16, 8, 4, 8, None), 1, "q:"),
    (lambda L, q: L.lazymar_block8_pack_weight(0, 16, 8, None, None, 4, 8, None), 1, "q or qt"),
    (lambda L, q: L.lazymar_block8_gelu_backward(0, 16, 8, None, 0, None, 0, None, None, 0, 4, 8, None, 0, None), 1,
     "no output"),
    (lambda L, q: L.lazymar_block8_linear(3, q.addr, q.addr, None, None, 0, 0, 16, 8, None, None, 4, 8, 8, None), 1,
     "epilogue"),
    (lambda L, q: L.lazymar_block8_linear(0, q.addr, q.addr, None, None, 0, 0, None, 8, None, None, 4, 8, 8, None), 1,
     "out or out8"),
    (lambda L, q: L.lazymar_block8_linear(0, q.addr, q.addr, None, None, 0, 0, 16, 8, None, q.addr, 4, 8, 8, None), 1,
     "u8 is for"),
    (lambda L, q: L.lazymar_block8_linear(0, q.addr, q.addr, None, 16, 8, 0, 16, 8, None, None, 4, 8, 8, None), 1,
     "residual is for"),
    (lambda L, q: L.lazymar_block8_linear(2, q.addr, q.addr, None, 16, 8, 1, 16, 8, None, None, 4, 8, 8, None), 1,
     "RESIDUAL"),
    (lambda L, q: L.lazymar_block8_linear(0, q.addr, q.addr, None, None, 0, 0, 16, 8, None, None, 4, 8, 0, None), 1,
     "K >= 1"),
    (lambda L, q: L.lazymar_block8_wgrad(16, 8, q.addr, 16, 8, 0, 4, 8, 0, None, 0, None), 1, "K >= 1"),
    (lambda L, q: L.lazymar_block8_wgrad(16, 8, q.addr, 16, 8, 0, (1 << 30) + 1, 8, 8, None, 0, None), 6, "2^30"),
    (lambda L, q: L.lazymar_block8_pack(0, 16, 8, q.addr, (1 << 30) + 1, 8, None), 6, "2^30"),
])
def test_refusals_before_touching_the_device(lib, call, status, word):
    q = _b8()
    assert call(lib, q) == status
    assert word in lib.lazymar_last_error().decode()


def test_empty_calls_succeed_without_a_device(lib):
    q = _b8()
    assert lib.lazymar_layernorm_forward(0, None, 8, None, None, 0, 16, 8, None, None, None, None, 0, 8, 1e-6, None) == 0
    assert lib.lazymar_block8_pack(0, None, 8, q.addr, 0, 8, None) == 0
    assert lib.lazymar_block8_unpack(q.addr, 0, None, 8, 0, 8, None) == 0
    assert lib.lazymar_block8_pack_weight(0, None, 8, q.addr, None, 0, 8, None) == 0
    assert lib.lazymar_block8_linear(0, q.addr, q.addr, None, None, 0, 0, 16, 8, None, None, 0, 8, 8, None) == 0
    assert lib.lazymar_block8_wgrad(None, 8, q.addr, None, 8, 0, 4, 0, 8, None, 0, None) == 0


def test_workspaces_cover_small_and_large_sizes(lib):
    assert lm.lazymar_layernorm_backward_workspace(0, 768) == 0
    assert lm.lazymar_layernorm_backward_workspace(1, 768) == 2 * 768 * 4
    assert lm.lazymar_layernorm_backward_workspace(40960, 1280) <= 8 << 20
    assert lm.lazymar_block8_gelu_backward_workspace(0, 768) == 0
    assert lm.lazymar_block8_gelu_backward_workspace(40960, 5120) <= 16 << 20


def test_weight_pack_refuses_more_columns_than_it_counts(lib):
    q = _b8()
    for k in ((1 << 30) + 1, (1 << 31) - 1):
        assert lib.lazymar_block8_pack_weight(0, 16, k, q.addr, None, 8, k, None) == 6
        assert "2^30" in lib.lazymar_last_error().decode()


def test_descriptor_takes_rows_of_bytes_only():
    torch = pytest.importorskip("torch")
    q, scale = torch.zeros((8, 256), dtype=torch.uint8), torch.zeros((2, 8), dtype=torch.uint8)
    d = lm.lazymar_block8(q, scale)
    assert (d.ldq, d.lds) == (256, 8)
    d = lm.lazymar_block8(q[:, :128].view(torch.float8_e4m3fn), scale[:1])
    assert (d.ldq, d.lds) == (256, 8)
    d = lm.lazymar_block8(q[:0], scale[:, :0])
    assert d.ldq == 256
    for bad_q, bad_scale in ((q.float(), scale), (q, scale.float()), (q[:, ::2], scale), (q, scale[:, ::2]),
                             (q.t(), scale), (q, scale.t()), (q[0], scale), (q, scale[0])):
        with pytest.raises(lm.LazymarError, match="bytes"):
            lm.lazymar_block8(bad_q, bad_scale)


def test_empty_tensors_without_an_address_are_fine(lib):
    q = _b8()
    assert lib.lazymar_layernorm_forward(0, None, 8, None, None, 0, None, 8, None, None, None, None, 0, 8, 1e-6, None) == 0
    for epilogue in (0, 1, 2):
        assert lib.lazymar_block8_linear(epilogue, q.addr, q.addr, None, None, 8, 0, None, 8, None, None, 0, 8, 8, None) == 0
        assert lib.lazymar_block8_linear(epilogue, q.addr, q.addr, None, None, 8, 0, None, 8, None, None, 4, 0, 8, None) == 0
    # what cannot be meant is refused all the same
    assert lib.lazymar_block8_linear(2, q.addr, q.addr, None, None, 8, 1, None, 8, None, None, 0, 8, 8, None) == 1
    assert lib.lazymar_block8_linear(0, q.addr, None, None, None, 8, 0, None, 8, None, None, 0, 8, 8, None) == 1


def test_in_place_needs_the_same_layout(lib):
    q = _b8()
    for dtype, ld in ((0, 8), (1, 16)):
        assert lib.lazymar_block8_gelu_backward(1, 16, 8, None, dtype, 16, ld, None, None, 0, 4, 8, None, 0, None) == 1
        assert "in place" in lib.lazymar_last_error().decode()
    assert lib.lazymar_block8_linear(2, q.addr, q.addr, None, 16, 8, 0, 16, 16, None, None, 4, 8, 8, None) == 1
    assert "in place" in lib.lazymar_last_error().decode()


def test_layernorm_backward_in_place_of_the_residual_needs_its_layout(lib):
    """dx over dres as bf16, or in rows further apart, would overwrite rows of dres that are still to be read."""
    def call(dx_dtype, lddx, M=4):
        return lib.lazymar_layernorm_backward(1, 32, 8, 1, 64, 8, None, 128, 256, None, 16, 8, dx_dtype, 16, lddx, None,
                                              None, 0, M, 8, None, 0, None)
    for dx_dtype, lddx, M in ((1, 8, 4), (1, 16, 4), (0, 16, 4), (1, 8, 1)):
        assert call(dx_dtype, lddx, M) == 1
        assert "in place" in lib.lazymar_last_error().decode()
    for lddx, M in ((8, 4), (16, 1)):  # its own layout: refused only for what is no device memory here
        assert call(0, lddx, M) == 1
        assert "in place" not in lib.lazymar_last_error().decode()


def test_layernorm_in_place_of_its_input_needs_the_same_layout(lib):
    """y over x, dx over dy or x: another type or stride would overwrite rows that are still to be read."""
    def forward(dtype, ldy, M=4):
        return lib.lazymar_layernorm_forward(1, 16, 8, None, None, dtype, 16, ldy, None, None, None, None, M, 8, 1e-6, None)

    def backward(dy, x, dtype, lddx, M=4):
        return lib.lazymar_layernorm_backward(1, dy, 8, 1, x, 8, None, 128, 256, None, None, 0, dtype, 16, lddx, None, None,
                                              0, M, 8, None, 0, None)
    for f in (forward, lambda *a: backward(16, 32, *a), lambda *a: backward(32, 16, *a)):
        for dtype, ld, M, refused in ((0, 8, 4, True), (1, 16, 4, True), (1, 8, 4, False), (1, 16, 1, False)):
            assert f(dtype, ld, M) == 1
            assert ("in place" in lib.lazymar_last_error().decode()) == refused, (dtype, ld, M)


def _host_program(tmp_path, source):
    """Compiles C++ that includes the library's host headers and returns what it prints."""
    src, exe = tmp_path / "host.cpp", tmp_path / "host"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2503_12450_gb300", "csrc"), str(src), "-o", str(exe)], check=True, timeout=120)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=120).stdout


def test_product_in_parts_of_k_fits_the_device(tmp_path):
    """A launch with K in parts has one cluster a tile, all at once, on devices with fewer SMs too; and parts are still
    chosen on a whole one."""
    text = _host_program(tmp_path, r"""
#include <cstdio>
#include <initializer_list>
#include "linear8_shape.h"
int main() {
  for (int sms : {2, 8, 20, 60, 76, 100, 127, 132, 152})
    for (int M : {33, 100, 128, 300, 500, 1000, 4000})
      for (int N : {1, 128, 250, 1024, 1280, 2048, 5120})
        for (int K : {1, 128, 512, 1024, 2048, 4096, 16384}) {
          const lm::l8::Shape s = lm::l8::choose(sms, M, N, K);
          std::printf("%d %d %d %d %d %d %lld\n", sms, M, N, K, (int)s.pair, s.parts, s.tiles);
        }
}
""")
    split = 0
    for line in text.splitlines():
        sms, M, N, K, pair, parts, tiles = map(int, line.split())
        t = 256 if pair else 128
        assert tiles == -(-M // t) * -(-N // t)
        if parts > 1:
            assert not pair and parts in (2, 4, 8) and tiles * parts <= min(sms, 128), line
            split += sms == 152
    assert split >= 20


def test_absent_tensors_do_not_take_the_product_off_whole_accesses(tmp_path):
    """Without a residual its stride says nothing about the output's rows."""
    text = _host_program(tmp_path, r"""
#include <cstdio>
#include "linear8_shape.h"
int main() {
  using lm::l8::rows_on_four;
  void* const p = reinterpret_cast<void*>(uintptr_t(1024));
  void* const q = reinterpret_cast<void*>(uintptr_t(1024 + 8));
  std::printf("%d%d%d%d %d%d%d%d", rows_on_four(nullptr, 7, 4), rows_on_four(nullptr, 0, 2), rows_on_four(p, 8, 4),
              rows_on_four(q, 8, 2), rows_on_four(q, 8, 4), rows_on_four(p, 7, 4), rows_on_four(p, 6, 2),
              rows_on_four(nullptr, 8, 4));
}
""")
    assert text == "1111 0001"
    source = open(os.path.join(ROOT, "paper_2503_12450_gb300", "csrc", "k_linear8.cu")).read()
    assert "rows_on_four(x.out.p" in source and "rows_on_four(x.residual.p" in source


def test_missing_tensors_are_not_taken_for_calls_in_place(lib):
    q = _b8()
    assert lib.lazymar_layernorm_forward(0, None, 8, None, None, 1, None, 0, q.addr, None, None, None, 4, 8, 1e-6, None) == 1
    assert "x:" in lib.lazymar_last_error().decode() and "in place" not in lib.lazymar_last_error().decode()
    assert lib.lazymar_layernorm_backward(1, None, 8, 0, None, 0, q.addr, 16, 16, None, None, 0, 0, None, 8, None, None, 0,
                                          4, 8, None, 0, None) == 1
    assert "dy:" in lib.lazymar_last_error().decode()
