"""Parity of the training operators with the fp64 oracle (oracle/training.py),
through the C ABI, at the sizes, strides, types and values where they can go wrong."""
import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import lazymar as lm
from _gpu import DT, torch_cuda

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24          # half an ulp of fp32
BF = 2.0 ** -8          # half an ulp of bf16, relative to the value's binade
E4 = 2.0 ** -4          # half an ulp of E4M3


def sync():
    torch_cuda().cuda.synchronize()
    lm.lazymar_device_check()


def rng(*key):
    return np.random.default_rng(list(key))


def dev(a, dtype="fp32", pad=0, offset=0):
    """A device tensor [rows, cols] whose rows are cols + pad apart and start `offset` elements into the buffer,
    the gaps filled with NaN; and the values it holds, in fp64."""
    torch = torch_cuda()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows, cols = a.shape
    buf = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=t, device="cuda")
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda())
    return v, v.double().cpu().numpy()


def out(rows, cols, dtype="fp32", pad=0, offset=0):
    return dev(np.full((rows, cols), np.nan, np.float32), dtype, pad, offset)[0]


def vec(a):
    torch = torch_cuda()
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


class Held:
    """A block8 tensor on the device; the bytes outside it are 0xAB."""

    def __init__(self, rows, cols, more=0, lds=None, scale_rows=None):
        torch = torch_cuda()
        self.rows, self.cols = rows, cols
        nb, sr = -(-cols // 128), rows if scale_rows is None else scale_rows
        self.q = torch.full((rows, -(-cols // 16) * 16 + more), 0xAB, dtype=torch.uint8, device="cuda")
        self.scale = torch.full((nb, (sr if lds is None else lds)), 0xAB, dtype=torch.uint8, device="cuda")
        self.sr = sr
        self.d = lm.lazymar_block8(self.q, self.scale)

    def set(self, q, scale):
        torch = torch_cuda()
        self.q[:, :self.cols] = torch.from_numpy(q).cuda()
        self.scale[:, :self.sr] = torch.from_numpy(scale).cuda()
        return self

    def get(self):
        q, s = self.q.cpu().numpy(), self.scale.cpu().numpy()
        assert (q[:, self.cols:] == 0xAB).all() and (s[:, self.sr:] == 0xAB).all(), "written outside the tensor"
        return q[:, :self.cols], s[:, :self.sr]


def held(x, **kw):
    h = Held(*x.shape, **kw).set(*T.pack(x))
    return h, T.unpack(*h.get())


def held_weight(w, **kw):
    h = Held(*w.shape, scale_rows=-(-w.shape[0] // 128), **kw).set(*T.pack_weight(w))
    return h, T.unpack_weight(*h.get())


def bytes_equal(a, b):
    """E4M3 bytes, any NaN equal to any."""
    nan = (b & 0x7F) == 0x7F
    assert ((a & 0x7F) == 0x7F)[nan].all()
    assert (a[~nan] == b[~nan]).all()


def close(got, want, bound):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else got
    assert got.shape == want.shape
    assert not np.isnan(got).any()
    bad = np.abs(got - want) > bound
    assert not bad.any(), "%d of %d off, worst %.3g of its bound" % (
        bad.sum(), bad.size, (np.abs(got - want) / np.broadcast_to(bound, want.shape)).max())


def close8(h, want, bound):
    """An 8-bit output against 64-bit values that the kernel knows to within `bound`: one rounding to E4M3 (with the
    subnormals' fixed spacing), under the scale of a maximum that `bound` allows."""
    q, s = h.get()
    bound = np.broadcast_to(bound, want.shape)

    def exponents(a):
        return T.exponent(np.stack([a[:, i:i + 128].max(1) for i in range(0, a.shape[1], 128)]))
    e = s.astype(int) - 127
    assert (e >= exponents(np.maximum(np.abs(want) - bound, 0))).all() and (e <= exponents(np.abs(want) + bound)).all()
    sub = np.exp2(e - 10.0)[np.arange(want.shape[1]) // 128].T
    close(T.unpack(q, s), want, bound * (1 + E4) + np.abs(want) * E4 + sub)


def rounded(bound, want, dtype):
    return bound + (np.abs(want) + bound) * BF if dtype == "bf16" else bound


# --------------------------------------------------------------------------
# The 8-bit format
# --------------------------------------------------------------------------
def _values(rows, cols, seed):
    r = rng(rows, cols, seed)
    x = r.standard_normal((rows, cols)) * np.exp2(r.integers(-12, 12, (rows, 1)).astype(float))
    return (x * np.exp2(3 * r.standard_normal((1, cols)))).astype(np.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 3, 1), (5, 777, 0, 0),
                                                  (64, 1024, 0, 0), (257, 2060, 4, 4), (33, 127, 1, 0), (2, 16, 8, 8)])
def test_pack_and_unpack_exact(rows, cols, pad, offset, dtype):
    x, v = dev(_values(rows, cols, 1), dtype, pad, offset)
    h = Held(rows, cols, more=16 * (pad % 3), lds=rows + pad)
    lm.lazymar_block8_pack(DT[dtype], x, cols + pad, h.d, rows, cols)
    sync()
    q, s = T.pack(v)
    got_q, got_s = h.get()
    assert (got_s == s).all()
    bytes_equal(got_q, q)
    y = out(rows, cols, dtype, pad, offset)
    lm.lazymar_block8_unpack(h.d, DT[dtype], y, cols + pad, rows, cols)
    sync()
    assert (y.double().cpu().numpy() == T.unpack(q, s)).all()  # exact in bf16 too


def test_pack_special_values():
    """Infinities and NaN become NaN and leave their block's scale alone; zeros, subnormals, the largest numbers, and
    maxima on and beside the limit 448 2^e."""
    x = _values(12, 300, 2)
    x[0] = 0
    x[1, 5], x[1, 140], x[1, 299] = np.inf, -np.inf, np.nan
    x[2, :128] = np.inf
    x[3, :128] = np.nan
    x[4] = 3.4e38
    x[5] = 1e-45
    x[6] = 1e-39
    x[7, :128] = 1.0
    x[7, 3] = 448.0
    x[8, :128] = 1.0
    x[8, 3] = np.nextafter(np.float32(448), np.float32(1e9))
    x[9] = -0.0
    x[10] = np.float32(2.0 ** -127)
    t, v = dev(x)
    h = Held(12, 300)
    lm.lazymar_block8_pack(lm.LAZYMAR_F32, t, 300, h.d, 12, 300)
    sync()
    q, s = T.pack(v)
    got_q, got_s = h.get()
    assert (got_s == s).all()
    bytes_equal(got_q, q)
    assert s[0, 7] == 127 and s[0, 8] == 128 and (got_q[2, :128] & 0x7F == 0x7F).all()
    y = out(12, 300)
    lm.lazymar_block8_unpack(h.d, lm.LAZYMAR_F32, y, 300, 12, 300)
    sync()
    with np.errstate(over="ignore"):  # 3.4e38 rounds to 2^128, which reads back as infinity
        np.testing.assert_array_equal(y.cpu().numpy(), T.unpack(q, s).astype(np.float32))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,K,pad", [(1, 1, 0), (128, 128, 0), (129, 255, 1), (300, 77, 0), (256, 1024, 4), (5, 640, 3)])
def test_pack_weight_and_its_transpose_exact(N, K, pad, dtype):
    w, v = dev(_values(N, K, 3), dtype, pad)
    if N > 2 and K > 2:
        w[1, 2] = float("nan")
        w[2, 1] = float("inf")
        v[1, 2], v[2, 1] = np.nan, np.inf
    h = Held(N, K, scale_rows=-(-N // 128))
    t = Held(K, N, scale_rows=-(-K // 128), more=16)
    lm.lazymar_block8_pack_weight(DT[dtype], w, K + pad, h.d, t.d, N, K)
    one = Held(K, N, scale_rows=-(-K // 128))
    lm.lazymar_block8_pack_weight(DT[dtype], w, K + pad, None, one.d, N, K)
    sync()
    q, s = T.pack_weight(v)
    got_q, got_s = h.get()
    assert (got_s == s).all()
    bytes_equal(got_q, q)
    for x in (t, one):
        got_q, got_s = x.get()
        assert (got_s == s.T).all()
        bytes_equal(got_q, q.T)


# --------------------------------------------------------------------------
# LayerNorm
# --------------------------------------------------------------------------
LN_SHAPES = [(1, 1, 0, 0), (1, 768, 0, 0), (5, 777, 0, 0), (3, 1024, 4, 0), (9, 1024, 0, 0), (17, 130, 2, 1),
             (300, 1280, 0, 0), (11, 2000, 0, 0), (4, 2560, 0, 0), (7, 4097, 3, 0), (2, 5120, 0, 0), (3, 8192, 0, 0),
             (2, 6001, 1, 1), (21, 128, 0, 0), (10, 256, 0, 0), (6, 512, 8, 4)]


def _ln_bounds(x, g, b):
    """fp32 rounding of mean, rstd and y: sums of D terms in trees of lanes and blocks (at most 40 adds in a row), two
    handfuls of operations on each element. mean: 48 u mean|x|; deviations carry it, so y's error is that over the
    standard deviation times |g|, and 64 u of y itself."""
    _, mean, rstd = T.layernorm(x, None, None, EPS)
    off = 48 * U * np.abs(x).mean(1)
    big = np.abs(g).max() if g is not None else 1.0
    y = T.layernorm(x, g, b, EPS)[0]
    # rstd's relative error: its squares' sum, and the mean's error where the row varies less than that
    rel = 64 * U + (off * rstd) ** 2
    return off, rel, (off * rstd)[:, None] * big + (64 * U + rel[:, None]) * (np.abs(y) + (np.abs(b).max() if b is not None else 0)) + 1e-12


@pytest.mark.parametrize("x_dtype,y_dtype", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("M,D,pad,offset", LN_SHAPES)
def test_layernorm_forward(M, D, pad, offset, x_dtype, y_dtype):
    r = rng(M, D, 4)
    x, v = dev(r.standard_normal((M, D)) * np.exp(r.standard_normal((M, 1))) + 0.5, x_dtype, pad, offset)
    g, b = 1 + 0.1 * r.standard_normal(D).astype(np.float32), 0.02 * r.standard_normal(D).astype(np.float32)
    tg, tb = vec(g), vec(b)
    y, y8, x8 = out(M, D, y_dtype, pad, offset), Held(M, D), Held(M, D, lds=M + 3)
    mean, rstd = vec(np.zeros(M)), vec(np.zeros(M))
    lm.lazymar_layernorm_forward(DT[x_dtype], x, D + pad, tg, tb, DT[y_dtype], y, D + pad, y8.d, x8.d, mean, rstd, M, D,
                                 EPS)
    sync()
    want, wm, wr = T.layernorm(v, g, b, EPS)
    off, rel, bound = _ln_bounds(v, g, b)
    close(mean, wm, off + 1e-12)
    close(rstd, wr, rel * wr)
    close(y, want, rounded(bound, want, y_dtype))
    close8(y8, want, bound)
    q, s = T.pack(v)
    got_q, got_s = x8.get()
    assert (got_s == s).all()
    bytes_equal(got_q, q)


def test_layernorm_forward_without_parameters_or_statistics():
    r = rng(5)
    x, v = dev(r.standard_normal((6, 1024)))
    y = out(6, 1024)
    for g, b in [(None, None), (r.standard_normal(1024), None), (None, r.standard_normal(1024))]:
        lm.lazymar_layernorm_forward(0, x, 1024, None if g is None else vec(g), None if b is None else vec(b), 0, y,
                                     1024, None, None, None, None, 6, 1024, EPS)
        sync()
        f = lambda a: None if a is None else a.astype(np.float32).astype(float)  # noqa: E731
        close(y, T.layernorm(v, f(g), f(b), EPS)[0], _ln_bounds(v, f(g), f(b))[2])


def test_layernorm_rows_that_do_not_vary_or_are_not_finite():
    """A constant row gives the shift and zero gradient terms; a row with NaN or infinity is NaN and leaves the others
    alone."""
    torch = torch_cuda()
    x = rng(6).standard_normal((4, 300)).astype(np.float32)
    x[0] = 3.0
    x[1, 7] = np.inf
    x[2, 9] = np.nan
    t = torch.from_numpy(x).cuda()
    b = vec(np.arange(300))
    y, mean, rstd = out(4, 300), vec(np.zeros(4)), vec(np.zeros(4))
    y8 = Held(4, 300)
    lm.lazymar_layernorm_forward(0, t, 300, None, b, 0, y, 300, y8.d, None, mean, rstd, 4, 300, EPS)
    sync()
    got = y.cpu().numpy()
    assert (got[0] == np.arange(300)).all()
    assert np.isnan(got[1]).all() and np.isnan(got[2]).all() and np.isfinite(got[3]).all()
    q, _ = y8.get()
    assert (q[1:3] & 0x7F == 0x7F).all() and not (q[[0, 3]] & 0x7F == 0x7F).any()


def _ln_grad_bounds(dy, xh, rstd, g):
    """fp32 rounding of dx: the two row sums (48 u of their mean magnitudes) and 16 operations on the terms; of the
    column sums: at most M adds in a row, u each, of the terms' magnitudes, whose factors carry 16 u."""
    a = np.abs(dy if g is None else dy * g)
    m1, m2 = a.mean(1, keepdims=True), (a * np.abs(xh)).mean(1, keepdims=True)
    dx = rstd[:, None] * (16 * U * a + 64 * U * (m1 + np.abs(xh) * m2)) + 1e-30
    n = dy.shape[0] + 48
    return dx, n * U * np.abs(dy * xh).sum(0) + 1e-30, n * U * np.abs(dy).sum(0) + 1e-30


@pytest.mark.parametrize("dy_dtype,x_kind,dx_dtype,res", [("bf16", "block8", "fp32", True), ("bf16", "bf16", "bf16", False),
                                                          ("fp32", "fp32", "fp32", False), ("fp32", "block8", "bf16", True),
                                                          ("bf16", "fp32", "fp32", True)])
@pytest.mark.parametrize("M,D,pad,offset", LN_SHAPES + [(2500, 320, 0, 0)])
def test_layernorm_backward(M, D, pad, offset, dy_dtype, x_kind, dx_dtype, res):
    torch = torch_cuda()
    r = rng(M, D, 7)
    x = r.standard_normal((M, D)) * np.exp(r.standard_normal((M, 1)))
    x8, xt = None, None
    if x_kind == "block8":
        x8, v = held(x, lds=M + 2)
    else:
        xt, v = dev(x, x_kind, pad, offset)
    _, mean, rstd = T.layernorm(v, None, None, EPS)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    dy, dyv = dev(r.standard_normal((M, D)) * 1e-3, dy_dtype, pad, offset)
    dres, resv = dev(r.standard_normal((M, D)) * 1e-3, "fp32", pad) if res else (None, 0.0)
    g = 1 + 0.1 * r.standard_normal(D).astype(np.float32)
    want, wg, wb = T.layernorm_grad(dyv, v, mean.astype(float), rstd.astype(float), g)
    xh = (v - mean.astype(float)[:, None]) * rstd.astype(float)[:, None]
    bx, bg, bb = _ln_grad_bounds(dyv, xh, rstd.astype(float), g)
    want = want + resv
    bx = bx + 2 * U * np.abs(want)
    ws = torch.full((lm.lazymar_layernorm_backward_workspace(M, D),), 0xFF, dtype=torch.uint8, device="cuda")
    dx = out(M, D, dx_dtype, pad, offset)
    dg, db = vec(np.ones(D)), vec(np.ones(D))
    tg, tm, tr = vec(g), vec(mean), vec(rstd)

    def call(dx, dg, db, accumulate):
        lm.lazymar_layernorm_backward(DT[dy_dtype], dy, D + pad, DT.get(x_kind, 0), xt, D + pad, x8.d if x8 else None, tm,
                                      tr, tg, dres, D + pad, DT[dx_dtype], dx, D + pad, dg, db, accumulate, M, D, ws,
                                      ws.numel())
    call(dx, dg, db, False)
    sync()
    close(dx, want, rounded(bx, want, dx_dtype))
    close(dg, wg, bg)
    close(db, wb, bb)
    first, fg = dx.clone(), dg.clone()
    call(dx, dg, db, True)  # adds to the parameter gradients, and gives the same again
    sync()
    assert torch.equal(dx, first) and torch.equal(dg, fg + fg)
    if res and dx_dtype == "fp32":  # in place of the residual stream's gradient
        lm.lazymar_layernorm_backward(DT[dy_dtype], dy, D + pad, DT.get(x_kind, 0), xt, D + pad, x8.d if x8 else None, tm,
                                      tr, tg, dres, D + pad, 0, dres, D + pad, None, None, False, M, D, None, 0)
        sync()
        assert torch.equal(dres, first)


@pytest.mark.parametrize("D", [1288, 1536, 1664, 2056, 2176, 2568, 3080, 3592, 4096, 4104])
def test_layernorm_backward_of_wide_rows(D):
    """Widths beyond 1280, among them those that leave some of a row's warps without columns."""
    test_layernorm_backward(1300, D, 0, 0, "bf16", "block8", "fp32", True)


def test_layernorm_backward_without_rows():
    torch = torch_cuda()
    dg, db = vec(np.ones(300)), vec(np.ones(300))
    args = (0, None, 300, 0, None, 300, None, None, None, None, None, 0, 0, None, 300)
    lm.lazymar_layernorm_backward(*args, dg, db, True, 0, 300, None, 0)
    sync()
    assert (dg == 1).all() and (db == 1).all()
    lm.lazymar_layernorm_backward(*args, dg, db, False, 0, 300, None, 0)
    sync()
    assert (dg == 0).all() and (db == 0).all()
    assert torch.isfinite(dg).all()


# --------------------------------------------------------------------------
# GELU's gradient
# --------------------------------------------------------------------------
@pytest.mark.parametrize("da_dtype,du_dtype,with8,with_u", [("bf16", "bf16", True, True), ("fp32", "fp32", False, True),
                                                            ("bf16", None, True, False), ("fp32", "bf16", True, True)])
@pytest.mark.parametrize("M,D,pad,offset", [(1, 1, 0, 0), (1, 1024, 0, 0), (7, 130, 1, 1), (300, 768, 0, 0),
                                            (61, 5000, 8, 0), (2500, 96, 0, 0), (5, 4096, 4, 4)])
def test_gelu_backward(M, D, pad, offset, da_dtype, du_dtype, with8, with_u):
    torch = torch_cuda()
    r = rng(M, D, 8)
    da, dv = dev(r.standard_normal((M, D)) * 1e-3, da_dtype, pad, offset)
    # every size of u: negative tails, zeros, values beyond the range where the gradient varies
    h, u = held(r.standard_normal((M, D)) * np.exp2(r.integers(-40, 7, (M, 1)).astype(float)), lds=M + 1)
    grad = T.gelu_grad(u) if with_u else np.ones_like(u)
    want = dv * grad
    bound = np.abs(dv) * 5e-7 + 4 * U * np.abs(want) + 1e-30  # the gradient's absolute error
    du = out(M, D, du_dtype, pad, offset) if du_dtype else None
    du8 = Held(M, D, lds=M + 5) if with8 else None
    db = vec(np.ones(D))
    ws = torch.full((lm.lazymar_block8_gelu_backward_workspace(M, D),), 0xFF, dtype=torch.uint8, device="cuda")
    args = (DT[da_dtype], da, D + pad, h.d if with_u else None, DT.get(du_dtype, 0), du, D + pad, du8.d if with8 else None)
    lm.lazymar_block8_gelu_backward(*args, db, False, M, D, ws, ws.numel())
    sync()
    if du is not None:
        close(du, want, rounded(bound, want, du_dtype))
    if with8:
        close8(du8, want, bound)
    close(db, want.sum(0), bound.sum(0) + (M + 16) * U * np.abs(want).sum(0))
    first = db.clone()
    lm.lazymar_block8_gelu_backward(*args, db, True, M, D, ws, ws.numel())
    sync()
    assert torch.equal(db, first + first)


@pytest.mark.parametrize("cols,pad", [(512, 0), (300, 1)])
def test_gelu_backward_in_place(cols, pad):
    torch = torch_cuda()
    r = rng(23)
    da, _ = dev(r.standard_normal((70, cols)), "bf16", pad)
    h, _ = held(r.standard_normal((70, cols)))
    du = out(70, cols, "bf16", pad)
    lm.lazymar_block8_gelu_backward(1, da, cols + pad, h.d, 1, du, cols + pad, None, None, False, 70, cols, None, 0)
    lm.lazymar_block8_gelu_backward(1, da, cols + pad, h.d, 1, da, cols + pad, None, None, False, 70, cols, None, 0)
    sync()
    assert torch.equal(da, du)


def test_gelu_backward_keeps_nan():
    x = rng(9).standard_normal((4, 200)).astype(np.float32)
    da, _ = dev(x)
    x[1, 3], x[2, 150] = np.nan, np.inf
    h, _ = held(x)
    du = out(4, 200)
    lm.lazymar_block8_gelu_backward(0, da, 200, h.d, 0, du, 200, None, None, False, 4, 200, None, 0)
    sync()
    got = np.isnan(du.cpu().numpy())
    assert got[1, 3] and got[2, 150] and got.sum() == 2


# --------------------------------------------------------------------------
# The 8-bit product
# --------------------------------------------------------------------------
LINEAR_SHAPES = [(1, 1, 1), (1, 1024, 128), (2, 300, 77), (5, 128, 1000), (129, 257, 130), (300, 128, 640),
                 (64, 1000, 520), (1111, 300, 2060), (128, 640, 4096), (2, 4096, 1024), (9, 768, 5120), (17, 520, 300),
                 (33, 1280, 1279)]


def _product(M, N, K, seed, a_lds=0):
    r = rng(M, N, K, seed)
    a, av = held(r.standard_normal((M, K)) * np.exp(r.standard_normal((M, 1))) * np.exp2(r.integers(-9, 9, (1, K))),
                 lds=M + a_lds)
    w, wv = held_weight(0.05 * r.standard_normal((N, K)))
    b = r.standard_normal(N).astype(np.float32)
    return a, w, b, av @ wv.T + b, np.abs(av) @ np.abs(wv).T + np.abs(b)


def _product_bound(mag, K):
    """The products of E4M3 values and powers of two are exact. Each step of 32 columns adds to an fp32 accumulator
    that may truncate, on terms lined up with the largest: 4 u of the sum of magnitudes a step, and 16 steps more for
    the bias and what follows."""
    return (K / 32 + 16) * 4 * U * mag + 1e-30


@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES)
@pytest.mark.parametrize("out_dtype,pad", [("fp32", 0), ("bf16", 0), ("bf16", 3), ("fp32", 5)])
def test_linear_bias(M, N, K, out_dtype, pad):
    torch = torch_cuda()
    a, w, b, want, mag = _product(M, N, K, 10, pad)
    tb = vec(b)
    y, y8 = out(M, N, out_dtype, pad, pad % 2), Held(M, N, lds=M + 3)
    args = (0, a.d, w.d, tb, None, 0, DT[out_dtype], y, N + pad, y8.d, None, M, N, K)
    lm.lazymar_block8_linear(*args)
    sync()
    bound = _product_bound(mag, K)
    close(y, want, rounded(bound, want, out_dtype))
    close8(y8, want, bound)
    first, f8 = y.clone(), y8.q.clone()
    lm.lazymar_block8_linear(*args)
    sync()
    assert torch.equal(y, first) and torch.equal(y8.q, f8)


@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES)
@pytest.mark.parametrize("out_dtype", ["bf16", None])
def test_linear_gelu_and_checkpoint(M, N, K, out_dtype):
    a, w, b, u, mag = _product(M, N, K, 11)
    y = out(M, N, out_dtype) if out_dtype else None
    y8 = None if out_dtype else Held(M, N)
    u8 = Held(M, N, lds=M + 1)
    lm.lazymar_block8_linear(1, a.d, w.d, vec(b), None, 0, DT.get(out_dtype, 0), y, N, y8.d if y8 else None, u8.d, M, N, K)
    sync()
    bound = _product_bound(mag, K)
    want = T.gelu(u)
    gb = bound * 1.13 + 4e-7 * np.maximum(1, np.abs(u))  # |GELU'| < 1.13, the kernels' GELU to 2.8e-7 max(1, |u|)
    close8(u8, u, bound)
    if y is not None:
        close(y, want, rounded(gb, want, out_dtype))
    else:
        close8(y8, want, gb)


@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES)
@pytest.mark.parametrize("pad", [0, 1])
def test_linear_residual(M, N, K, pad):
    torch = torch_cuda()
    a, w, b, y, mag = _product(M, N, K, 12)
    res, rv = dev(rng(M, N, 13).standard_normal((M, N)), "fp32", pad)
    o = out(M, N, "fp32", pad)
    args = (a.d, w.d, None, res, N + pad, 0)
    lm.lazymar_block8_linear(2, *args, o, N + pad, None, None, M, N, K)
    sync()
    want = y - b + rv
    close(o, want, _product_bound(mag, K) + 2 * U * np.abs(want))
    lm.lazymar_block8_linear(2, *args, res, N + pad, None, None, M, N, K)  # in place
    sync()
    assert torch.equal(res, o)


@pytest.mark.parametrize("M,N,K", [(2700, 2000, 384), (9900, 520, 700), (4100, 1300, 1000)])
def test_linear_many_tiles(M, N, K):
    """Enough 256 x 256 tiles for CTA pairs, several a pair, with ragged edges."""
    a, w, b, want, mag = _product(M, N, K, 14)
    y, y8, u8 = out(M, N), Held(M, N), Held(M, N)
    lm.lazymar_block8_linear(0, a.d, w.d, vec(b), None, 0, 0, y, N, y8.d, None, M, N, K)
    o = out(M, N)
    lm.lazymar_block8_linear(2, a.d, w.d, vec(b), y, N, 0, o, N, None, None, M, N, K)
    g8 = Held(M, N)
    lm.lazymar_block8_linear(1, a.d, w.d, vec(b), None, 0, 0, None, 0, g8.d, u8.d, M, N, K)
    sync()
    bound = _product_bound(mag, K)
    close(y, want, bound)
    close8(y8, want, bound)
    close(o, 2 * want, 2 * bound + 2 * U * np.abs(want))
    close8(u8, want, bound)
    close8(g8, T.gelu(want), bound * 1.13 + 4e-7 * np.maximum(1, np.abs(want)))


@pytest.mark.parametrize("M", [3, 40, 400])
def test_linear_scales_far_from_one(M):
    """Factors whose product leaves fp32's range where the result does not: a zero stays zero, and large times small
    is exact."""
    r = rng(24)
    x = r.standard_normal((M, 256))
    x[:, :128] *= 2.0 ** 100
    x[:, 128:] *= 2.0 ** -100
    w = r.standard_normal((128, 256))
    w[:, :128] *= 2.0 ** -100
    w[:, 128:] *= 2.0 ** 100
    x[1] = 0
    a, av = held(x.astype(np.float32))
    v, wv = held_weight(w.astype(np.float32))
    y = out(M, 128)
    lm.lazymar_block8_linear(0, a.d, v.d, None, None, 0, 0, y, 128, None, None, M, 128, 256)
    sync()
    close(y, av @ wv.T, _product_bound(np.abs(av) @ np.abs(wv).T, 256))
    assert (y[1] == 0).all()


def test_linear_ignores_padding_bytes_and_keeps_nan_in_its_row():
    r = rng(15)
    a, av = held(r.standard_normal((200, 200)), more=32)
    w, wv = held_weight(r.standard_normal((150, 200)), more=16)
    a.q[7, 11] = 0x7F
    y, y8 = out(200, 150), Held(200, 150)
    lm.lazymar_block8_linear(0, a.d, w.d, None, None, 0, 0, y, 150, y8.d, None, 200, 150, 200)
    sync()
    got = np.isnan(y.cpu().numpy())
    assert got[7].all() and got.sum() == 150
    q, _ = y8.get()
    assert (q[7] & 0x7F == 0x7F).all() and ((q & 0x7F) == 0x7F).sum() == 150


# --------------------------------------------------------------------------
# The weight gradient
# --------------------------------------------------------------------------
def _wgrad_bound(mag, M):
    """Products of two bf16 values are exact in fp32. Within 512 tokens, 32 steps of 16 on an accumulator that may
    truncate with its terms lined up: 4 u a step; then one rounding for each 512 tokens and each split."""
    return (48 * 4 + M / 512 + 34) * U * mag + 1e-30


@pytest.mark.parametrize("M,N,K,pad", [(1, 1, 1, 0), (1, 128, 128, 0), (63, 130, 77, 1), (64, 64, 64, 0),
                                       (65, 256, 256, 4), (700, 300, 200, 0), (3211, 1000, 776, 0), (5000, 8, 300, 3),
                                       (129, 2100, 1100, 0), (1600, 1280, 1024, 0), (4096, 129, 1, 0), (513, 4096, 1024, 0)])
def test_wgrad(M, N, K, pad):
    torch = torch_cuda()
    r = rng(M, N, K, 21)
    ldy = -(-(N + pad) // 8) * 8
    dy, dyv = dev(r.standard_normal((M, N)) * np.exp(r.standard_normal((M, 1))), "bf16", ldy - N)
    x, xv = held(r.standard_normal((M, K)) * np.exp2(r.integers(-20, 20, (M, 1)).astype(float)), lds=M + pad)
    dw = out(N, K, "fp32", pad)
    ws = torch.full((lm.lazymar_block8_wgrad_workspace(M, N, K) + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    args = (dy, ldy, x.d, dw, K + pad)
    lm.lazymar_block8_wgrad(*args, False, M, N, K, ws, ws.numel())
    sync()
    want, bound = dyv.T @ xv, _wgrad_bound(np.abs(dyv).T @ np.abs(xv), M)
    close(dw, want, bound)
    first = dw.clone()
    lm.lazymar_block8_wgrad(*args, True, M, N, K, ws, ws.numel())
    sync()
    assert torch.equal(dw, first + first)


def test_wgrad_without_rows():
    dw = vec(np.ones((300, 70)))
    lm.lazymar_block8_wgrad(None, 300, None, dw, 70, True, 0, 300, 70, None, 0)
    sync()
    assert (dw == 1).all()
    lm.lazymar_block8_wgrad(None, 300, None, dw, 70, False, 0, 300, 70, None, 0)
    sync()
    assert (dw == 0).all()


def test_wgrad_keeps_nan_and_the_range_of_scales():
    """A NaN byte reaches its column of dw and no other; scales at both ends of their range; bytes beyond K are not
    read as values."""
    r = rng(22)
    v = r.standard_normal((200, 150)) * 1e-3
    v[0], v[1] = 2.0 ** 100, 2.0 ** -120
    x, xv = held(v.astype(np.float32), more=32)
    x.q[9, 17] = 0xFF
    dy, dyv = dev(r.standard_normal((200, 136)), "bf16")
    dyv[0] = 0
    dy[0] = 0
    dw = out(136, 150)
    lm.lazymar_block8_wgrad(dy, 136, x.d, dw, 150, False, 200, 136, 150, None if not
                            lm.lazymar_block8_wgrad_workspace(200, 136, 150) else
                            torch_cuda().empty(lm.lazymar_block8_wgrad_workspace(200, 136, 150), dtype=torch_cuda().uint8,
                                               device="cuda"), lm.lazymar_block8_wgrad_workspace(200, 136, 150))
    sync()
    got = dw.double().cpu().numpy()
    assert np.isnan(got[:, 17]).all() and np.isnan(got).sum() == 136
    keep = np.arange(150) != 17
    xv[0] = 0
    want = dyv.T @ xv
    assert (np.abs(got - want) <= _wgrad_bound(np.abs(dyv).T @ np.abs(xv), 200))[:, keep].all()


# --------------------------------------------------------------------------
# Streams, offsets, refusals
# --------------------------------------------------------------------------
def test_calls_follow_the_callers_stream():
    """Everything on a side stream, behind work that is still running there."""
    torch = torch_cuda()
    r = rng(16)
    a, w, b, want, mag = _product(300, 256, 512, 17)
    x, v = dev(r.standard_normal((300, 512)))
    h = Held(300, 512)
    y = out(300, 256)
    st = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    src = a.q.clone()
    a.q.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for _ in range(8):
            big = big @ big * 1e-3
        a.q.copy_(src)
        lm.lazymar_block8_linear(0, a.d, w.d, vec(b), None, 0, 0, y, 256, None, None, 300, 256, 512)
        lm.lazymar_block8_pack(0, x, 512, h.d, 300, 512)
    st.synchronize()
    lm.lazymar_device_check()
    close(y, want, _product_bound(mag, 512))
    assert (h.get()[1] == T.pack(v)[1]).all()


def test_calls_can_be_captured():
    torch = torch_cuda()
    a, w, b, want, mag = _product(300, 256, 512, 18)
    y, tb = out(300, 256), vec(b)
    x, v = dev(rng(18).standard_normal((40, 777)))
    m, rs = vec(np.zeros(40)), vec(np.zeros(40))
    z = out(40, 777)

    def both():
        lm.lazymar_block8_linear(0, a.d, w.d, tb, None, 0, 0, y, 256, None, None, 300, 256, 512)
        lm.lazymar_layernorm_forward(0, x, 777, None, None, 0, z, 777, None, None, m, rs, 40, 777, EPS)
    both()
    sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    y.zero_()
    z.zero_()
    g.replay()
    sync()
    close(y, want, _product_bound(mag, 512))
    close(z, T.layernorm(v, None, None, EPS)[0], _ln_bounds(v, None, None)[2])


def test_offsets_beyond_32_bits():
    """Rows that start more than 2^32 bytes into their buffer."""
    torch = torch_cuda()
    ld = (1 << 30) + 16
    x = torch.zeros(3 * ld, dtype=torch.bfloat16, device="cuda").view(3, ld)[:, :640]
    v = rng(19).standard_normal((3, 640)).astype(np.float32)
    x.copy_(torch.from_numpy(v))
    v = x.double().cpu().numpy()
    q = torch.zeros(5 * ld, dtype=torch.uint8, device="cuda").view(5, ld)
    scale = torch.zeros((5, 5), dtype=torch.uint8, device="cuda")
    h = lm.lazymar_block8(q[:3], scale, lds=5)
    m, rs = vec(np.zeros(3)), vec(np.zeros(3))
    y = torch.zeros(3 * ld, dtype=torch.bfloat16, device="cuda").view(3, ld)[:, :640]
    lm.lazymar_layernorm_forward(1, x, ld, None, None, 1, y, ld, None, h, m, rs, 3, 640, EPS)
    back = out(3, 640)
    lm.lazymar_block8_unpack(h, 0, back, 640, 3, 640)
    w, wv = held_weight(rng(20).standard_normal((64, 640)))
    o = out(3, 64)
    lm.lazymar_block8_linear(0, h, w.d, None, None, 0, 0, o, 64, None, None, 3, 64, 640)
    sync()
    want, _, _ = T.layernorm(v, None, None, EPS)
    close(y, want, rounded(_ln_bounds(v, None, None)[2], want, "bf16"))
    vals = T.unpack(*T.pack(v))
    assert (back.double().cpu().numpy() == vals).all()
    close(o, vals @ wv.T, _product_bound(np.abs(vals) @ np.abs(wv).T, 640))


def test_refusals():
    torch = torch_cuda()
    x = out(4, 256)
    h, w = Held(4, 256), Held(8, 256, scale_rows=1)
    host = torch.zeros((4, 256))

    def refuses(f, word):
        with pytest.raises(lm.LazymarError) as e:
            f()
        assert e.value.status == 1 and word in str(e.value)

    b8 = lm.lazymar_block8
    refuses(lambda: lm.lazymar_block8_pack(0, host, 256, h.d, 4, 256), "x:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 255, h.d, 4, 256), "x:")
    refuses(lambda: lm.lazymar_block8_pack(2, x, 256, h.d, 4, 256), "x:")
    refuses(lambda: lm.lazymar_block8_pack(0, x.data_ptr() + 2, 256, h.d, 4, 256), "x:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 256, b8(h.q, h.scale, ldq=264), 4, 256), "q:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 256, b8(h.q, h.scale, ldq=240), 4, 256), "q:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 256, b8(h.q, h.scale, lds=3), 4, 256), "q:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 256, b8(h.q.data_ptr() + 8, h.scale, 256, 4), 4, 256), "q:")
    refuses(lambda: lm.lazymar_block8_pack(0, x, 256, b8(h.q, None, 256, 4), 4, 256), "q:")
    refuses(lambda: lm.lazymar_block8_unpack(h.d, 0, host, 256, 4, 256), "x:")
    refuses(lambda: lm.lazymar_block8_linear(0, h.d, b8(w.q, w.scale, lds=0), None, None, 0, 0, x, 256, None, None, 4, 8,
                                             256), "w:")
    refuses(lambda: lm.lazymar_block8_linear(0, h.d, w.d, None, None, 0, 0, x, 7, None, None, 4, 8, 256), "out:")
    refuses(lambda: lm.lazymar_block8_linear(2, h.d, w.d, None, None, 8, 0, x, 8, None, None, 4, 8, 256), "residual")
    db = vec(np.zeros(256))
    refuses(lambda: lm.lazymar_block8_gelu_backward(0, x, 256, None, 0, None, 0, None, db, False, 4, 256, None, 0),
            "workspace")
    refuses(lambda: lm.lazymar_layernorm_backward(0, x, 256, 0, x, 256, None, db, db, None, None, 0, 0, x, 256, db, db,
                                                  False, 4, 256, x, 64), "workspace")
    sync()  # none of them has launched anything


@pytest.mark.parametrize("M,D,pad", [(1, 512, 0), (300, 1024, 0), (300, 1280, 8), (301, 777, 0), (40, 5000, 3)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_layernorm_in_place_of_its_input(M, D, pad, dtype):
    """y over x and dx over dy or x, with their type and stride, give what they give elsewhere."""
    torch = torch_cuda()
    r = rng(M, D, 30)
    x, _ = dev(r.standard_normal((M, D)), dtype, pad)
    dy, _ = dev(r.standard_normal((M, D)), dtype, pad)
    t, ld, g = DT[dtype], D + pad, vec(1 + 0.1 * r.standard_normal(D))
    mean, rstd = vec(np.zeros(M)), vec(np.zeros(M))

    def forward(x, y):
        lm.lazymar_layernorm_forward(t, x, ld, g, None, t, y, ld, None, None, mean, rstd, M, D, EPS)

    def backward(dy, x, dx):
        lm.lazymar_layernorm_backward(t, dy, ld, t, x, ld, None, mean, rstd, g, None, 0, t, dx, ld, None, None, False, M,
                                      D, None, 0)
    y, dx = out(M, D, dtype, pad), out(M, D, dtype, pad)
    forward(x, y)
    backward(dy, x, dx)
    for over_x in (False, True):
        a, b = dev(dy.float().cpu().numpy(), dtype, pad)[0], dev(x.float().cpu().numpy(), dtype, pad)[0]
        backward(a, b, b if over_x else a)
        sync()
        assert torch.equal(b if over_x else a, dx)
    z, _ = dev(x.float().cpu().numpy(), dtype, pad)
    forward(z, z)
    sync()
    assert torch.equal(z, y)


@pytest.mark.parametrize("M", [3, 20, 32, 40, 400, 2700])
@pytest.mark.parametrize("ea,ew,small", [(119, -115, False), (112, -108, False), (-115, 119, False), (-125, 100, True),
                                         (-120, 112, True), (100, -125, True)])
def test_linear_scales_at_both_ends(M, ea, ew, small):
    """Scales near the ends of their range whose product is an ordinary number: neither factor may be applied to a
    block's sum on its own (2^24 2^112 overflows, 2^-18 2^-126 loses digits). `small`: E4M3's subnormals alone."""
    r = rng(M, ea + 200, 25)
    N, K = 136, 384
    a, w = Held(M, K), Held(N, K, scale_rows=2)
    q = np.r_[1:8, 0x81:0x88] if small else np.r_[1:0x7F, 0x81:0xFF]  # no NaN

    def fill(h, rows, e, scales):
        h.set(r.choice(q, (rows, K)).astype(np.uint8), (127 + r.integers(e - 1, e + 2, (3, scales))).astype(np.uint8))
    fill(a, M, ea, M)
    fill(w, N, ew, 2)
    av, wv = T.unpack(*a.get()), T.unpack_weight(*w.get())
    y = out(M, N)
    lm.lazymar_block8_linear(0, a.d, w.d, None, None, 0, 0, y, N, None, None, M, N, K)
    sync()
    close(y, av @ wv.T, _product_bound(np.abs(av) @ np.abs(wv).T, K))


def test_smallest_scales_in_bf16():
    """Every byte under the smallest scales: fp32 holds their values, bf16 those in steps of 2^-133 (all of them from
    scales of 2^-124 on, and from 2^-130 on under any), others rounded to nearest even. The weight gradient's operand
    is the same."""
    torch = torch_cuda()
    rows = 8
    q = np.arange(256, dtype=np.uint8)[None].repeat(rows, 0)
    q[(q & 0x7F) == 0x7F] = 0
    h = Held(rows, 256).set(q, np.arange(1, rows + 1, dtype=np.uint8)[None].repeat(2, 0))
    x = T.unpack(*h.get())
    wide, narrow = out(rows, 256), out(rows, 256, "bf16")
    lm.lazymar_block8_unpack(h.d, 0, wide, 256, rows, 256)
    lm.lazymar_block8_unpack(h.d, 1, narrow, 256, rows, 256)
    step = np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -140))) - 7), 2.0 ** -133)
    held16 = np.rint(x / step) * step  # rint: ties to even
    assert (held16[2:] == x[2:]).all() and (held16 == x)[np.abs(x) >= 2.0 ** -130].all() and (held16 != x).any()
    dy, dyv = dev(np.eye(rows) * 2.0 ** 60, "bf16")
    dw = out(rows, 256)
    n = lm.lazymar_block8_wgrad_workspace(rows, rows, 256)
    lm.lazymar_block8_wgrad(dy, rows, h.d, dw, 256, False, rows, rows, 256, torch.empty(n + 16, dtype=torch.uint8,
                                                                                        device="cuda"), n)
    sync()
    assert (wide.double().cpu().numpy() == x).all()
    assert (narrow.double().cpu().numpy() == held16).all()
    assert (dw.double().cpu().numpy() == dyv.T @ held16).all()


@pytest.mark.parametrize("M", [1, 20, 40, 400, 2700])
@pytest.mark.parametrize("out_dtype", ["fp32", "bf16"])
def test_linear_gelu_within_its_bound(M, out_dtype):
    """With a zero operand GELU's argument is the bias, exactly. The polynomial of degree six is within
    1.1e-7 max(1, |u|) in fp32 arithmetic, exp2's approximation adds 2^-22 of |u| h(|u|) <= 0.17."""
    N = 4097
    b = np.linspace(-12, 12, N).astype(np.float32)
    a, w = held(np.zeros((M, 128)))[0], held_weight(rng(27).standard_normal((N, 128)))[0]
    y = out(M, N, out_dtype)
    lm.lazymar_block8_linear(1, a.d, w.d, vec(b), None, 0, DT[out_dtype], y, N, None, None, M, N, 128)
    sync()
    u = b.astype(float)[None].repeat(M, 0)
    want = T.gelu(u[:1]).repeat(M, 0)
    bound = 1.1e-7 * np.maximum(1, np.abs(u)) + 0.17 * 2.0 ** -22 + U * np.abs(want)
    close(y, want, rounded(bound, want, out_dtype))


@pytest.mark.parametrize("M,N,K", [(3, 136, 384), (12, 300, 384), (32, 136, 384), (400, 136, 384), (128, 640, 4096),
                                   (2700, 2000, 384)])
@pytest.mark.parametrize("gelu", [False, True])
def test_linear_overflow_stays_in_its_element(M, N, K, gelu):
    """A sum beyond fp32's range is infinite (or NaN after GELU) in fp32 and NaN in the 8-bit outputs, whose scale is
    that of the block's finite values."""
    torch = torch_cuda()
    r = rng(M, N, K, 26)
    x, v = r.standard_normal((M, K)).astype(np.float32), 0.05 * r.standard_normal((N, K)).astype(np.float32)
    x[1, :128], v[:, :128] = 3.0, 0
    v[3, :128], v[70, :128] = 2.0, -2.0
    a, w = held(x)[0], held_weight(v)[0]
    a.scale[0, 1], w.scale[0, 0] = 247, 127 + 100
    av, wv = T.unpack(*a.get()), T.unpack_weight(*w.get())
    u, mag = av @ wv.T, np.abs(av) @ np.abs(wv).T
    inf = np.abs(u) > 2.0 ** 128
    assert inf.sum() == 2 and (np.abs(u[~inf]) < 2.0 ** 127).all()
    y, y8, u8 = out(M, N), Held(M, N), Held(M, N)
    lm.lazymar_block8_linear(int(gelu), a.d, w.d, None, None, 0, 0, y, N, y8.d, u8.d if gelu else None, M, N, K)
    sync()
    bound = np.where(inf, 0, _product_bound(mag, K))
    finite = np.where(inf, 0, u)
    got = y.cpu().numpy()
    assert (np.isfinite(got) == ~inf).all()
    assert got[1, 3] == np.inf and (np.isnan(got[1, 70]) if gelu else got[1, 70] == -np.inf)
    for h, want, b in ((y8, T.gelu(finite) if gelu else finite,
                        np.where(inf, 0, bound * 1.13 + 4e-7 * np.maximum(1, np.abs(finite))) if gelu else bound),
                       (u8, finite, bound))[:1 + gelu]:
        q, _ = h.get()
        assert (((q & 0x7F) == 0x7F) == inf).all()
        h.q[:, :N][torch.from_numpy(inf).cuda()] = 0
        close8(h, want, b)


@pytest.mark.parametrize("D,x_kind", [(1024, "bf16"), (1024, "block8"), (777, "fp32"), (777, "block8"), (4104, "bf16")])
def test_layernorm_backward_of_rows_that_are_not_finite(D, x_kind):
    """NaN in a row's input or infinity in its gradient: that row of dx is lost, and of dg and db what it adds to; the
    other rows are as without it."""
    torch = torch_cuda()
    r = rng(D, 28)
    M = 70
    x, g = r.standard_normal((M, D)).astype(np.float32), vec(1 + 0.1 * r.standard_normal(D))
    dy = r.standard_normal((M, D)).astype(np.float32)
    ws = torch.empty(lm.lazymar_layernorm_backward_workspace(M, D), dtype=torch.uint8, device="cuda")

    def run(x, dy):
        if x_kind == "block8":
            h, v = held(x)
            t = None
        else:
            h, (t, v) = None, dev(x, x_kind)
        with np.errstate(invalid="ignore"):
            _, mean, rstd = T.layernorm(v, None, None, EPS)
        dx, dg, db = out(M, D), vec(np.zeros(D)), vec(np.zeros(D))
        td, _ = dev(dy)
        lm.lazymar_layernorm_backward(0, td, D, DT.get(x_kind, 0), t, D, h.d if h else None, vec(mean), vec(rstd), g, None,
                                      0, 0, dx, D, dg, db, False, M, D, ws, ws.numel())
        sync()
        return [a.cpu().numpy() for a in (dx, dg, db)]
    clean = run(x, dy)
    assert all(np.isfinite(a).all() for a in clean)
    others = np.arange(M) != 9
    bad = x.copy()
    bad[9, 5] = np.nan
    dx, dg, db = run(bad, dy)
    assert np.isnan(dx[9]).all() and (dx[others] == clean[0][others]).all()
    assert np.isnan(dg).all() and (db == clean[2]).all()
    bad = dy.copy()
    bad[9, 5] = np.inf
    dx, dg, db = run(x, bad)
    assert not np.isfinite(dx[9]).any() and (dx[others] == clean[0][others]).all()
    there = np.arange(D) == 5
    for got, was in ((dg, clean[1]), (db, clean[2])):
        assert np.isinf(got[there]).all() and (got[~there] == was[~there]).all()


def _spread(a, dtype, ld):
    """A device tensor whose rows are `ld` elements apart, with nothing set between them."""
    torch = torch_cuda()
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "byte": torch.uint8}[dtype]
    v = torch.empty(a.shape[0] * ld, dtype=t, device="cuda").view(a.shape[0], ld)[:, :a.shape[1]]
    v.copy_(torch.from_numpy(a).cuda())
    return v


@pytest.mark.parametrize("D,ld", [(640, (1 << 26) + 8), (636, (1 << 26) + 5)])
def test_backward_offsets_beyond_32_bits(D, ld):
    """LayerNorm's and GELU's gradients and the weight gradient of rows that start more than 2^32 bytes into their
    buffers: the same as from rows next to each other."""
    torch = torch_cuda()
    M, N, ld8 = 40, 48, (1 << 27) + 16
    r = rng(D, 29)
    x, dy, res = (r.standard_normal((M, D)).astype(np.float32) for _ in range(3))
    near, v = held(x)
    q, s = near.get()
    far = lm.lazymar_block8(_spread(q, "byte", ld8), near.scale)
    _, mean, rstd = T.layernorm(v, None, None, EPS)
    tm, tr = vec(mean), vec(rstd)
    n = max(lm.lazymar_layernorm_backward_workspace(M, D), lm.lazymar_block8_gelu_backward_workspace(M, D),
            lm.lazymar_block8_wgrad_workspace(M, N, D), 16)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = []
    for h, stride, make in ((near.d, D, lambda a, t: dev(a, t)[0]), (far, ld, lambda a, t: _spread(a, t, ld))):
        tdy, tres = make(dy, "bf16"), make(res, "fp32")
        dx = make(np.zeros_like(x), "fp32")
        dg, db, du_db = (vec(np.zeros(D)) for _ in range(3))
        lm.lazymar_layernorm_backward(1, tdy, stride, 0, None, 0, h, tm, tr, None, tres, stride, 0, dx, stride, dg, db,
                                      False, M, D, ws, n)
        du = make(np.zeros_like(x), "bf16")
        lm.lazymar_block8_gelu_backward(1, tdy, stride, h, 1, du, stride, None, du_db, False, M, D, ws, n)
        sync()
        outs.append([a.clone() for a in (dx, dg, db, du, du_db)])
        del tdy, tres, dx, du
    want, wg, wb = T.layernorm_grad(dev(dy, "bf16")[1], v, mean.astype(np.float32).astype(float),
                                    rstd.astype(np.float32).astype(float), None)
    xh = (v - mean.astype(np.float32)[:, None]) * rstd.astype(np.float32)[:, None]
    bx, bg, bb = _ln_grad_bounds(dev(dy, "bf16")[1], xh, rstd, None)
    for dx, dg, db, du, du_db in outs:
        close(dx, want + res, bx + 2 * U * np.abs(want + res))
        close(dg, wg, bg)
        close(db, wb, bb)
    assert torch.equal(outs[0][3], outs[1][3])
    grad = dev(dy, "bf16")[1] * T.gelu_grad(v)
    bound = np.abs(dev(dy, "bf16")[1]) * 5e-7 + 4 * U * np.abs(grad) + 1e-30
    for o in outs:
        close(o[4], grad.sum(0), bound.sum(0) + (M + 16) * U * np.abs(grad).sum(0))
    # the weight gradient: dy in rows of multiples of eight
    dn = r.standard_normal((M, N)).astype(np.float32)
    a, b = out(N, D), out(N, D)
    lm.lazymar_block8_wgrad(dev(dn, "bf16")[0], N, near.d, a, D, False, M, N, D, ws, n)
    lm.lazymar_block8_wgrad(_spread(dn, "bf16", (1 << 26) + 8), (1 << 26) + 8, far, b, D, False, M, N, D, ws, n)
    sync()
    assert torch.equal(a, b)


def test_product_offsets_beyond_32_bits():
    """The product of more rows than the few-row kernel takes, every operand and output with rows that start more than
    2^32 bytes into its buffer."""
    torch = torch_cuda()
    M, N, K, ld8, ld = 40, 160, 384, (1 << 27) + 16, (1 << 26) + 4
    a, w, b, want, mag = _product(M, N, K, 31)
    tb = vec(b)
    far = lm.lazymar_block8(_spread(a.get()[0], "byte", ld8), a.scale)
    far_w = lm.lazymar_block8(_spread(w.get()[0], "byte", ld8), w.scale)
    zeros = np.zeros((M, N), np.float32)
    y, z = out(M, N), _spread(zeros, "fp32", ld)
    y8, z8 = Held(M, N), _spread(zeros.astype(np.uint8), "byte", ld8)
    s8 = torch.zeros((2, M), dtype=torch.uint8, device="cuda")
    lm.lazymar_block8_linear(0, a.d, w.d, tb, None, 0, 0, y, N, y8.d, None, M, N, K)
    lm.lazymar_block8_linear(0, far, far_w, tb, None, 0, 0, z, ld, lm.lazymar_block8(z8, s8), None, M, N, K)
    sync()
    close(z, want, _product_bound(mag, K))
    assert torch.equal(y, z) and torch.equal(y8.q[:, :N], z8) and torch.equal(y8.scale, s8)
    lm.lazymar_block8_linear(2, far, far_w, tb, z, ld, 0, z, ld, None, None, M, N, K)
    sync()
    close(z, 2 * want, 2 * _product_bound(mag, K) + 2 * U * np.abs(want))


def _backward_calls():
    """LayerNorm's, GELU's and the weight gradient with workspaces, as a function of no arguments, its inputs and its
    outputs."""
    torch = torch_cuda()
    M, D, N = 3000, 320, 256
    r = rng(32)
    h, v = held(r.standard_normal((M, D)))
    _, mean, rstd = T.layernorm(v, None, None, EPS)
    tm, tr = vec(mean), vec(rstd)
    dy, dn = dev(r.standard_normal((M, D)), "bf16")[0], dev(r.standard_normal((M, N)), "bf16")[0]
    ws = [torch.empty(n + 16, dtype=torch.uint8, device="cuda") for n in (
        lm.lazymar_layernorm_backward_workspace(M, D), lm.lazymar_block8_gelu_backward_workspace(M, D),
        lm.lazymar_block8_wgrad_workspace(M, N, D))]
    assert ws[2].numel() > 16  # in parts, with a sum of its own
    outs = [out(M, D), vec(np.zeros(D)), vec(np.zeros(D)), out(M, D, "bf16"), vec(np.zeros(D)), out(N, D)]
    dx, dg, db, du, dbu, dw = outs

    def call():
        lm.lazymar_layernorm_backward(1, dy, D, 0, None, 0, h.d, tm, tr, None, None, 0, 0, dx, D, dg, db, False, M, D,
                                      ws[0], ws[0].numel())
        lm.lazymar_block8_gelu_backward(1, dy, D, h.d, 1, du, D, None, dbu, False, M, D, ws[1], ws[1].numel())
        lm.lazymar_block8_wgrad(dn, N, h.d, dw, D, False, M, N, D, ws[2], ws[2].numel())
    return call, (h.q, dy, dn), outs


def test_calls_with_workspaces_can_be_captured():
    torch = torch_cuda()
    call, _, outs = _backward_calls()
    call()
    sync()
    want = [t.clone() for t in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for t in outs:
        t.zero_()
    g.replay()
    sync()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_with_workspaces_follow_the_callers_stream():
    """On a side stream, behind work that is still running there and then sets their inputs."""
    torch = torch_cuda()
    call, inputs, outs = _backward_calls()
    call()
    sync()
    want, kept = [t.clone() for t in outs], [t.clone() for t in inputs]
    for t in inputs + tuple(outs):
        t.zero_()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for _ in range(8):
            big = big @ big * 1e-3
        for t, k in zip(inputs, kept):
            t.copy_(k)
        call()
    st.synchronize()
    lm.lazymar_device_check()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_in_a_row_do_not_see_each_others_workspace():
    """Two sets of inputs in turn through one workspace, launched without a wait in between: every result is its own."""
    torch = torch_cuda()
    M, D, N = 3000, 320, 256
    r = rng(33)
    sets = []
    for scale in (1.0, 3.0):
        h, v = held(scale * r.standard_normal((M, D)))
        _, mean, rstd = T.layernorm(v, None, None, EPS)
        sets.append((h, vec(mean), vec(rstd), dev(r.standard_normal((M, D)), "bf16")[0], dev(r.standard_normal((M, N)), "bf16")[0]))
    n = max(lm.lazymar_layernorm_backward_workspace(M, D), lm.lazymar_block8_gelu_backward_workspace(M, D),
            lm.lazymar_block8_wgrad_workspace(M, N, D))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def run(o, h, mean, rstd, dy, dn):
        lm.lazymar_layernorm_backward(1, dy, D, 0, None, 0, h.d, mean, rstd, None, None, 0, 0, o[0], D, o[1], o[2], False, M,
                                      D, ws, n)
        lm.lazymar_block8_gelu_backward(1, dy, D, h.d, 0, None, 0, None, o[3], False, M, D, ws, n)
        lm.lazymar_block8_wgrad(dn, N, h.d, o[4], D, False, M, N, D, ws, n)
    made = [[out(M, D), vec(np.zeros(D)), vec(np.zeros(D)), vec(np.zeros(D)), out(N, D)] for _ in range(42)]
    want = made[:2]
    for o, s in zip(want, sets):
        run(o, *s)
        sync()
    for i, o in enumerate(made[2:]):
        run(o, *sets[i % 2])
    sync()
    for i, o in enumerate(made[2:]):
        assert all(torch.equal(a, b) for a, b in zip(o, want[i % 2])), i
