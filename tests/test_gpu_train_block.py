"""The training operators together: the MLP half of a block against fp64, its
gradient against differences of the function that it computes, and the example."""
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import training as T
from _gpu import torch_cuda

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _params(D, H, seed):
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s)  # noqa: E731
    return dict(ln_g=1 + 0.1 * n(D), ln_b=0.02 * n(D), w1=n(H, D) / np.sqrt(D), b1=0.02 * n(H), w2=n(D, H) / np.sqrt(H),
                b2=0.02 * n(D))


def _exact(p, x, dy):
    """y, dx and the parameters' gradients in fp64, with nothing rounded to 8 bits."""
    h, mean, rstd = T.layernorm(x, p["ln_g"], p["ln_b"], 1e-6)
    u = h @ p["w1"].T + p["b1"]
    a = T.gelu(u)
    y = x + a @ p["w2"].T + p["b2"]
    du = (dy @ p["w2"]) * T.gelu_grad(u)
    dx, dg, db = T.layernorm_grad(du @ p["w1"], x, mean, rstd, p["ln_g"])
    return y, dx + dy, dict(ln_g=dg, ln_b=db, w1=du.T @ h, b1=du.sum(0), w2=dy.T @ a, b2=dy.sum(0))


def _block(p):
    torch = torch_cuda()
    from paper_2503_12450_gb300.mlp_block8 import MlpBlock8
    return MlpBlock8({k: torch.from_numpy(v.astype(np.float32)).cuda() for k, v in p.items()})


@pytest.mark.parametrize("M,D,H", [(1, 128, 512), (333, 200, 800), (1500, 256, 1024), (64, 777, 1554)])
def test_mlp_block_against_fp64(M, D, H):
    """Every 8-bit tensor is off by at most 2^-4 of each element, about 2^-4 / sqrt(3) of its norm where the errors are
    independent; a result passes through at most six such tensors, so its norm is off by at most
    sqrt(6) 2^-4 / sqrt(3) < 9 %. y and dx carry the residual stream in fp32 besides."""
    torch = torch_cuda()
    p = _params(D, H, 1)
    r = np.random.default_rng(M)
    x, dy = r.standard_normal((M, D)), 1e-3 * r.standard_normal((M, D))
    x, dy = x.astype(np.float32).astype(float), dy.astype(np.float32).astype(float)
    b = _block(p)
    y = b.forward(torch.from_numpy(x.astype(np.float32)).cuda())
    dx = b.backward(torch.from_numpy(dy.astype(np.float32)).cuda())
    torch.cuda.synchronize()
    wy, wdx, wg = _exact(p, x, dy)
    off = lambda a, w: np.linalg.norm(a.double().cpu().numpy() - w) / np.linalg.norm(w)  # noqa: E731
    assert off(y, wy) < 0.09 and off(dx, wdx) < 0.09
    for k, w in wg.items():
        assert off(b.grads[k], w) < 0.09, k
    # serving the same rows keeps nothing and gives the same
    s = b.forward(torch.from_numpy(x.astype(np.float32)).cuda(), train=False)
    assert torch.equal(s, y)
    # accumulation adds a second pass's gradients
    first = {k: v.clone() for k, v in b.grads.items()}
    b.forward(torch.from_numpy(x.astype(np.float32)).cuda())
    b.backward(torch.from_numpy(dy.astype(np.float32)).cuda(), accumulate=True)
    for k, v in b.grads.items():
        assert torch.equal(v, first[k] + first[k]), k


def test_mlp_block_gradient_against_differences():
    """The directional derivative of the loss along the gradient, by differences of the forward pass itself: rounding to
    8 bits makes the loss a staircase, so the step is large against a stair and the agreement that of its noise."""
    torch = torch_cuda()
    D, H, M = 256, 1024, 2048
    p = _params(D, H, 5)
    b = _block(p)
    g = torch.Generator(device="cuda").manual_seed(6)
    x, t = (torch.randn((M, D), device="cuda", generator=g) for _ in range(2))

    def loss():
        return float(((b.forward(x) - t).double() ** 2).sum() / 2)
    y = b.forward(x)
    b.backward(y - t)
    for k in ("w1", "w2", "b1", "ln_g"):
        d = b.grads[k].clone()
        slope = float((d.double() ** 2).sum())
        h = 0.1 * float(b.p[k].norm() / d.norm())
        keep = b.p[k].clone()
        b.p[k].copy_(keep + h * d)
        b.pack()
        up = loss()
        b.p[k].copy_(keep - h * d)
        b.pack()
        down = loss()
        b.p[k].copy_(keep)
        b.pack()
        got = (up - down) / (2 * h)
        # the third-order term of a 10 % step and the 8-bit noise of two losses
        assert abs(got - slope) < 0.15 * slope, (k, got, slope)


def test_example_learns():
    torch_cuda()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import tune_mlp
    finally:
        sys.path.pop(0)
    losses, student, _ = tune_mlp.tune(256, 2048, 25)
    assert losses[-1] < 0.5 * losses[0] and all(np.isfinite(losses))
    assert student.saved_bytes() < 0.53 * 4 * 2048 * (256 + 1024)


def test_example_runs_from_the_command_line():
    torch_cuda()
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "tune_mlp.py"), "--width", "256", "--rows", "640",
                        "--steps", "4"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "ms a step" in r.stdout and "8 bits" in r.stdout


def _tensors(M, D, seed):
    torch = torch_cuda()
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((M, D), device="cuda", generator=g) for _ in range(2)]


def test_serving_between_forward_and_backward_leaves_what_was_kept():
    torch = torch_cuda()
    b = _block(_params(256, 1024, 7))
    x, dy = _tensors(300, 256, 8)
    b.forward(x)
    want_dx = b.backward(dy)
    want = {k: v.clone() for k, v in b.grads.items()}
    for rows in (300, 7):  # as many rows as are kept, and another number
        b.forward(x)
        b.forward(3 * _tensors(rows, 256, 9)[0], train=False)
        assert torch.equal(b.backward(dy), want_dx)
        for k, v in b.grads.items():
            assert torch.equal(v, want[k]), k


def test_backward_needs_its_forward_pass():
    torch_cuda()
    from paper_2503_12450_gb300.lazymar import LazymarError
    b = _block(_params(256, 1024, 7))
    x, dy = _tensors(300, 256, 8)
    with pytest.raises(LazymarError, match="forward"):
        b.backward(dy)
    b.forward(x, train=False)
    with pytest.raises(LazymarError, match="forward"):
        b.backward(dy)
    b.forward(x)
    for other in (dy[:299], dy[:, :255]):
        with pytest.raises(LazymarError, match="dy"):
            b.backward(other)


def test_block_takes_fp32_rows_of_any_stride_only():
    torch = torch_cuda()
    from paper_2503_12450_gb300.lazymar import LazymarError
    b = _block(_params(256, 1024, 7))
    x, dy = _tensors(300, 256, 8)
    y = b.forward(x)
    dx = b.backward(dy)
    wide = [torch.zeros((300, 301), device="cuda") for _ in range(2)]
    for w, v in zip(wide, (x, dy)):
        w[:, 1:257] = v
    assert torch.equal(b.forward(wide[0][:, 1:257]), y)
    # (the gradient of the residual stream comes in rows off the boundary, which another kernel sums)
    got = b.backward(wide[1][:, 1:257])
    assert float((got - dx).norm() / dx.norm()) < 1e-5
    one = torch.empty((1, 512), device="cuda")[:, :256].copy_(x[:1])
    assert torch.equal(b.forward(one), b.forward(x[:1]))
    for other in (x.double(), x.bfloat16(), x[:, :255], x[0], torch.zeros((300, 512), device="cuda")[:, ::2]):
        with pytest.raises(LazymarError, match="x:"):
            b.forward(other)
        with pytest.raises(LazymarError, match="x:"):
            b.forward(other, train=False)
    b.forward(x)
    for other in (dy.double(), dy.bfloat16(), torch.zeros((300, 512), device="cuda")[:, ::2]):
        with pytest.raises(LazymarError, match="dy"):
            b.backward(other)


def test_block_without_rows():
    torch = torch_cuda()
    b = _block(_params(256, 1024, 7))
    none = torch.empty((0, 256), device="cuda")
    assert b.forward(none, train=False).shape == (0, 256)
    assert b.forward(none).shape == (0, 256)
    for v in b.grads.values():
        v.fill_(1.0)
    assert b.backward(none).shape == (0, 256)
    torch.cuda.synchronize()
    for k, v in b.grads.items():
        assert not v.any(), k


def test_example_leaves_its_teacher(monkeypatch):
    torch = torch_cuda()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import tune_mlp
    finally:
        sys.path.pop(0)
    made = []

    class Kept(tune_mlp.MlpBlock8):
        def __init__(self, *args):
            super().__init__(*args)
            made.append((self, {k: v.clone() for k, v in self.p.items()}))
    monkeypatch.setattr(tune_mlp, "MlpBlock8", Kept)
    tune_mlp.tune(256, 512, 3)
    teacher, was = made[0]
    for k, v in teacher.p.items():
        assert torch.equal(v, was[k]), k


FIRST_CALLS = """
import torch
from paper_2503_12450_gb300 import lazymar as lm
F, B = (lm.LAZYMAR_F32, torch.float32), (lm.LAZYMAR_BF16, torch.bfloat16)
bad = []
for D, dy_t, x_t, res in %s:
    M = 40
    dy_t = {"f": F, "b": B}[dy_t]
    dy = torch.zeros((M, D), dtype=dy_t[1], device="cuda")
    x, x8 = None, None
    if x_t == "8":
        q, s = torch.zeros((M, D), dtype=torch.uint8, device="cuda"), torch.ones((-(-D // 128), M), dtype=torch.uint8, device="cuda")
        x8 = lm.lazymar_block8(q, s)
        x_t = F
    else:
        x_t = {"f": F, "b": B}[x_t]
        x = torch.zeros((M, D), dtype=x_t[1], device="cuda")
    mean, rstd = torch.zeros(M, device="cuda"), torch.ones(M, device="cuda")
    dres = torch.zeros((M, D), device="cuda") if res else None
    dx = torch.ones((M, D), device="cuda")
    try:
        lm.lazymar_layernorm_backward(dy_t[0], dy, D, x_t[0], x, D, x8, mean, rstd, None, dres, D, F[0], dx, D, None,
                                      None, False, M, D, None, 0)
        torch.cuda.synchronize()
        assert not dx.any()
    except Exception as e:
        bad.append((D, str(e)))
assert not bad, bad
"""


@pytest.mark.parametrize("calls", [
    [(128, "f", "f", True), (256, "b", "f", False), (512, "b", "f", False), (768, "b", "b", False),
     (1536, "b", "b", False), (1024, "b", "8", False), (2048, "b", "8", False), (4096, "b", "8", False)],
    [(256, "f", "b", False), (512, "f", "b", False), (1280, "b", "8", True), (640, "b", "f", True)]])
def test_first_layernorm_backward_of_a_process(calls):
    """Every kernel's first call: what an earlier, larger call has set up does not carry it."""
    torch_cuda()
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % calls], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
