"""Lists whose tensors do not lie alike, and sizes around the kernels' pieces of 8192 elements (a tensor's first has up to
seven more, in front of its first boundary of eight): gradient norm, clipping and AdamW against the fp64 oracle."""
import math

import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import lazymar as lm
from _gpu import torch_cuda
from test_gpu_optim import adam_bounds, read, state, tensors
from test_gpu_train import BF, U, close, sync

pytestmark = pytest.mark.gpu

PIECE = 8192
SIZES = [[8191], [8192], [8193], [1, 0, 7, 8, 9, 8191, 8192, 8193, 16383, 16385], [8195, 8199, 8200, 24581, 3], [5] * 300,
         [1 << 18, 777]]
PARTS = ("g", "p", "m", "v", "ema", "copy")


def around(offset):
    """Tensors of one list each: a piece, and a piece behind the head, less one, and more by one."""
    head = -offset % 8
    return [[PIECE + head + d] for d in (-1, 0, 1)] + [[2 * PIECE + head + d] for d in (-1, 0, 1)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 3, 7])
def test_norm_around_a_piece(offset, dtype):
    """Sums of eight squares in fp32 (their roundings, 4 U), then in two fp32 numbers or fp64; the norm has half of
    that, and its own rounding."""
    for sizes in SIZES + around(offset):
        _, g, v = tensors(sizes, dtype, offset, seed=30)
        s = state()
        lm.lazymar_grad_norm(lm.lazymar_params_create([dict(g=t) for t in g]), s, 1.0)
        norm, factor, steps, _ = read(s)
        want, f = T.clip_factor(v, 1.0, 1.0)
        assert abs(norm - want) <= 4 * U * want and abs(factor - f) <= 6 * U * f and steps == 1


@pytest.mark.parametrize("scale,most", [(1.0, 1.0), (1.0, 0.25), (2.0 ** -10, 1e-5), (0.5, 3.0)])
def test_factors_below_the_smallest_normal_number(scale, most):
    """Gradients near fp32's end: max_norm / norm is subnormal, a multiple of 2^-149, and clips to max_norm all the same."""
    torch = torch_cuda()
    g = torch.tensor([2.5e38, -1e38, 3e37, 1e30, 0.0], device="cuda")
    v = g.double().cpu().numpy()
    h, s = lm.lazymar_params_create([dict(g=g)]), state()
    lm.lazymar_grad_norm(h, s, most, scale)
    want, f = T.clip_factor([v], scale, most)
    norm, factor, steps, _ = read(s)
    assert f < 2.0 ** -126 and abs(norm - want) <= 4 * U * want and steps == 1
    off = 2.0 ** -150 + 4 * U * f  # half a step of fp32's subnormal numbers
    assert abs(factor - f) <= off
    lm.lazymar_clip_grads(h, s)
    sync()
    close(g, v * f, np.abs(v) * off + U * np.abs(v * f) + 2.0 ** -150)


@pytest.mark.parametrize("src,dst", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("from_, to", [(0, 1), (3, 0), (1, 2), (7, 4), (5, 5), (0, 0)])
def test_clip_to_tensors_that_lie_otherwise(from_, to, src, dst):
    """One rounding to fp32 and one to the output's type; what lies around the outputs stays."""
    torch = torch_cuda()
    for sizes in SIZES + around(from_):
        _, g, v = tensors(sizes, src, from_, seed=31)
        buf, o, _ = tensors(sizes, dst, to, seed=32)
        outside = buf.isnan()
        h = lm.lazymar_params_create([dict(g=a, out=b) for a, b in zip(g, o)])
        for factor in (0.3, 1.0, 0.0):
            lm.lazymar_clip_grads(h, state(1, factor))
            sync()
            f = float(np.float32(factor))
            for a, w in zip(o, v):
                close(a, w * f, np.abs(w * f) * (U + (BF if dst == "bf16" else 0)) * 1.01 + 1e-45)
            assert torch.equal(buf.isnan(), outside)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("where", ["alike"] + ["%s elsewhere" % k for k in PARTS] + ["each elsewhere"])
@pytest.mark.parametrize("offset", [0, 3])
def test_adamw_of_tensors_that_lie_otherwise(offset, where, dtype):
    """A packed gradient buffer with weights of their own, one of a list's buffers displaced, none like another."""
    torch = torch_cuda()
    places = {k: offset for k in PARTS}
    if where == "each elsewhere":
        places = {k: offset + i for i, k in enumerate(PARTS)}
    elif where != "alike":
        places[where.split()[0]] = offset + 1
    for sizes in SIZES + around(places["g"]):
        e, vals, bufs = [dict() for _ in sizes], [dict() for _ in sizes], {}
        for i, (k, d, std) in enumerate(zip(PARTS, (dtype,) + ("fp32",) * 4 + ("bf16",), (1e-2, 1.0, 1e-3, 1e-2, 1.0, 1.0))):
            bufs[k], t, v = tensors(sizes, d, places[k], 33 + i, std)
            for j, (a, b) in enumerate(zip(t, v)):
                if k == "v":
                    a.copy_(a * a)
                    b = a.double().cpu().numpy()
                e[j][k], vals[j][k] = a, b
        outside = {k: b.isnan() for k, b in bufs.items()}
        for i, d in enumerate(e):
            d["weight_decay"] = (0.0, 0.1)[i % 2]
        factor, t = float(np.float32(0.37)), 3
        lm.lazymar_adamw(lm.lazymar_params_create(e), state(t, factor), 1e-2, 0.9, 0.95, 1e-6, ema_decay=0.999)
        sync()
        for d, v in zip(e, vals):
            if not v["p"].size:
                continue
            p, m, vv = T.adamw(v["g"], v["p"], v["m"], v["v"], t, factor, 1e-2, 0.9, 0.95, 1e-6, d["weight_decay"])
            ep, em, ev = adam_bounds(v, t, factor, 1e-2, 0.9, 0.95, 1e-6, d["weight_decay"])
            close(d["p"], p, ep)
            close(d["m"], m, em)
            close(d["v"], vv, ev)
            close(d["ema"], v["ema"] + (1 - 0.999) * (p - v["ema"]), ep + 4 * U * (np.abs(v["ema"]) + np.abs(p)))
            assert torch.equal(d["copy"], d["p"].bfloat16())
        for k, b in bufs.items():
            assert torch.equal(b.isnan(), outside[k]), k


def test_lists_with_pieces_of_twice_the_size():
    """From 2^33 elements on pieces are a multiple of 8192: every element still counts, and is clipped, once."""
    torch = torch_cuda()
    n = (1 << 33) + 3 * PIECE + 5
    buf = torch.zeros(n + 3 + 70001, dtype=torch.bfloat16, device="cuda")
    g, small = buf[3:3 + n], buf[3 + n:]
    at = (0, 4, 5, 2 * PIECE + 4, 2 * PIECE + 5, (1 << 33) - 1, n - 1)
    for i, k in enumerate(at):
        g[k] = 2.0 ** i
    small.fill_(0.125)
    s = state()
    h = lm.lazymar_params_create([dict(g=g), dict(g=small)])
    lm.lazymar_grad_norm(h, s, 1.0)
    want = math.sqrt(sum(4.0 ** i for i in range(len(at))) + 70001 / 64)
    norm, factor, _, _ = read(s)
    assert abs(norm - want) <= 4 * U * want
    lm.lazymar_clip_grads(h, s)
    sync()
    for i, k in enumerate(at):
        assert abs(float(g[k]) - 2.0 ** i * factor) <= BF * 2.0 ** i * factor
    assert (small == (torch.tensor(0.125, device="cuda") * factor).bfloat16()).all()
    assert sum(int(part.count_nonzero()) for part in g.split(1 << 31)) == len(at)
    del buf, g, small, h
    torch.cuda.empty_cache()
