"""Parity of the gradient norm, clipping and AdamW over lists of tensors with the fp64 oracle
(oracle/training.py), through the C ABI, at the sizes, types, alignments and values where they can go wrong."""
import math

import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import lazymar as lm
from _gpu import torch_cuda
from test_gpu_train import BF, U, close, rng, sync

pytestmark = pytest.mark.gpu

PIECE = 4096


def state(steps=0, factor=0.0, skipped=0):
    torch = torch_cuda()
    s = torch.zeros(4, device="cuda")
    s[1] = factor
    s.view(torch.int32)[2], s.view(torch.int32)[3] = steps, skipped
    return s


def read(s):
    torch = torch_cuda()
    sync()
    i = s.view(torch.int32).cpu()
    return float(s[0]), float(s[1]), int(i[2]), int(i[3])


def tensors(sizes, dtype="fp32", offset=0, seed=1, std=1.0, guard=float("nan")):
    """Tensors in one buffer, `offset` elements into it and three elements apart (offset 0: on boundaries of 64), between
    guards; and their values."""
    torch = torch_cuda()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = rng(len(sizes), offset, seed)
    at, places = offset, []
    for n in sizes:
        places.append(at)
        at += n + 3 if offset else -(-n // 64) * 64 + 64
    buf = torch.full((at + 64,), guard, dtype=t, device="cuda")
    views = [buf[a:a + n] for a, n in zip(places, sizes)]
    for i, v in enumerate(views):
        v.copy_(torch.from_numpy((std * r.standard_normal(v.numel()) * 2.0 ** (i % 5)).astype(np.float32)))
    return buf, views, [v.double().cpu().numpy() for v in views]


LISTS = [[1], [7], [8, 0, 1], [4096], [4097, 3], [100, 5000, 12345], [1 << 20], [65537, 2, 4095, 4096, 70001], [3] * 300,
         [1000 * 777, 777, 5]]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 5])
@pytest.mark.parametrize("sizes", LISTS, ids=str)
def test_norm(sizes, offset, dtype):
    """fp32 sums of 16 squares (their rounding and at most eight adds in a row: 10 U), then fp64; the norm has half of
    that, and its own rounding."""
    _, g, v = tensors(sizes, dtype, offset)
    h = lm.lazymar_params_create([dict(g=t) for t in g])
    s = state(5)
    for scale, most in ((1.0, 1e30), (0.25, 0.5), (3.0, math.inf)):
        lm.lazymar_grad_norm(h, s, most, scale)
        norm, factor, steps, skipped = read(s)
        want, f = T.clip_factor(v, scale, most)
        assert abs(norm - want) <= 8 * U * want and abs(factor - f) <= 10 * U * f
    assert (steps, skipped) == (8, 0)


def test_norm_of_values_whose_squares_leave_fp32():
    torch = torch_cuda()
    for big in (1e30, 3e37, 1e-30, 1e-42, 1.0):
        x = torch.zeros(10000, device="cuda")
        x[::7] = big
        x[5000:5100] = 1e-44  # squares vanish beside others, and are all there is elsewhere
        h = lm.lazymar_params_create([dict(g=x)])
        s = state()
        lm.lazymar_grad_norm(h, s, math.inf)
        want = T.clip_factor([x.double().cpu().numpy()], 1.0, math.inf)[0]
        norm, factor, steps, skipped = read(s)
        if want >= 2.0 ** 128:  # 3e37 sqrt(1429) = 1.1e39, which fp32 does not hold: as documented
            assert (norm, factor, steps, skipped) == (math.inf, 0.0, 0, 1)
            continue
        assert abs(norm - want) <= 8 * U * want + 2.0 ** -149 and factor == 1.0 and steps == 1
    # one small value among zeros
    x = torch.zeros(9000, device="cuda")
    x[8999] = 1e-25
    s = state()
    lm.lazymar_grad_norm(lm.lazymar_params_create([dict(g=x)]), s, 1.0)
    assert abs(read(s)[0] - 1e-25) <= 1e-31
    # a factor that fp32 has no number for is not taken for a skipped step (of 16 elements the norm, 4e38, is no fp32 number)
    for n, taken in ((16, 0), (9, 1)):
        x = torch.full((n,), 1e38, device="cuda")
        s = state()
        lm.lazymar_grad_norm(lm.lazymar_params_create([dict(g=x)]), s, 1e-30)
        norm, factor, steps, skipped = read(s)
        assert (factor > 0.0) == bool(taken) and factor <= 2.0 ** -126 and (steps, skipped) == (taken, 1 - taken)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 4095, 50000, 99999])
def test_norm_that_is_not_finite_skips(at, value, dtype):
    torch = torch_cuda()
    g = torch.ones(100000, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    g[at] = value
    h = lm.lazymar_params_create([dict(g=g), dict(g=torch.ones(3, device="cuda"))])
    s = state(4, 0.5, 2)
    lm.lazymar_grad_norm(h, s, 1.0)
    norm, factor, steps, skipped = read(s)
    assert not math.isfinite(norm) and factor == 0.0 and (steps, skipped) == (4, 3)


def test_norm_beyond_fp32_skips():
    torch = torch_cuda()
    g = torch.full((100,), 3e38, device="cuda")
    s = state()
    lm.lazymar_grad_norm(lm.lazymar_params_create([dict(g=g)]), s, 1.0)
    assert read(s)[1:] == (0.0, 0, 1)
    lm.lazymar_grad_norm(lm.lazymar_params_create([dict(g=g)]), s, 1.0, scale=0.05)  # 1.5e38 is one
    norm, factor, steps, skipped = read(s)
    assert abs(norm - 1.5e38) < 1e32 and (steps, skipped) == (1, 1)


def test_empty_lists():
    torch = torch_cuda()
    none = torch.empty(0, device="cuda")
    for h in (lm.lazymar_params_create([]), lm.lazymar_params_create([dict(g=none), dict(g=none)])):
        s = state(1)
        lm.lazymar_grad_norm(h, s, 1.0, scale=0.5)
        lm.lazymar_clip_grads(h, s)
        lm.lazymar_adamw(h, s, 1e-3)
        assert read(s) == (0.0, 0.5, 2, 0)


def test_norm_of_a_tensor_beyond_32_bits():
    torch = torch_cuda()
    n = (1 << 32) + 4097
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[1 << 31], g[1 << 32], g[n - 1] = 1.0, 2.0, 3.0, 4.0
    h = lm.lazymar_params_create([dict(g=g)])
    s = state()
    lm.lazymar_grad_norm(h, s, 1.0)
    norm, factor, _, _ = read(s)
    assert abs(norm - math.sqrt(30.0)) <= 8 * U * math.sqrt(30.0)
    lm.lazymar_clip_grads(h, s)
    sync()
    for at, v in ((0, 1.0), (1 << 31, 2.0), (1 << 32, 3.0), (n - 1, 4.0)):
        assert abs(float(g[at]) - v * factor) <= BF * v * factor
    del g, h
    torch.cuda.empty_cache()


# --------------------------------------------------------------------------
# Clipping
# --------------------------------------------------------------------------
@pytest.mark.parametrize("src,dst", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("sizes", [[1], [4097, 3, 0, 8191], [1 << 18, 777], [5] * 200], ids=str)
def test_clip(sizes, offset, src, dst):
    torch = torch_cuda()
    _, g, v = tensors(sizes, src, offset, 2)
    buf, o, _ = tensors(sizes, dst, offset, 3)
    outside = buf.isnan()
    h = lm.lazymar_params_create([dict(g=a, out=b) for a, b in zip(g, o)])
    for factor in (0.3, 1.0, 7.5):
        lm.lazymar_clip_grads(h, state(1, factor))
        sync()
        f = float(np.float32(factor))
        for a, w in zip(o, v):
            close(a, w * f, np.abs(w * f) * (U + (BF if dst == "bf16" else 0)) * 1.01 + 1e-45)
        assert torch.equal(buf.isnan(), outside)
    if src == dst:
        want = [a.clone() for a in o]
        inplace = lm.lazymar_params_create([dict(g=a) for a in g])
        lm.lazymar_clip_grads(inplace, state(1, 1.0))
        sync()
        for a, w in zip(g, v):
            assert (a.double().cpu().numpy() == w).all()
        lm.lazymar_clip_grads(inplace, state(1, 7.5))
        sync()
        for a, w in zip(g, want):
            assert torch.equal(a, w)


def test_clip_of_a_skipped_step_gives_zeros():
    torch = torch_cuda()
    g = torch.ones(5001, device="cuda")
    g[7], g[5000] = float("inf"), float("nan")
    o = torch.ones(5001, dtype=torch.bfloat16, device="cuda")
    for h, t in ((lm.lazymar_params_create([dict(g=g, out=o)]), o), (lm.lazymar_params_create([dict(g=g)]), g)):
        s = state()
        lm.lazymar_grad_norm(h, s, 1.0)
        lm.lazymar_clip_grads(h, s)
        sync()
        assert not t.any()


# --------------------------------------------------------------------------
# AdamW
# --------------------------------------------------------------------------
def adam_bounds(v, t, factor, lr, b1, b2, eps, wd):
    """m and v: a few roundings of their terms. The step's relative error: 1 - beta^t (the logarithm's rounding, its
    product with t, expm1 and a division: 8 U, half of that behind the square root), root, sum and two divisions;
    and what m's and v's own errors move it by."""
    g = np.abs(v["g"] * factor)
    m, vv = b1 * np.abs(v["m"]) + (1 - b1) * g, b2 * v["v"] + (1 - b2) * g * g
    em, ev = 4 * U * (np.abs(v["m"]) + (1 - b1) * g + m), 5 * U * (v["v"] + (1 - b2) * g * g + vv)
    c1, c2 = 1 - b1 ** t, 1 - b2 ** t
    root = np.sqrt(vv / c2)
    den = root + eps
    step = m / c1 / den
    es = step * 24 * U + em / c1 / den + step * np.where(vv > 0, ev / np.maximum(2 * vv, 1e-300), 0) * root / den
    ep = lr * es + 4 * U * (np.abs(v["p"]) * (1 + lr * wd) + lr * step)
    return ep + 1e-44, em + 1e-44, ev + 1e-44


def weights(sizes, dtype="fp32", offset=0, ema=True, copy=True, seed=4):
    e, vals, bufs = [dict() for _ in sizes], [dict() for _ in sizes], {}
    for i, (k, d, std) in enumerate((("g", dtype, 1e-2), ("p", "fp32", 1.0), ("m", "fp32", 1e-3), ("v", "fp32", 1e-2),
                                     ("ema", "fp32", 1.0), ("copy", "bf16", 1.0))):
        if (k == "ema" and not ema) or (k == "copy" and not copy):
            continue
        bufs[k], t, v = tensors(sizes, d, offset, seed + i, std)
        for j, (a, b) in enumerate(zip(t, v)):
            if k == "v":
                a.copy_(a * a)
                b = a.double().cpu().numpy()
            e[j][k], vals[j][k] = a, b
    return e, vals, bufs


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset,ema,copy", [(0, True, True), (3, True, True), (0, False, False), (1, False, True)])
@pytest.mark.parametrize("sizes", [[1], [4097, 3, 0, 8191], [1 << 18, 777], [5] * 200], ids=str)
def test_adamw(sizes, offset, ema, copy, dtype):
    torch = torch_cuda()
    e, vals, bufs = weights(sizes, dtype, offset, ema, copy)
    outside = {k: b.isnan() for k, b in bufs.items()}
    for i, d in enumerate(e):
        d["lr_scale"], d["weight_decay"] = (1.0, 0.5, 2.0)[i % 3], (0.0, 0.1)[i % 2]
    h = lm.lazymar_params_create(e)
    kw = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6)
    factor, t = float(np.float32(0.37)), 3
    lm.lazymar_adamw(h, state(t, factor), ema_decay=0.999, **kw)
    sync()
    for d, v in zip(e, vals):
        if not v["p"].size:
            continue
        lr, wd = 1e-2 * d["lr_scale"], d["weight_decay"]
        p, m, vv = T.adamw(v["g"], v["p"], v["m"], v["v"], t, factor, lr, 0.9, 0.95, 1e-6, wd)
        ep, em, ev = adam_bounds(v, t, factor, lr, 0.9, 0.95, 1e-6, wd)
        close(d["p"], p, ep)
        close(d["m"], m, em)
        close(d["v"], vv, ev)
        if ema:
            close(d["ema"], v["ema"] + (1 - 0.999) * (p - v["ema"]), ep + 4 * U * (np.abs(v["ema"]) + np.abs(p)))
        if copy:
            assert torch.equal(d["copy"], d["p"].bfloat16())
    for k, b in bufs.items():
        assert torch.equal(b.isnan(), outside[k]), k


def test_adamw_first_and_late_steps():
    """1 - beta^t from the first step (1e-4 at beta 0.9999) to where it is 1, against the formula in fp64."""
    torch = torch_cuda()
    for t in (1, 2, 10, 1000, 10 ** 6, 2 ** 31 - 1):
        for b1, b2 in ((0.9, 0.999), (0.0, 0.9999), (0.95, 0.0)):
            e, vals, _ = weights([1000], seed=t % 1000 + 5)
            v = vals[0]
            lm.lazymar_adamw(lm.lazymar_params_create(e), state(t, 1.0), 1e-3, b1, b2, 1e-8)
            sync()
            p, m, vv = T.adamw(v["g"], v["p"], v["m"], v["v"], t, 1.0, 1e-3, b1, b2, 1e-8)
            ep, em, ev = adam_bounds(v, t, 1.0, 1e-3, b1, b2, 1e-8, 0.0)
            close(e[0]["p"], p, ep)
            close(e[0]["m"], m, em)
            close(e[0]["v"], vv, ev)


def test_adamw_without_state_with_a_learning_rate_on_the_device_and_skipped():
    torch = torch_cuda()
    e, _, _ = weights([5000, 33], seed=6)
    keep = [{k: t.clone() for k, t in d.items()} for d in e]
    h = lm.lazymar_params_create(e)

    def back():
        for d, k in zip(e, keep):
            for n in k:
                d[n].copy_(k[n])
    lm.lazymar_adamw(h, state(7, 0.5), 1e-3, ema_decay=0.9)
    want = [{k: t.clone() for k, t in d.items()} for d in e]
    back()
    lm.lazymar_adamw(h, None, 1e-3, ema_decay=0.9, factor=0.5, steps=7)
    sync()
    assert all(torch.equal(d[k], w[k]) for d, w in zip(e, want) for k in w)
    back()
    lm.lazymar_adamw(h, state(7, 0.5), 123.0, ema_decay=0.9, lr_device=torch.tensor([1e-3], device="cuda"))
    sync()
    assert all(torch.equal(d[k], w[k]) for d, w in zip(e, want) for k in w)
    back()
    e[0]["g"][3] = float("nan")
    s = state(7, 0.5)
    lm.lazymar_grad_norm(h, s, 1.0)
    lm.lazymar_adamw(h, s, 1e-3)
    assert read(s)[1:] == (0.0, 7, 1)
    for d, k in zip(e, keep):
        for n in ("p", "m", "v", "ema", "copy"):
            assert torch.equal(d[n], k[n])


def test_adamw_needs_weights():
    torch = torch_cuda()
    h = lm.lazymar_params_create([dict(g=torch.ones(4, device="cuda"))])
    with pytest.raises(lm.LazymarError, match="no weights"):
        lm.lazymar_adamw(h, state(1, 1.0), 1e-3)
    with pytest.raises(lm.LazymarError, match="state"):
        lm.lazymar_clip_grads(h, None)
    with pytest.raises(lm.LazymarError, match="state"):
        lm.lazymar_grad_norm(h, torch.zeros(4), 1.0)
    h.close()
    h.close()


def test_lists_refuse_overlapping_tensors():
    """A weight that is in a list twice would be updated twice at once."""
    torch = torch_cuda()
    new = lambda: torch.zeros(100, device="cuda")  # noqa: E731
    one = lambda **k: dict(dict(g=new(), p=new(), m=new(), v=new()), **k)  # noqa: E731
    a, buf = one(), torch.zeros(300, device="cuda")
    for entries in ([a, a], [a, one(p=a["p"])], [one(m=a["m"], v=a["m"])], [one(g=buf[:100], p=buf[99:199])], [one(out=a["p"], p=a["p"])],
                    [one(), one(p=buf[:100], ema=buf[50:150])]):
        with pytest.raises(lm.LazymarError, match="overlap"):
            lm.lazymar_params_create(entries)
    lm.lazymar_params_create([one(g=buf[:100], p=buf[100:200], m=buf[200:300]), one(out=None)]).close()
    g = new()
    lm.lazymar_params_create([dict(g=g, out=g), dict(g=buf[:0]), dict(g=buf[:100], out=buf[100:200])]).close()


def test_norm_of_zeros_with_a_few_others():
    torch = torch_cuda()
    for t in (torch.float32, torch.bfloat16):
        x = torch.zeros(200001, dtype=t, device="cuda")
        h, s = lm.lazymar_params_create([dict(g=x)]), state()
        for values in ({}, {17: 1e-38, 199999: -1e-38}, {5: -0.0, 100000: 3.0}):
            x.zero_()
            for i, w in values.items():
                x[i] = w
            want = math.sqrt(float((x.double() ** 2).sum()))
            lm.lazymar_grad_norm(h, s, math.inf)
            assert abs(read(s)[0] - want) <= 2 * U * want  # the squares' sum is exact, or in fp64


def test_lists_mix_tensors_with_and_without_averages():
    torch = torch_cuda()
    e, vals, _ = weights([4096, 4096, 100], seed=7)
    del e[0]["ema"], e[1]["copy"]
    h = lm.lazymar_params_create(e)
    lm.lazymar_adamw(h, state(2, 1.0), 1e-3, ema_decay=0.5)
    sync()
    for d, v in zip(e, vals):
        p = T.adamw(v["g"], v["p"], v["m"], v["v"], 2, 1.0, 1e-3, 0.9, 0.999, 1e-8)[0]
        close(d["p"], p, adam_bounds(v, 2, 1.0, 1e-3, 0.9, 0.999, 1e-8, 0.0)[0])
        if "ema" in d:
            assert float((d["ema"].double() - 0.5 * (torch.from_numpy(v["ema"]).cuda() + d["p"].double())).abs().max()) < 1e-6
        if "copy" in d:
            assert torch.equal(d["copy"], d["p"].bfloat16())


# --------------------------------------------------------------------------
# Together
# --------------------------------------------------------------------------
def test_steps_in_a_row_against_fp64_and_in_a_graph():
    """Norm and update of ten steps, the gradients changing: eagerly, and captured once and replayed, bit for bit the
    same; and the weights near those of fp64 (an error of a step's bound each)."""
    torch = torch_cuda()
    sizes = [70000, 4096, 33, 5]
    r = rng(8)
    steps = [[(s * r.standard_normal(n)).astype(np.float32) for n in sizes] for s in (0.01, 1.0, 0.1, 5.0, 0.02, np.inf, 0.3, 1.0, 2.0, 0.5)]
    for i in range(len(sizes)):
        steps[5][i][~np.isfinite(steps[5][i])] = 0
        steps[5][i][0] = np.nan
    kw = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, ema_decay=0.99)
    ends = []
    for captured in (False, True):
        e, vals, _ = weights(sizes, seed=9)
        h, s = lm.lazymar_params_create(e), state()
        graph = None
        for k, grads in enumerate(steps):
            for d, g in zip(e, grads):
                d["g"].copy_(torch.from_numpy(g))
            if captured and k == 3:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    lm.lazymar_grad_norm(h, s, 1.0)
                    lm.lazymar_adamw(h, s, **kw)
            if graph is not None:
                graph.replay()
            else:
                lm.lazymar_grad_norm(h, s, 1.0)
                lm.lazymar_adamw(h, s, **kw)
        assert read(s)[2:] == (9, 1)
        ends.append([{k: t.clone() for k, t in d.items()} for d in e])
    assert all(torch.equal(a[k], b[k]) for a, b in zip(*ends) for k in ("p", "m", "v", "ema", "copy"))
    want = [(v["p"], v["m"], v["v"]) for v in vals]
    t = 0
    for grads in steps:
        f = T.clip_factor(grads, 1.0, 1.0)[1]
        if f == 0.0:
            continue
        t += 1
        want = [T.adamw(g, *w, t, f, 1e-3, 0.9, 0.95, 1e-8) for g, w in zip(grads, want)]
    for d, w in zip(ends[0], want):
        assert float(np.abs(d["p"].double().cpu().numpy() - w[0]).max()) < 9 * (4 * U * 6 + 1e-3 * 200 * U)


def test_norm_is_the_same_from_call_to_call_and_on_another_stream():
    torch = torch_cuda()
    _, g, _ = tensors([1 << 20, 12345, 7], "bf16", 0, 10)
    h, s = lm.lazymar_params_create([dict(g=t) for t in g]), state()
    lm.lazymar_grad_norm(h, s, 0.1)
    want = read(s)[:2]
    for _ in range(5):
        lm.lazymar_grad_norm(h, s, 0.1)
        assert read(s)[:2] == want
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lm.lazymar_grad_norm(h, s, 0.1)
    side.synchronize()
    assert read(s)[:2] == want
