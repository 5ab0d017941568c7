"""The residual join, the 8-bit products, the gradient norm and AdamW together: a stack of modulated, gated MLP
blocks against fp64, its gradient against differences, training steps eagerly and from a graph."""
import math

import numpy as np
import pytest

from oracle import training as T
from _gpu import torch_cuda

pytestmark = pytest.mark.gpu


def _blocks(depth, D, H, seed):
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    return [dict(w1=n(H, D) / np.float32(D ** 0.5), b1=0.02 * n(H), w2=n(D, H) / np.float32(H ** 0.5), b2=0.02 * n(D))
            for _ in range(depth)]


def _stack(blocks):
    torch = torch_cuda()
    from paper_2503_12450_gb300.gated_mlp8 import GatedMlpStack8
    return GatedMlpStack8([{k: torch.from_numpy(v.copy()).cuda() for k, v in b.items()} for b in blocks])


def _exact(blocks, x, mod, group, dz):
    """z, dx, dmod and the parameters' gradients in fp64, with nothing rounded to 8 bits."""
    M, D = x.shape
    at = lambda i, j: mod[:, (3 * i + j) * D:(3 * i + j + 1) * D]  # noqa: E731
    kept, z = [], x
    for i, b in enumerate(blocks):
        o = T.join(z, None, pre="layer", group=group, shift=at(i, 0), scale=at(i, 1))
        u = o["h"] @ b["w1"].astype(float).T + b["b1"]
        a = T.gelu(u)
        y = a @ b["w2"].astype(float).T + b["b2"]
        kept.append((z, o, u, a, y))
        z = T.join(z, y, group=group, gate=at(i, 2))["z"]
    dmod, grads, d = np.zeros_like(mod), {}, dz
    for i in range(len(blocks) - 1, -1, -1):
        b, (zi, o, u, a, y) = blocks[i], kept[i]
        g = T.join_grad(None, d, None, y, group=group, gate=at(i, 2))
        dmod[:, (3 * i + 2) * D:(3 * i + 3) * D] = g["dgate"]
        du = (g["dy"] @ b["w2"].astype(float)) * T.gelu_grad(u)
        grads.update({"%d.w2" % i: g["dy"].T @ a, "%d.b2" % i: g["dy"].sum(0), "%d.w1" % i: du.T @ o["h"], "%d.b1" % i: du.sum(0)})
        g = T.join_grad(du @ b["w1"].astype(float), g["dx"], zi, None, pre="layer", group=group, scale=at(i, 1), z_mean=o["z_mean"],
                        z_rstd=o["z_rstd"])
        dmod[:, 3 * i * D:(3 * i + 1) * D], dmod[:, (3 * i + 1) * D:(3 * i + 2) * D] = g["dshift"], g["dscale"]
        d = g["dx"]
    return z, d, dmod, grads


def _inputs(depth, M, D, group, seed):
    r = np.random.default_rng(seed)
    rows = -(-M // group) if group else 1
    x, dz = r.standard_normal((M, D)).astype(np.float32), (1e-3 * r.standard_normal((M, D))).astype(np.float32)
    mod = (0.3 * r.standard_normal((rows, 3 * D * depth))).astype(np.float32)
    mod.reshape(rows, depth, 3, D)[:, :, 2] += 0.7  # gates
    return x, dz, mod


@pytest.mark.parametrize("M,D,H,group", [(1, 128, 512, 1), (333, 200, 800, 0), (1500, 256, 1024, 100), (640, 384, 768, 1),
                                         (64, 777, 1554, 7)])
def test_stack_against_fp64(M, D, H, group):
    """Every 8-bit tensor is off by about 2^-4 / sqrt(3) = 3.6 % of its norm. Two blocks: a gradient passes through at most
    twelve such tensors (h, w1, u, a, w2 and y of either block, forward or back), so it is off by at most sqrt(12) 3.6 % =
    12.5 %; the modulation's bf16 rounding is far below that. z and dx carry the stream in fp32 besides."""
    torch = torch_cuda()
    blocks = _blocks(2, D, H, 1)
    x, dz, mod = _inputs(2, M, D, group, M)
    s = _stack(blocks)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    z = s.forward(dev(x), dev(mod), group)
    dx, dmod = s.backward(dev(dz))
    torch.cuda.synchronize()
    wz, wdx, wdmod, wg = _exact(blocks, x.astype(float), mod.astype(float), group, dz.astype(float))
    off = lambda a, w: np.linalg.norm(a.double().cpu().numpy() - w) / np.linalg.norm(w)  # noqa: E731
    assert off(z, wz) < 0.125 and off(dx, wdx) < 0.125 and off(dmod, wdmod) < 0.125
    for k, w in wg.items():
        assert off(s.grads[k], w) < 0.125, k
    assert torch.equal(s.forward(dev(x), dev(mod), group, train=False), z)
    # a second pass adds; bf16 modulation gives bf16 gradients
    first = {k: v.clone() for k, v in s.grads.items()}
    s.backward(dev(dz), accumulate=True)
    for k, v in s.grads.items():
        assert torch.equal(v, first[k] + first[k]), k
    half = dev(mod).bfloat16()
    s.forward(dev(x), half, group)
    assert s.backward(dev(dz))[1].dtype == torch.bfloat16


def test_stack_gradient_against_differences():
    """By differences of the forward pass itself, whose 8-bit roundings make it a staircase: a step of 10 % of each input's
    norm is large against a stair; what is left is the third-order term and the noise of two losses."""
    torch = torch_cuda()
    D, H, M, group = 256, 1024, 2048, 128
    s = _stack(_blocks(2, D, H, 5))
    x, _, mod = _inputs(2, M, D, group, 6)
    x, mod = torch.from_numpy(x).cuda(), torch.from_numpy(mod).cuda()
    t = torch.randn((M, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7))

    def loss():
        return float(((s.forward(x, mod, group) - t).double() ** 2).sum() / 2)
    z = s.forward(x, mod, group)
    dx, dmod = s.backward(z - t)
    grads = dict({k: v.clone() for k, v in s.grads.items()}, x=dx, mod=dmod)
    for k, v in dict(s.p, x=x, mod=mod).items():
        d = grads[k]
        slope, h = float((d.double() ** 2).sum()), 0.1 * float(v.norm() / d.norm())
        keep = v.clone()
        ends = []
        for sign in (1, -1):
            v.copy_(keep + sign * h * d)
            s.pack()
            ends.append(loss())
        v.copy_(keep)
        s.pack()
        assert abs((ends[0] - ends[1]) / (2 * h) - slope) < 0.15 * slope, k


def test_stack_refuses_what_does_not_fit():
    torch = torch_cuda()
    from paper_2503_12450_gb300.lazymar import LazymarError
    s = _stack(_blocks(2, 128, 256, 8))
    x, dz, mod = (torch.from_numpy(a).cuda() for a in _inputs(2, 20, 128, 4, 9))
    with pytest.raises(LazymarError, match="forward"):
        s.backward(dz)
    for bad in (mod[:4], mod[:, :-1], mod[0]):
        with pytest.raises(LazymarError, match="mod"):
            s.forward(x, bad, 4)
    with pytest.raises(LazymarError, match="x:"):
        s.forward(x.bfloat16(), mod, 4)
    s.forward(x, mod, 4)
    with pytest.raises(LazymarError, match="dz"):
        s.backward(dz[:19])
    none = torch.empty((0, 128), device="cuda")
    assert s.forward(none, torch.empty((0, 768), device="cuda"), 4, train=False).shape == (0, 128)
    dx, dmod = s.backward(dz)  # serving in between leaves what was kept
    s.forward(x, mod, 4)
    dx2, dmod2 = s.backward(dz)
    assert torch.equal(dx, dx2) and torch.equal(dmod, dmod2)


def _optimizer(s, **kw):
    from paper_2503_12450_gb300.adamw import AdamW
    return AdamW(s.p, s.grads, 1e-3, (0.9, 0.95), 1e-8, weight_decay=0.1, max_norm=1.0, ema_decay=0.99, **kw)


def test_training_steps_eagerly_and_from_a_graph_are_the_same():
    """Forward, backward, norm, update and repacking of a step: five eager ones against two eager and three replayed, bit
    for bit; with the learning rate on the device."""
    torch = torch_cuda()
    D, H, M, group = 128, 512, 300, 50
    x, dz, mod = (torch.from_numpy(a).cuda() for a in _inputs(2, M, D, group, 10))
    ends = []
    for captured in (False, True):
        s = _stack(_blocks(2, D, H, 11))
        opt = _optimizer(s)
        opt.lr = torch.tensor([1e-3], device="cuda")

        def step():
            z = s.forward(x, mod, group)
            s.backward(z * 1e-2)
            opt.step()
            s.pack()
        step()
        step()
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
            torch.cuda.current_stream().wait_stream(side)
        for i in range(3):
            opt.lr.fill_(1e-3 * (i + 1))
            graph.replay() if captured else step()
        norm, factor, steps, skipped = opt.read()
        assert (steps, skipped) == (5, 0) and abs(factor - min(1.0, 1.0 / norm)) < 1e-6
        ends.append([t.clone() for d in (s.p, opt.m, opt.v, opt.ema) for t in d.values()])
    assert all(torch.equal(a, b) for a, b in zip(*ends))


def test_optimizer_state_and_skipped_steps():
    torch = torch_cuda()
    from paper_2503_12450_gb300.adamw import AdamW
    from paper_2503_12450_gb300.lazymar import LazymarError
    g = torch.Generator(device="cuda").manual_seed(12)
    p = {k: torch.randn(s, device="cuda", generator=g) for k, s in (("w", (33, 65)), ("b", (65,)))}
    copies = {"w": torch.zeros((33, 65), dtype=torch.bfloat16, device="cuda")}
    grads = {k: torch.randn(v.shape, device="cuda", generator=g) for k, v in p.items()}
    ref = {k: v.clone().requires_grad_() for k, v in p.items()}
    opt = AdamW(p, grads, 1e-2, weight_decay=0.1, copies=copies)
    want = torch.optim.AdamW([dict(params=[ref["w"]], weight_decay=0.1), dict(params=[ref["b"]], weight_decay=0.0)], lr=1e-2)
    for i in range(4):
        for k, v in grads.items():
            v.copy_(torch.randn(v.shape, device="cuda", generator=g))
            ref[k].grad = v.clone()
        want.step()
        opt.step()
        for k in p:  # each step's rounding: a few units in the last place of weights and step
            assert float((p[k].detach() - ref[k].detach()).abs().max()) < 4 * 2.0 ** -22 * (i + 1)
        assert torch.equal(copies["w"], p["w"].bfloat16())
    saved, weights = opt.state_dict(), {k: v.clone() for k, v in p.items()}
    opt.step()
    after = {k: v.clone() for k, v in p.items()}
    for k, v in p.items():
        v.copy_(weights[k])
    opt.load_state_dict(saved)
    opt.step()
    assert all(torch.equal(p[k], after[k]) for k in p)
    grads["b"][3] = float("inf")
    opt.step()
    assert all(torch.equal(p[k], after[k]) for k in p) and opt.read()[2:] == (5, 1)
    opt.clip()
    assert not grads["b"].any() and not grads["w"].any()
    grads["w"].fill_(2.0)
    opt.max_norm = 1.0
    opt.clip(scale=0.5)
    assert abs(float(grads["w"].norm()) - 1.0) < 1e-5
    with pytest.raises(LazymarError, match="names"):
        AdamW(p, {"w": grads["w"]}, 1e-3)
    with pytest.raises(LazymarError, match="averaged"):
        AdamW(p, grads, 1e-3, ema_decay=0.9).load_state_dict(saved)
    assert math.isinf(AdamW(p, grads, 1e-3).max_norm)
