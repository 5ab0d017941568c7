"""Parity of the residual join and its gradient with the fp64 oracle (oracle/training.py),
through the C ABI, at the sizes, groups, strides, types and values where they can go wrong."""
import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import lazymar as lm
from _gpu import torch_cuda
from test_gpu_train import U, Held, close, close8, dev, held, out, rng, rounded, sync, vec

pytestmark = pytest.mark.gpu

EPS = 1e-6
NORM = dict(none=lm.LAZYMAR_NORM_NONE, layer=lm.LAZYMAR_NORM_LAYER, rms=lm.LAZYMAR_NORM_RMS)


# --------------------------------------------------------------------------
# Bounds. U is half an ulp of fp32; a sum over a row is a tree of lanes, warps and at most
# 32 adds in a row, 48 U with its terms' own rounding. Every bound is per element.
# --------------------------------------------------------------------------
def _norm_bound(v, err, kind, n, mean, rstd):
    """Of norm(v) where v is known to within err: the deviations from the mean, and rstd, which the squares' sum and the
    deviations' errors move."""
    if kind == "none":
        return err, 0 * mean, 0 * rstd
    off = (48 * U * np.abs(v).mean(1) + err.mean(1)) if kind == "layer" else 0 * mean
    d = v - (mean[:, None] if kind == "layer" else 0.0)
    ed = err + off[:, None] + 2 * U * np.abs(d)
    rel = 64 * U + rstd ** 2 * (np.abs(d) * ed + ed ** 2).mean(1)
    return ed * rstd[:, None] + np.abs(n) * (rel[:, None] + 4 * U), off, rel * rstd


def join_bounds(a, o, post, pre, group, res):
    """Bounds of z, h and the statistics, from the oracle's values."""
    x = a["x"]
    r = T.mod_row(x.shape[0], group)
    b = {}
    one = lambda k, d: d if a.get(k) is None else np.asarray(a[k])  # noqa: E731
    zb = 2 * U * np.abs(res * x)
    if a.get("y") is not None:
        u = T.norm(a["y"], post, EPS)[0]
        eu, b["y_mean"], b["y_rstd"] = _norm_bound(a["y"], 0 * u, post, u, o["y_mean"], o["y_rstd"])
        g, s = one("post_g", 1.0), one("post_b", 0.0)
        ev = eu * np.abs(g) + 2 * U * (np.abs(u * g) + np.abs(s))
        gate = one("gate", np.ones((int(r[-1]) + 1, 1)))[r]
        zb = zb + np.abs(gate) * ev + 3 * U * np.abs(gate) * (np.abs(u * g) + np.abs(s)) + U * np.abs(o["z"])
    b["z"] = zb
    if pre != "none":
        n = T.norm(o["z"], pre, EPS)[0]
        en, b["z_mean"], b["z_rstd"] = _norm_bound(o["z"], zb, pre, n, o["z_mean"], o["z_rstd"])
        g, s = one("pre_g", 1.0), one("pre_b", 0.0)
        t = np.abs(n * g) + np.abs(s)
        more = 1 + np.abs(one("scale", np.zeros((int(r[-1]) + 1, 1)))[r])
        b["h"] = (en * np.abs(g) + 2 * U * t) * more + 4 * U * (t * more + np.abs(one("shift", np.zeros((int(r[-1]) + 1, 1)))[r]))
    return {k: v + 1e-30 for k, v in b.items()}


def make(M, D, group, x="fp32", y="fp32", mod="fp32", pad=0, offset=0, seed=1, params=True, gate=True, scale=True, eight=False):
    """Device tensors and the values that they hold."""
    r = rng(M, D, group, seed)
    G = -(-M // group) if group else 1
    big = np.exp(r.standard_normal((M, 1)))
    t, v = {}, {}
    t["x"], v["x"] = dev(r.standard_normal((M, D)) * big + 0.3, x, pad, offset)
    if eight:
        h, v["y"] = held(r.standard_normal((M, D)) * big)
        t["y"] = lm.lazymar_rows(h.q[:, :], h.scale)
    elif y:
        t["y"], v["y"] = dev(0.5 * r.standard_normal((M, D)) * big - 0.2, y, pad, offset)
    names = (["gate"] if gate and (y or eight) else []) + (["scale", "shift"] if scale else [])
    if names:  # side by side, as a linear layer gives them
        wide = 0.4 * r.standard_normal((G, D * len(names)))
        buf, val = dev(wide, mod, pad, offset)
        for i, k in enumerate(names):
            t[k], v[k] = buf[:, i * D:(i + 1) * D], val[:, i * D:(i + 1) * D]
    if params:
        for k in (["post_g", "post_b"] if (y or eight) else []) + ["pre_g", "pre_b"]:
            w = (1.0 if k[-1] == "g" else 0.0) + 0.1 * r.standard_normal(D).astype(np.float32)
            t[k], v[k] = vec(w), np.asarray(w, np.float32).astype(float)
    return t, v


def stats(M):
    return {k: vec(np.full(M, np.nan)) for k in ("y_mean", "y_rstd", "z_mean", "z_rstd")}


SHAPES = [(1, 1, 0), (1, 768, 1), (5, 777, 2), (3, 1024, 1), (300, 1280, 7), (640, 256, 320), (111, 130, 0), (97, 2000, 10),
          (9, 4097, 4), (10, 8192, 3), (2, 8192, 0), (70, 512, 1), (130, 1024, 32), (7, 300, 100), (33, 4096, 5), (19, 6001, 0)]


@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms"), ("layer", "layer")])
@pytest.mark.parametrize("M,D,group", SHAPES)
def test_join(M, D, group, post, pre):
    t, v = make(M, D, group)
    st = stats(M)
    z, h, h8, z8, y8 = out(M, D), out(M, D), Held(M, D), Held(M, D, lds=M + 5), Held(M, D, more=16)
    skip = ("y_mean", "y_rstd") if post == "none" else ()
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, post=NORM[post], pre=NORM[pre], res=0.75, eps=EPS, z=z, h=h,
                                         h8=lm.lazymar_rows(h8.q, h8.scale), z8=lm.lazymar_rows(z8.q, z8.scale),
                                         y8=lm.lazymar_rows(y8.q, y8.scale), **t,
                                         **{k: s for k, s in st.items() if k not in skip}))
    sync()
    o = T.join(post=post, pre=pre, group=group, res=0.75, eps=EPS, **v)
    b = join_bounds(v, o, post, pre, group, 0.75)
    close(z, o["z"], b["z"])
    close(h, o["h"], b["h"])
    close8(h8, o["h"], b["h"])
    close8(z8, o["z"], b["z"])
    q, s = T.pack(v["y"])
    assert (y8.get()[1] == s).all() and (y8.get()[0] == q).all()
    for k in st:
        if k not in skip:
            close(st[k], o[k], b[k] + 1e-30)


@pytest.mark.parametrize("x,y,z,h,mod,pad,offset", [
    ("bf16", "bf16", "bf16", "bf16", "bf16", 0, 0), ("fp32", "bf16", "fp32", "bf16", "bf16", 8, 0),
    ("fp32", "bf16", "bf16", "fp32", "fp32", 0, 0), ("bf16", "fp32", "fp32", "bf16", "bf16", 3, 1),
    ("fp32", "e4m3", "fp32", "bf16", "bf16", 0, 0), ("bf16", "e4m3", "bf16", "fp32", "fp32", 1, 5)])
@pytest.mark.parametrize("M,D,group", [(37, 768, 5), (6, 1280, 1), (21, 333, 0), (4, 5000, 2), (64, 1024, 16)])
def test_join_types_and_strides(M, D, group, x, y, z, h, mod, pad, offset):
    t, v = make(M, D, group, x, y, mod, pad, offset, seed=2, eight=y == "e4m3")
    zt, ht = out(M, D, z, pad, offset), out(M, D, h, pad, offset)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, post=NORM["rms"], pre=NORM["layer"], eps=EPS, z=zt, h=ht, **t))
    sync()
    o = T.join(post="rms", pre="layer", group=group, eps=EPS, **v)
    b = join_bounds(v, o, "rms", "layer", group, 1.0)
    close(zt, o["z"], rounded(b["z"], o["z"], z))
    close(ht, o["h"], rounded(b["h"], o["h"], h))  # from z before its own rounding


@pytest.mark.parametrize("x,y,z,h,mod,pad,offset", [
    ("fp32", "bf16", "fp32", "bf16", "bf16", 0, 0), ("bf16", "bf16", "bf16", "bf16", "fp32", 8, 0),
    ("fp32", "e4m3", "bf16", "fp32", "bf16", 0, 0), ("bf16", "bf16", "bf16", "bf16", "bf16", 1, 3),
    ("fp32", "fp32", "fp32", "fp32", "fp32", 3, 1), ("bf16", "e4m3", "fp32", "bf16", "fp32", 5, 0)])
@pytest.mark.parametrize("M,D,group", [(1300, 1024, 320), (2000, 256, 0), (1999, 130, 1), (2500, 512, 2), (1500, 1280, 11),
                                       (700, 4096, 100), (900, 2048, 1), (5000, 104, 3), (1200, 777, 7), (400, 5001, 9),
                                       (1000, 1281, 1)])
def test_join_many_rows(M, D, group, x, y, z, h, mod, pad, offset):
    """More rows than teams: several rows in a row, groups inside a team's range and across them, rows on and off
    the boundary, among them the tensor's first and last, whose neighbours are NaN here."""
    t, v = make(M, D, group, x, y, mod, pad, offset, seed=30, eight=y == "e4m3")
    zt, ht, h8, st = out(M, D, z, pad, offset), out(M, D, h, pad, offset), Held(M, D, more=16), stats(M)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, post=NORM["layer"], pre=NORM["rms"], res=0.75, eps=EPS, z=zt, h=ht,
                                         h8=lm.lazymar_rows(h8.q, h8.scale), **t, **st))
    sync()
    o = T.join(post="layer", pre="rms", group=group, res=0.75, eps=EPS, **v)
    b = join_bounds(v, o, "layer", "rms", group, 0.75)
    close(zt, o["z"], rounded(b["z"], o["z"], z))
    close(ht, o["h"], rounded(b["h"], o["h"], h))
    close8(h8, o["h"], b["h"])
    for k in st:
        close(st[k], o[k], b[k])
    if pad:  # what lies between the rows stays
        for a in (zt, ht):
            assert torch_cuda().isnan(a.as_strided((M - 1, pad), (D + pad, 1), a.storage_offset() + D)).all()


@pytest.mark.parametrize("pad,offset", [(0, 0), (0, 1), (1, 3)])
@pytest.mark.parametrize("D,group", [(1, 0), (1, 400), (2, 1), (3, 7), (5, 2), (7, 300)])
def test_join_and_gradient_of_narrow_rows(D, group, pad, offset):
    """Several rows lie between two 16-byte boundaries."""
    M = 1000
    t, v = make(M, D, group, "bf16", "bf16", "bf16", pad, offset)
    st = stats(M)
    z, h = out(M, D, "bf16", pad, offset), out(M, D, "bf16", pad, offset)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, post=NORM["rms"], pre=NORM["rms"], res=0.75, eps=EPS, z=z, h=h, **t, **st))
    sync()
    o = T.join(post="rms", pre="rms", group=group, res=0.75, eps=EPS, **v)
    b = join_bounds(v, o, "rms", "rms", group, 0.75)
    close(z, o["z"], rounded(b["z"], o["z"], "bf16"))
    close(h, o["h"], rounded(b["h"], o["h"], "bf16"))
    Grad(M, D, group, "rms", "rms", "bf16", "bf16", "bf16", "bf16", "bf16", "bf16", "bf16", pad, offset, seed=21).check()


@pytest.mark.parametrize("fields", [("gate",), ("scale",), ("post_g",), ("post_b",), ("pre_g",), ("pre_b",), ("shift",), ()])
def test_join_with_some_of_its_parts(fields):
    M, D, group = 11, 777, 3
    t, v = make(M, D, group, seed=3)
    t, v = ({k: a for k, a in d.items() if k in ("x", "y") + fields} for d in (t, v))
    z, h = out(M, D), out(M, D)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, pre=NORM["rms"], eps=EPS, z=z, h=h, **t))
    sync()
    o = T.join(pre="rms", group=group, eps=EPS, **v)
    b = join_bounds(v, o, "none", "rms", group, 1.0)
    close(z, o["z"], b["z"])
    close(h, o["h"], b["h"])


@pytest.mark.parametrize("D", [1024, 777])
def test_join_without_a_branch_or_without_a_norm(D):
    M = 9
    t, v = make(M, D, 2, y="", seed=4)
    z, h = out(M, D), out(M, D)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=2, pre=NORM["layer"], res=0.5, eps=EPS, z=z, h=h, **t))
    o = T.join(y=None, pre="layer", group=2, res=0.5, eps=EPS, **v)
    b = join_bounds(v, o, "none", "layer", 2, 0.5)
    sync()
    close(z, o["z"], b["z"])
    close(h, o["h"], b["h"])
    t, v = make(M, D, 2, scale=False, params=False, seed=5)
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=2, post=NORM["layer"], eps=EPS, z=z, **t))
    o = T.join(post="layer", group=2, eps=EPS, **v)
    sync()
    close(z, o["z"], join_bounds(v, o, "layer", "none", 2, 1.0)["z"])


@pytest.mark.parametrize("M", [70, 2000])
@pytest.mark.parametrize("D,pad,offset", [(1024, 0, 0), (777, 2, 1), (4099, 0, 0)])
def test_join_in_place(D, pad, offset, M):
    """z over x, h over y, with their types and strides; the rows around them stay."""
    torch = torch_cuda()
    t, v = make(M, D, 7, "fp32", "bf16", pad=pad, offset=offset, seed=6)
    z, h = out(M, D), out(M, D, "bf16")
    kw = dict(group=7, post=NORM["layer"], pre=NORM["rms"], eps=EPS)
    lm.lazymar_join(lm.lazymar_join_args(M, D, z=z, h=h, **t, **kw))
    lm.lazymar_join(lm.lazymar_join_args(M, D, z=t["x"], h=t["y"], **t, **kw))
    sync()
    assert torch.equal(t["x"], z) and torch.equal(t["y"], h)
    if pad:
        assert torch.isnan(t["x"].as_strided((M, pad), (D + pad, 1), t["x"].storage_offset() + D)).all()


@pytest.mark.parametrize("M", [40, 900])
def test_join_8_bit_outputs_in_place(M):
    """h8 over an 8-bit y, and dy8 over it in the gradient."""
    torch = torch_cuda()
    D = 520
    t, v = make(M, D, 9, eight=True, seed=31)
    h8 = Held(M, D)
    kw = dict(group=9, pre=NORM["layer"], eps=EPS)
    lm.lazymar_join(lm.lazymar_join_args(M, D, h8=lm.lazymar_rows(h8.q, h8.scale), **t, **kw))
    y = t["y"].keep[0]
    lm.lazymar_join(lm.lazymar_join_args(M, D, h8=t["y"], **t, **kw))
    sync()
    assert torch.equal(y[:, :D], h8.q[:, :D]) and torch.equal(t["y"].keep[1], h8.scale)
    g = Grad(M, D, 9, "rms", "layer", y="e4m3", seed=32).check()
    lm.lazymar_join_grad(g.args(dy8=g.t["y"]))
    sync()
    assert torch.equal(g.t["y"].keep[0][:, :D], g.dy8.q[:, :D]) and torch.equal(g.t["y"].keep[1], g.dy8.scale)


@pytest.mark.parametrize("M,D", [(12, 1000), (1200, 1000), (1200, 999)])
@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
def test_join_rows_that_are_not_finite_stay_alone(post, pre, M, D):
    torch = torch_cuda()
    t, v = make(M, D, 0, seed=7)
    z, h, h8 = out(M, D), out(M, D), Held(M, D)
    kw = dict(post=NORM[post], pre=NORM[pre], eps=EPS, z=z, h=h, h8=lm.lazymar_rows(h8.q, h8.scale))
    lm.lazymar_join(lm.lazymar_join_args(M, D, **t, **kw))
    sync()
    want_z, want_h, want_q = z.clone(), h.clone(), h8.q.clone()
    t["x"][2, 5], t["y"][4, D - 1], t["x"][6, 0], t["y"][8] = float("nan"), float("inf"), -float("inf"), 0.0
    lm.lazymar_join(lm.lazymar_join_args(M, D, **t, **kw))
    sync()
    for i in (2, 4, 6):
        assert torch.isnan(h[i]).all() or not torch.isfinite(h[i]).all()
    assert torch.isnan(h[2]).all() and torch.isfinite(h[8]).all()
    same = [i for i in range(M) if i not in (2, 4, 6, 8)]
    assert torch.equal(z[same], want_z[same]) and torch.equal(h[same], want_h[same]) and torch.equal(h8.q[same], want_q[same])


def test_join_constant_rows_and_large_offsets():
    """Rows that do not vary (1 / deviation is 1 / sqrt(eps)), and rows whose mean is large against their deviations."""
    M, D = 6, 1536
    r = rng(8)
    x = np.zeros((M, D))
    x[1] = 3.0
    x[2] = 1000.0 + r.standard_normal(D)
    x[3] = -1e5 + 10 * r.standard_normal(D)
    x[4] = 1e-20 * r.standard_normal(D)
    x[5] = 1e15 * r.standard_normal(D)
    t, v = dev(x)
    z, h, st = out(M, D), out(M, D), stats(M)
    for pre in ("layer", "rms"):
        lm.lazymar_join(lm.lazymar_join_args(M, D, t, pre=NORM[pre], eps=EPS, z=z, h=h, z_mean=st["z_mean"], z_rstd=st["z_rstd"]))
        sync()
        o = T.join(v, None, pre=pre, eps=EPS)
        b = join_bounds(dict(x=v), o, "none", pre, 0, 1.0)
        close(z, o["z"], b["z"])
        close(h, o["h"], b["h"])
        close(st["z_mean"], o["z_mean"], b["z_mean"])
        close(st["z_rstd"], o["z_rstd"], b["z_rstd"])


# --------------------------------------------------------------------------
# Gradient
# --------------------------------------------------------------------------
def grad_bounds(v, o, post, pre, group, res):
    """Bounds of the gradients: products of a few rounded factors, sums over a row as above, sums over rows in chains of
    at most 128 (a team's rows, 32 slices of teams, the slices)."""
    some = v["dh"] if v.get("dh") is not None else v["dz"]
    M, D = some.shape
    r = T.mod_row(M, group)
    G = int(r[-1]) + 1
    one = lambda k, d: d if v.get(k) is None else np.asarray(v[k])  # noqa: E731
    b = {}

    def by_group(t):
        s = np.zeros((G, D))
        np.add.at(s, r, t)
        return s
    S = 128 * U
    Z, eZ = one("dz", np.zeros((M, D))), 0.0
    if pre != "none":
        n = T._normalised(v["z"], pre, v.get("z_mean"), v["z_rstd"])
        en = 4 * U * np.abs(n)
        more = 1 + one("scale", np.zeros((G, 1)))[r]
        g, s = one("pre_g", 1.0), one("pre_b", 0.0)
        dh = np.abs(v["dh"])
        b["dshift"] = S * by_group(dh)
        nb = by_group(dh * np.abs(n))
        b["dscale"] = np.abs(g) * (S + 8 * U) * nb + np.abs(s) * (S + 8 * U) * by_group(dh) + 0 * nb
        b["dpre_g"], b["dpre_b"] = (S + 8 * U) * (dh * np.abs(more) * np.abs(n)).sum(0), (S + 4 * U) * (dh * np.abs(more)).sum(0)
        d = v["dh"] * more * g
        ed = 4 * U * np.abs(d)
        m1 = np.abs(d).mean(1, keepdims=True) if pre == "layer" else 0.0
        m2 = np.abs(d * n).mean(1, keepdims=True)
        inner = np.abs(d) + m1 + np.abs(n) * m2
        eZ = v["z_rstd"][:, None] * (ed + 52 * U * m1 + np.abs(n) * 60 * U * m2 + en * m2 + 6 * U * inner)
        Z = Z + T._norm_grad(d, n, v["z_rstd"], pre)
        eZ = eZ + 2 * U * (np.abs(Z) + np.abs(one("dz", 0.0)))
    b["dx"] = np.abs(res) * eZ + U * np.abs(res * Z)
    gate = one("gate", np.ones((G, 1)))[r]
    V = Z * gate
    eV = eZ * np.abs(gate) + U * np.abs(V)
    b["dpost_b"] = S * np.abs(V).sum(0) + np.sum(eV + 0 * V, 0)
    g, s = one("post_g", 1.0), one("post_b", 0.0)
    d = V * g
    ed = eV * np.abs(g) + 2 * U * np.abs(d)
    b["dy"] = ed
    if v.get("y") is not None:
        u = T._normalised(v["y"], post, v.get("y_mean"), v.get("y_rstd"))
        eu = 4 * U * np.abs(u) * (post != "none")
        t = np.abs(u * g) + np.abs(s)
        b["dgate"] = by_group((S + 8 * U) * np.abs(Z) * t + eZ * t + np.abs(Z) * eu * np.abs(g))
        b["dpost_g"] = ((S + 4 * U) * np.abs(V * u) + eV * np.abs(u) + np.abs(V) * eu).sum(0)
        if post != "none":
            m1 = np.abs(d).mean(1, keepdims=True) if post == "layer" else 0.0
            e1 = ed.mean(1, keepdims=True) if post == "layer" else 0.0
            m2 = np.abs(d * u).mean(1, keepdims=True)
            inner = np.abs(d) + m1 + np.abs(u) * m2
            b["dy"] = v["y_rstd"][:, None] * (ed + 52 * U * m1 + e1 + np.abs(u) * (60 * U * m2 + (ed * np.abs(u)).mean(1, keepdims=True))
                                              + eu * m2 + 6 * U * inner)
    return {k: w + 1e-30 for k, w in b.items()}


class Grad:
    """One call of the gradient: inputs, outputs filled with NaN, and the comparison."""

    def __init__(self, M, D, group, post, pre, dh="fp32", dz="fp32", z="fp32", y="fp32", dx="fp32", dy="fp32", mod="fp32",
                 pad=0, offset=0, seed=1, res=0.75, params=True, gate=True, scale=True, more=0):
        r = rng(M, D, group, seed)
        self.M, self.D, self.group, self.post, self.pre, self.res = M, D, group, post, pre, res
        self.types = dict(dx=dx, dy=dy, dgate=mod, dscale=mod, dshift=mod)
        G = -(-M // group) if group else 1
        t, v = make(M, D, group, "fp32", "fp32", mod, pad, offset, seed, params, gate, scale and pre != "none")
        for k in ("x", "y", "shift"):
            t.pop(k, None), v.pop(k, None)
        if pre == "none":
            for k in ("pre_g", "pre_b"):
                t.pop(k, None), v.pop(k, None)
        big = np.exp(r.standard_normal((M, 1)))
        for k, dtype, on in (("dh", dh, pre != "none"), ("dz", dz, bool(dz)), ("z", z, pre != "none"), ("y", y, bool(y))):
            if not on:
                continue
            a = r.standard_normal((M, D)) * (big if k in "zy" else 1e-3) + (0.2 if k in "zy" else 0.0)
            if dtype == "e4m3":
                h, v[k] = held(a)
                t[k] = lm.lazymar_rows(h.q, h.scale)
            else:
                t[k], v[k] = dev(a, dtype, pad, offset)
        for k, kind in (("y", post), ("z", pre)):
            if kind != "none":
                _, mean, rstd = T.norm(v[k], kind, EPS)
                for s, w in ((k + "_mean", mean), (k + "_rstd", rstd)):
                    if s.endswith("rstd") or kind == "layer":
                        t[s] = vec(w)
                        v[s] = np.asarray(w, np.float32).astype(float)
        self.t, self.v = t, v
        o = dict(dx=out(M, D, dx, pad, offset), dy=out(M, D, dy, pad, offset))
        self.dy8 = Held(M, D, more=more)
        wide = out(G, 3 * D, mod, pad, offset)
        if pre != "none":
            o.update(dshift=wide[:, :D], dscale=wide[:, D:2 * D])
            o.update({k: vec(np.full(D, np.nan)) for k in ("dpre_g", "dpre_b")})
        if y:
            o.update(dgate=wide[:, 2 * D:], dpost_g=vec(np.full(D, np.nan)))
        o["dpost_b"] = vec(np.full(D, np.nan))
        self.o = o
        n = lm.lazymar_join_grad_workspace(M, D, group)
        self.ws = torch_cuda().full((n,), 0xFF, dtype=torch_cuda().uint8, device="cuda")

    def args(self, **kw):
        f = dict(group=self.group, post=NORM[self.post], pre=NORM[self.pre], res=self.res, workspace=self.ws,
                 dy8=lm.lazymar_rows(self.dy8.q, self.dy8.scale), **self.t, **self.o)
        return lm.lazymar_join_grad_args(self.M, self.D, **dict(f, **kw))

    def want(self):
        w = T.join_grad(self.v.get("dh"), self.v.get("dz"), self.v.get("z"), self.v.get("y"), post=self.post, pre=self.pre,
                        group=self.group, res=self.res,
                        **{k: self.v.get(k) for k in ("gate", "scale", "post_g", "post_b", "pre_g", "pre_b", "y_mean", "y_rstd",
                                                      "z_mean", "z_rstd")})
        return w, grad_bounds(self.v, w, self.post, self.pre, self.group, self.res)

    def check(self):
        lm.lazymar_join_grad(self.args())
        sync()
        w, b = self.want()
        for k, t in self.o.items():
            close(t, w[k], rounded(np.broadcast_to(b[k], w[k].shape), w[k], self.types.get(k)))
        close8(self.dy8, w["dy"], np.broadcast_to(b["dy"], w["dy"].shape))
        return self


@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms"), ("layer", "none")])
@pytest.mark.parametrize("M,D,group", SHAPES)
def test_join_grad(M, D, group, post, pre):
    Grad(M, D, group, post, pre).check()


@pytest.mark.parametrize("M,D,group", [(1300, 1024, 320), (2000, 256, 0), (1999, 130, 1), (2500, 512, 2), (1500, 1280, 11),
                                       (700, 4096, 100), (400, 8192, 9), (5000, 100, 3), (4000, 64, 4000), (3000, 257, 2999)])
def test_join_grad_many_rows(M, D, group):
    """More rows than teams: ranges of several rows, groups inside a range, across two and across many."""
    Grad(M, D, group, "layer", "layer", seed=9).check()


@pytest.mark.parametrize("dh,dz,z,y,dx,dy,mod,pad,offset", [
    ("bf16", "fp32", "e4m3", "e4m3", "fp32", "bf16", "bf16", 0, 0), ("bf16", "bf16", "bf16", "bf16", "bf16", "bf16", "bf16", 8, 0),
    ("fp32", "", "e4m3", "bf16", "bf16", "fp32", "fp32", 1, 3), ("bf16", "fp32", "fp32", "e4m3", "fp32", "bf16", "fp32", 0, 1)])
@pytest.mark.parametrize("M,D,group", [(37, 768, 5), (400, 1280, 1), (21, 333, 0), (4, 5000, 2), (700, 1024, 16)])
def test_join_grad_types_and_strides(M, D, group, dh, dz, z, y, dx, dy, mod, pad, offset):
    Grad(M, D, group, "rms", "layer", dh, dz, z, y, dx, dy, mod, pad, offset, seed=10, more=16).check()


@pytest.mark.parametrize("group", [0, 1, 3])
@pytest.mark.parametrize("params,gate,scale", [(False, False, False), (True, False, True), (False, True, True)])
def test_join_grad_with_some_of_its_parts(params, gate, scale, group):
    Grad(50, 777, group, "none", "rms", params=params, gate=gate, scale=scale, seed=11).check()
    Grad(50, 768, group, "layer", "layer", params=params, gate=gate, scale=scale, seed=12).check()


def test_join_grad_of_a_bare_addition_needs_no_branch():
    g = Grad(40, 512, 4, "none", "layer", y="", gate=False, seed=13)
    g.check()
    # and an input that nothing depends on is not read
    g.t["y"] = out(40, 512)
    g.check()


@pytest.mark.parametrize("group", [0, 1, 6])
def test_join_grad_single_outputs(group):
    """Each output alone is what it is among the others."""
    torch = torch_cuda()
    g = Grad(700, 640, group, "rms", "layer", seed=14).check()
    for k, t in g.o.items():
        alone = torch.full_like(t, float("nan"))
        none = {n: None for n in g.o}
        f = dict(group=group, post=NORM["rms"], pre=NORM["layer"], res=g.res, workspace=g.ws, **g.t)
        lm.lazymar_join_grad(lm.lazymar_join_grad_args(700, 640, **dict(f, **dict(none, **{k: alone}))))
        sync()
        assert torch.equal(alone, t), k
    q, s = g.dy8.q.clone(), g.dy8.scale.clone()
    g.dy8.q.fill_(0xAB), g.dy8.scale.fill_(0xAB)
    lm.lazymar_join_grad(g.args(**{n: None for n in g.o}, workspace=None, workspace_bytes=0))
    sync()
    assert torch.equal(g.dy8.q, q) and torch.equal(g.dy8.scale, s)


@pytest.mark.parametrize("mod", ["fp32", "bf16"])
@pytest.mark.parametrize("M,group", [(700, 0), (300, 1), (700, 9), (20, 20)])
def test_join_grad_accumulates(M, group, mod):
    """A second pass with accumulate adds: twice the gradient, exactly in fp32 (doubling), one rounding in bf16."""
    torch = torch_cuda()
    g = Grad(M, 1000, group, "rms", "layer", mod=mod, seed=15).check()
    first = {k: t.clone() for k, t in g.o.items()}
    lm.lazymar_join_grad(g.args(accumulate=True))
    sync()
    for k, t in g.o.items():
        if k in ("dx", "dy"):
            assert torch.equal(t, first[k])
        elif g.types.get(k) == "bf16":
            assert float((t.float() - 2 * first[k].float()).abs().max()) <= 2.0 ** -7 * float(first[k].float().abs().max())
        else:
            assert torch.equal(t, first[k] + first[k]), k


@pytest.mark.parametrize("D,pad,offset", [(1024, 0, 0), (777, 3, 1), (1280, 0, 0)])
def test_join_grad_in_place(D, pad, offset):
    torch = torch_cuda()
    M = 900
    for over in (("dz", "y"), ("dh", "z"), ("z", "dh"), ("y", "dz")):
        g = Grad(M, D, 30, "layer", "layer", pad=pad, offset=offset, seed=16).check()
        want = {k: t.clone() for k, t in g.o.items()}
        lm.lazymar_join_grad(g.args(dx=g.t[over[0]], dy=g.t[over[1]]))
        sync()
        assert torch.equal(g.t[over[0]], want["dx"]) and torch.equal(g.t[over[1]], want["dy"]), over
        for k in want:
            if k not in ("dx", "dy"):
                assert torch.equal(g.o[k], want[k]), (over, k)


def test_join_grad_is_the_same_from_call_to_call_and_leaves_the_rest():
    torch = torch_cuda()
    g = Grad(3000, 1280, 320, "none", "layer", "bf16", "fp32", "e4m3", "e4m3", "fp32", "bf16", "bf16", seed=17).check()
    want = {k: t.clone() for k, t in g.o.items()}
    for _ in range(3):
        for t in g.o.values():
            t.fill_(float("nan"))
        g.ws.fill_(0x7F)
        lm.lazymar_join_grad(g.args())
        sync()
        for k, t in g.o.items():
            assert torch.equal(t, want[k]), k
    # a workspace of just the size, between guards
    n = g.ws.numel()
    room = torch.full((n + 512,), 0xC3, dtype=torch.uint8, device="cuda")
    lm.lazymar_join_grad(g.args(workspace=room[256:256 + n]))
    sync()
    assert (room[:256] == 0xC3).all() and (room[256 + n:] == 0xC3).all()
    with pytest.raises(lm.LazymarError, match="workspace_bytes"):
        lm.lazymar_join_grad(g.args(workspace_bytes=n - 1))


@pytest.mark.parametrize("group", [0, 4])
def test_join_grad_without_rows(group):
    torch = torch_cuda()
    D = 300
    o = {k: torch.ones(D, device="cuda") for k in ("dpost_g", "dpost_b", "dpre_g", "dpre_b")}
    m = torch.ones((1 if group == 0 else 0, 3 * D), device="cuda")
    mods = {k: lm.lazymar_rows(m[:, i * D:(i + 1) * D], ld=3 * D) for i, k in enumerate(("dgate", "dscale", "dshift"))} if group == 0 else {}
    for accumulate in (True, False):
        lm.lazymar_join_grad(lm.lazymar_join_grad_args(0, D, group=group, pre=NORM["layer"], accumulate=accumulate, **o, **mods))
        sync()
        for t in list(o.values()) + ([m] if group == 0 else []):
            assert (t == (1.0 if accumulate else 0.0)).all()


def test_join_and_gradient_against_differences():
    """The directional derivative along the gradient by differences of the fp32 kernel's own outputs (summed in fp64). Rows
    are of sizes e^-2.5 to e^2.5 and the gradient of a norm goes with 1 / size, so a step of s of y's norm moves the smallest
    row by up to e^5 s of its own: the third-order term, (e^5 s)^2 = 2 at s = 1e-2, is 2e-4 at 1e-4. The losses' rounding,
    U 1e-3 sqrt(32768) = 1e-8, is 1e-6 of their difference there."""
    torch = torch_cuda()
    M, D, group = 64, 512, 16
    t, v = make(M, D, group, seed=18)
    st = stats(M)
    z, h = out(M, D), out(M, D)
    r = rng(19)
    dh, dz = dev(1e-3 * r.standard_normal((M, D)))[0], dev(1e-3 * r.standard_normal((M, D)))[0]
    kw = dict(group=group, post=NORM["layer"], pre=NORM["rms"], res=0.9)
    call = lm.lazymar_join_args(M, D, eps=EPS, z=z, h=h, **t, **st, **kw)

    def loss():
        lm.lazymar_join(call)
        return float((z.double() * dz.double()).sum() + (h.double() * dh.double()).sum())
    loss()
    G = M // group
    o = dict(dx=out(M, D), dy=out(M, D), dgate=out(G, D), dscale=out(G, D), dshift=out(G, D),
             **{k: vec(np.zeros(D)) for k in ("dpost_g", "dpost_b", "dpre_g", "dpre_b")})
    ws = torch.empty(lm.lazymar_join_grad_workspace(M, D, group), dtype=torch.uint8, device="cuda")
    zz = z.clone()
    lm.lazymar_join_grad(lm.lazymar_join_grad_args(
        M, D, dh=dh, dz=dz, z=zz, y=t["y"], gate=t["gate"], scale=t["scale"], workspace=ws,
        **{k: t[k] for k in ("post_g", "post_b", "pre_g", "pre_b")}, **st, **kw, **o))
    sync()
    for k in ("x", "y", "gate", "scale", "shift", "post_g", "post_b", "pre_g", "pre_b"):
        d = o["d" + k].double()
        slope = float((d * d).sum())
        step = 1e-4 * float(t[k].double().norm() / d.norm())
        keep = t[k].clone()
        t[k].copy_(keep + step * d)
        up = loss()
        t[k].copy_(keep - step * d)
        down = loss()
        t[k].copy_(keep)
        assert abs((up - down) / (2 * step) - slope) < 1e-2 * slope, k


# --------------------------------------------------------------------------
# Streams, graphs, large addresses
# --------------------------------------------------------------------------
def test_join_on_other_streams_and_in_graphs():
    """A call on a side stream, two graphs with a workspace each replayed in turn, and new values in the same buffers."""
    torch = torch_cuda()
    M, D, group = 500, 1024, 20
    t, v = make(M, D, group, seed=20)
    z, h = out(M, D), out(M, D)
    fwd = lm.lazymar_join_args(M, D, group=group, post=NORM["rms"], pre=NORM["layer"], eps=EPS, z=z, h=h, **t)
    grads = [Grad(M, D, group, "rms", "layer", seed=s) for s in (21, 22)]
    lm.lazymar_join(fwd)
    for g in grads:
        g.check()
    want = [z.clone(), h.clone()] + [t.clone() for g in grads for t in g.o.values()]

    def outputs():
        return [z, h] + [t for g in grads for t in g.o.values()]
    side = torch.cuda.Stream()
    calls = [(lm.lazymar_join, fwd)] + [(lm.lazymar_join_grad, g.args()) for g in grads]
    for t_ in outputs():
        t_.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for f, a in calls:
            f(a)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    graphs = []
    for f, a in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f(a)
        graphs.append(g)
    for _ in range(2):
        for t_ in outputs():
            t_.fill_(float("nan"))
        for g in graphs:
            g.replay()
        sync()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    t["x"].mul_(0.5)
    graphs[0].replay()
    sync()
    o = T.join(post="rms", pre="layer", group=group, eps=EPS, **dict(v, x=0.5 * v["x"]))
    close(z, o["z"], join_bounds(dict(v, x=0.5 * v["x"]), o, "rms", "layer", group, 1.0)["z"])


def test_join_rows_beyond_32_bit_offsets():
    """Rows so far apart that elements lie beyond 2^32 of the first: the last rows are right, and what lies between stays."""
    torch = torch_cuda()
    M, D, ld = 5, 1024, (1 << 30) + 8
    n = (M - 1) * ld + D
    x, y, z = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    r = rng(23)
    xs, ys = r.standard_normal((M, D)), r.standard_normal((M, D))
    rows = [t.as_strided((M, D), (ld, 1)) for t in (x, y, z)]
    rows[0].copy_(torch.from_numpy(xs).cuda())
    rows[1].copy_(torch.from_numpy(ys).cuda())
    vx, vy = (t.double().cpu().numpy() for t in rows[:2])
    h = out(M, D)
    lm.lazymar_join(lm.lazymar_join_args(M, D, rows[0], rows[1], pre=NORM["layer"], eps=EPS, z=rows[2], h=h))
    sync()
    o = T.join(vx, vy, pre="layer", eps=EPS)
    b = join_bounds(dict(x=vx, y=vy), o, "none", "layer", 0, 1.0)
    close(rows[2], o["z"], rounded(b["z"], o["z"], "bf16"))
    close(h, o["h"], b["h"])
    # the gradient, with y's gradient in y's place
    st = vec(o["z_mean"]), vec(o["z_rstd"])
    dh, dx = dev(1e-3 * r.standard_normal((M, D)))[0], out(M, D)
    zv = rows[2].double().cpu().numpy()
    lm.lazymar_join_grad(lm.lazymar_join_grad_args(M, D, pre=NORM["layer"], dh=dh, z=rows[2], z_mean=st[0], z_rstd=st[1], dx=dx,
                                                   dy=rows[1]))
    sync()
    vals = dict(dh=dh.double().cpu().numpy(), z=zv, z_mean=st[0].double().cpu().numpy(), z_rstd=st[1].double().cpu().numpy())
    w = T.join_grad(vals["dh"], None, zv, None, pre="layer", z_mean=vals["z_mean"], z_rstd=vals["z_rstd"])
    gb = grad_bounds(vals, w, "none", "layer", 0, 1.0)
    close(dx, w["dx"], gb["dx"])
    close(rows[1], w["dy"], rounded(gb["dy"], w["dy"], "bf16"))
    del x, y, z, rows
    torch.cuda.empty_cache()
