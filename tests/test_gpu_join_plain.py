"""The residual join's kernels for a modulated block (a branch with gate, scale and shift, no norm behind it, no parameters
and none of their gradients): every element against the fp64 oracle, at all widths of a team, with a modulation for all
rows, for groups of them and for each."""
import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import lazymar as lm
from _gpu import torch_cuda
from test_gpu_join import EPS, NORM, Grad, join_bounds, make, stats
from test_gpu_train import Held, close, close8, out, rounded, sync

pytestmark = pytest.mark.gpu

# Teams of 1, 2, 3, 4, 5, 8 and 16 warps on and off the boundary; groups within a range of rows, across two and across
# many; the last group short.
SHAPES = [(1300, 1024, 320), (2000, 256, 0), (1999, 130, 1), (2500, 512, 2), (1500, 1280, 11), (700, 4096, 100), (900, 2048, 1),
          (5000, 104, 3), (1200, 777, 7), (1000, 1281, 64), (6000, 640, 5), (305, 768, 0), (640, 1536, 320), (3000, 257, 2999)]


@pytest.mark.parametrize("x,y,z,h,mod,pad,offset", [
    ("fp32", "bf16", "fp32", "fp32", "bf16", 0, 0), ("bf16", "fp32", "bf16", "bf16", "fp32", 8, 0),
    ("fp32", "e4m3", "fp32", "bf16", "bf16", 0, 0), ("bf16", "bf16", "bf16", "bf16", "bf16", 3, 1)])
@pytest.mark.parametrize("M,D,group", SHAPES)
def test_plain_join(M, D, group, x, y, z, h, mod, pad, offset):
    """All outputs at once; the modulated norm is of z before its own rounding."""
    t, v = make(M, D, group, x, y, mod, pad, offset, seed=50, params=False, eight=y == "e4m3")
    zt, ht, st = out(M, D, z, pad, offset), out(M, D, h, pad, offset), stats(M)
    h8, z8, y8 = Held(M, D, more=16), Held(M, D, lds=M + 5), Held(M, D)
    pre = "rms" if y == "fp32" else "layer"
    lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, pre=NORM[pre], res=0.75, eps=EPS, z=zt, h=ht,
                                         h8=lm.lazymar_rows(h8.q, h8.scale), z8=lm.lazymar_rows(z8.q, z8.scale),
                                         y8=lm.lazymar_rows(y8.q, y8.scale), z_mean=st["z_mean"], z_rstd=st["z_rstd"], **t))
    sync()
    o = T.join(pre=pre, group=group, res=0.75, eps=EPS, **v)
    b = join_bounds(v, o, "none", pre, group, 0.75)
    close(zt, o["z"], rounded(b["z"], o["z"], z))
    close(ht, o["h"], rounded(b["h"], o["h"], h))
    close8(h8, o["h"], b["h"])
    close8(z8, o["z"], b["z"])
    q, s = T.pack(v["y"])
    assert (y8.get()[1] == s).all() and (y8.get()[0] == q).all()
    for k in ("z_mean", "z_rstd"):
        close(st[k], o[k], b[k])


@pytest.mark.parametrize("D,group", [(1024, 320), (768, 1), (777, 0)])
@pytest.mark.parametrize("names", [("z",), ("h",), ("h8",), ("z8",), ("y8",), ("z_mean",), ("z_rstd",)], ids=lambda n: n[0])
def test_plain_join_single_outputs(names, D, group):
    """Each output alone is what it is among the others (the kernel is the same)."""
    torch = torch_cuda()
    M = 700
    t, _ = make(M, D, group, "fp32", "bf16", "bf16", seed=51, params=False)

    def outputs():
        return dict(z=out(M, D), h=out(M, D, "bf16"), h8=Held(M, D), z8=Held(M, D), y8=Held(M, D), z_mean=stats(M)["z_mean"],
                    z_rstd=stats(M)["z_rstd"])

    def call(o):
        f = {k: lm.lazymar_rows(a.q, a.scale) if isinstance(a, Held) else a for k, a in o.items()}
        lm.lazymar_join(lm.lazymar_join_args(M, D, group=group, pre=NORM["layer"], eps=EPS, **f, **t))
        sync()
    every = outputs()
    call(every)
    alone = {k: a for k, a in outputs().items() if k in names}
    call(alone)
    for k, a in alone.items():
        if isinstance(a, Held):
            assert torch.equal(a.q, every[k].q) and torch.equal(a.scale, every[k].scale)
        else:
            assert torch.equal(a, every[k])


class Plain(Grad):
    """A gradient without the parameters and without their gradients."""

    def __init__(self, M, D, group, **kw):
        super().__init__(M, D, group, "none", kw.pop("pre", "layer"), params=False, **kw)
        for k in ("dpost_g", "dpost_b", "dpre_g", "dpre_b"):
            del self.o[k]
        assert {"dz", "y", "gate", "scale"} <= set(self.t) and {"dgate", "dscale", "dshift"} <= set(self.o)


@pytest.mark.parametrize("dh,dz,z,y,dx,dy,mod,pad,offset", [
    ("bf16", "fp32", "e4m3", "e4m3", "fp32", "bf16", "bf16", 0, 0), ("fp32", "fp32", "fp32", "fp32", "fp32", "fp32", "fp32", 0, 0),
    ("bf16", "bf16", "bf16", "bf16", "bf16", "bf16", "fp32", 8, 0), ("fp32", "bf16", "e4m3", "bf16", "bf16", "fp32", "bf16", 1, 3)])
@pytest.mark.parametrize("M,D,group", SHAPES + [(1, 768, 1), (5, 777, 2), (37, 768, 5), (400, 8192, 9), (300, 5000, 1),
                                                (250, 4104, 0), (2, 1024, 0)])
def test_plain_join_grad(M, D, group, dh, dz, z, y, dx, dy, mod, pad, offset):
    Plain(M, D, group, pre="rms" if dx == "bf16" else "layer", dh=dh, dz=dz, z=z, y=y, dx=dx, dy=dy, mod=mod, pad=pad, offset=offset,
          seed=52, more=16).check()


@pytest.mark.parametrize("M,D,group", [(70000, 64, 200), (40000, 96, 7), (35000, 100, 320), (65000, 64, 0), (20000, 64, 1)])
def test_plain_join_grad_with_several_groups_in_a_range(M, D, group):
    """Ranges of 460 rows that hold groups of 200 whole, ranges of teams with several groups, and groups longer than a
    range, each finished by itself or joined behind the kernel."""
    Plain(M, D, group, dh="bf16", seed=53).check()


@pytest.mark.parametrize("group", [0, 1, 5, 320])
def test_plain_join_grad_single_modulations(group):
    """The modulation's gradients beside dx and dy, not all of them. With the gate's, the kernel and the ranges of rows are
    the same, and so are the bits. Without it nothing depends on y, and the general kernel divides the rows in
    another way: sums that are as near to the exact ones, in other last bits."""
    torch = torch_cuda()
    g = Plain(1500, 1280, group, seed=54).check()
    first = {k: t.clone() for k, t in g.o.items()}
    w, b = g.want()
    mods = ("dgate", "dscale", "dshift")
    for keep in (("dgate",), ("dgate", "dscale"), ("dgate", "dshift"), ("dscale",), ("dshift",), ("dscale", "dshift"), ()):
        for t in g.o.values():
            t.fill_(float("nan"))
        lm.lazymar_join_grad(g.args(**{k: None for k in mods if k not in keep}))
        sync()
        for k in ("dx", "dy") + keep:
            if "dgate" in keep:
                assert torch.equal(g.o[k], first[k]), (keep, k)
            else:
                close(g.o[k], w[k], np.broadcast_to(b[k], w[k].shape))
        for k in mods:
            assert k in keep or g.o[k].isnan().all()


@pytest.mark.parametrize("mod", ["fp32", "bf16"])
@pytest.mark.parametrize("M,D,group", [(700, 1000, 0), (300, 1000, 1), (700, 1000, 9), (1500, 777, 320), (60000, 64, 200)])
def test_plain_join_grad_accumulates(M, D, group, mod):
    """A second pass adds: twice the gradient, exactly in fp32, one rounding in bf16 (half a step of twice the value, 2^-8 of it)."""
    torch = torch_cuda()
    g = Plain(M, D, group, mod=mod, seed=55).check()
    first = {k: t.clone() for k, t in g.o.items()}
    lm.lazymar_join_grad(g.args(accumulate=True))
    sync()
    for k, t in g.o.items():
        if k in ("dx", "dy"):
            assert torch.equal(t, first[k])
        elif mod == "fp32":
            assert torch.equal(t, first[k] + first[k]), k
        else:  # the sum before its first rounding is within 2^-8 of the first result
            a, w = t.double(), first[k].double()
            assert bool(((a - 2 * w).abs() <= w.abs() * (2.0 ** -8 + 2.0 ** -7) + 1e-30).all()), k


@pytest.mark.parametrize("D,pad,offset", [(1024, 0, 0), (777, 3, 1), (1280, 0, 0)])
def test_plain_join_and_its_gradient_in_place(D, pad, offset):
    """z over x, h over y; dx over dz, dh or z and dy over y or dh: what the call beside them gives, bit for bit."""
    torch = torch_cuda()
    M = 900
    t, _ = make(M, D, 7, "fp32", "bf16", pad=pad, offset=offset, seed=56, params=False)
    z, h = out(M, D), out(M, D, "bf16")
    kw = dict(group=7, pre=NORM["layer"], eps=EPS)
    lm.lazymar_join(lm.lazymar_join_args(M, D, z=z, h=h, **t, **kw))
    lm.lazymar_join(lm.lazymar_join_args(M, D, z=t["x"], h=t["y"], **t, **kw))
    sync()
    assert torch.equal(t["x"], z) and torch.equal(t["y"], h)
    for over in (("dz", "y"), ("dh", "z"), ("z", "dh"), ("y", "dz")):
        g = Plain(M, D, 30, pad=pad, offset=offset, seed=57).check()
        want = {k: a.clone() for k, a in g.o.items()}
        lm.lazymar_join_grad(g.args(dx=g.t[over[0]], dy=g.t[over[1]]))
        sync()
        assert torch.equal(g.t[over[0]], want["dx"]) and torch.equal(g.t[over[1]], want["dy"]), over
        for k in ("dgate", "dscale", "dshift"):
            assert torch.equal(g.o[k], want[k]), (over, k)


def test_plain_rows_that_are_not_finite_stay_alone():
    torch = torch_cuda()
    M, D, group = 1200, 1000, 10
    t, _ = make(M, D, group, seed=58, params=False)
    z, h, h8 = out(M, D), out(M, D), Held(M, D)
    call = lm.lazymar_join_args(M, D, group=group, pre=NORM["layer"], eps=EPS, z=z, h=h, h8=lm.lazymar_rows(h8.q, h8.scale), **t)
    lm.lazymar_join(call)
    sync()
    want = [a.clone() for a in (z, h, h8.q)]
    t["x"][2, 5], t["y"][4, D - 1], t["x"][600, 0] = float("nan"), float("inf"), -float("inf")
    lm.lazymar_join(call)
    sync()
    bad = [2, 4, 600]
    for i in bad:
        assert not torch.isfinite(h[i]).all()
    same = torch.ones(M, dtype=torch.bool, device="cuda")
    same[bad] = False
    for a, w in zip((z, h, h8.q), want):
        assert torch.equal(a[same], w[same])
    g = Plain(M, D, group, seed=59).check()
    want = {k: a.clone() for k, a in g.o.items()}
    g.t["dh"][2, 5] = float("nan")
    lm.lazymar_join_grad(g.args())
    sync()
    assert torch.isnan(g.o["dx"][2]).all()
    same[:] = True
    same[2] = False
    assert torch.equal(g.o["dx"][same], want["dx"][same]) and torch.equal(g.o["dy"][same], want["dy"][same])
    for k in ("dgate", "dscale", "dshift"):  # of the other groups
        assert torch.equal(g.o[k][1:], want[k][1:]), k


def test_plain_gradient_against_differences():
    """The directional derivative along each gradient by differences of the kernel's own outputs; the bound's reasons are
    those of the general kernel's test (third-order term 2e-4, rounding 1e-6)."""
    torch = torch_cuda()
    M, D, group = 400, 256, 16
    t, _ = make(M, D, group, seed=60, params=False)
    z, h, st = out(M, D), out(M, D), stats(M)
    r = np.random.default_rng(61)
    dh, dz = (torch.from_numpy((1e-3 * r.standard_normal((M, D))).astype(np.float32)).cuda() for _ in range(2))
    call = lm.lazymar_join_args(M, D, group=group, pre=NORM["layer"], res=0.9, eps=EPS, z=z, h=h, z_mean=st["z_mean"],
                                z_rstd=st["z_rstd"], **t)

    def loss():
        lm.lazymar_join(call)
        return float((z.double() * dz.double()).sum() + (h.double() * dh.double()).sum())
    loss()
    G = M // group
    o = dict(dx=out(M, D), dy=out(M, D), dgate=out(G, D), dscale=out(G, D), dshift=out(G, D))
    ws = torch.empty(lm.lazymar_join_grad_workspace(M, D, group), dtype=torch.uint8, device="cuda")
    zz = z.clone()
    lm.lazymar_join_grad(lm.lazymar_join_grad_args(M, D, group=group, pre=NORM["layer"], res=0.9, dh=dh, dz=dz, z=zz, y=t["y"],
                                                   gate=t["gate"], scale=t["scale"], z_mean=st["z_mean"], z_rstd=st["z_rstd"],
                                                   workspace=ws, **o))
    sync()
    for k in ("x", "y", "gate", "scale", "shift"):
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
