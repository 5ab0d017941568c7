"""Workloads by which the speed of the residual join and of the optimizer's operators is judged.

Between two blocks of a transformer (or of the diffusion head's MLP) stand the norm behind a branch,
its gate, the residual addition and the norm in front of the next branch with its modulation; at the
end of a training step the norm of all gradients, their clipping and the weights' update:

  join       u = norm(y) post_g + post_b, z = res x + gate u, h = (norm(z) pre_g + pre_b) (1 + scale) + shift;
             gate, scale and shift for each row, for each group of rows, or for all; h also as the 8-bit
             operand of the next product, z and y also as 8-bit checkpoints
  join_grad  its gradient, from tensors or checkpoints, with those of gate, scale, shift and the norms' parameters
  norm       the norm over many tensors, the factor that clips it and the count of steps, on the device
  clip       the gradients times that factor, into tensors of their own
  adamw      the update of weights, moments, averaged weights and a bf16 copy, with that factor; `norm`: with the
             norm before it, as a training step ends

Widths, rows and depths are those of the repository's configurations (synth/inputs.py: widths 1024 and 1280,
320 tokens for each of up to 128 rows, 32 blocks of width 1024 the largest list here), and odd ones of the same
ranges. `own` chooses between the plain form of torch operations in fp32 and the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, BETA1, BETA2, ADAM_EPS, DECAY, EMA = 1e-4, 0.9, 0.95, 1e-8, 0.02, 0.9999
MOST = 404_000_000  # elements of the largest list


def listed():
    return [
        # the head's block of two rows (conditional and unconditional) of one token, each with its own modulation: latency
        dict(name="join-token", kind="join", M=2, D=1024, x="f32", y="bf16", z="f32", h="bf16", h8=False, z8=False, y8=False,
             post="none", pre="layer", group=1, mod="bf16", gate=True, scale=True, post_g=False, pre_g=False, res=1.0,
             pad=0),
        # a training step over 128 rows of 320 tokens, modulated by row: 8-bit operand and checkpoints
        dict(name="join-train", kind="join", M=40960, D=1024, x="f32", y="bf16", z="f32", h="", h8=True, z8=True, y8=True,
             post="none", pre="layer", group=320, mod="bf16", gate=True, scale=True, post_g=False, pre_g=False, res=1.0,
             pad=0),
        # norms on both sides of a block, a gate for all rows and a scaled residual, odd width, bf16 throughout
        dict(name="join-sandwich-odd", kind="join", M=4801, D=777, x="bf16", y="bf16", z="bf16", h="bf16", h8=False,
             z8=False, y8=False, post="rms", pre="rms", group=0, mod="f32", gate=True, scale=False, post_g=True,
             pre_g=True, res=0.8, pad=0),
        # the gradient of a training step from 8-bit checkpoints, modulation of each row of 320 tokens
        dict(name="join-grad-train", kind="join_grad", M=40960, D=1280, dh="bf16", dz="f32", z="block8", y="block8",
             dx="f32", dy="bf16", dy8=True, post="none", pre="layer", group=320, mod="bf16", gate=True, scale=True,
             post_g=False, pre_g=False, res=1.0, pad=0),
        # the head's training: every token has its own modulation, whose gradients are as large as the rows
        dict(name="join-grad-rows", kind="join_grad", M=16384, D=1024, dh="bf16", dz="f32", z="f32", y="bf16",
             dx="f32", dy="bf16", dy8=False, post="none", pre="layer", group=1, mod="bf16", gate=True, scale=True,
             post_g=False, pre_g=False, res=1.0, pad=0),
        # the gradient of norms on both sides at an odd width, with those of gains and gate
        dict(name="join-grad-sandwich-odd", kind="join_grad", M=4801, D=777, dh="bf16", dz="bf16", z="bf16", y="bf16",
             dx="bf16", dy="bf16", dy8=False, post="rms", pre="rms", group=0, mod="f32", gate=True, scale=False,
             post_g=True, pre_g=True, res=0.8, pad=0),
        # the gradients of the MLP half of one block
        dict(name="norm-mlp", kind="norm", layout="mlp", D=1024, depth=1, g="f32", packed=False),
        # the gradients of a whole model: 32 blocks of width 1024
        dict(name="norm-model", kind="norm", layout="block", D=1024, depth=32, g="f32", packed=False),
        # a block of odd width in one buffer, tensor behind tensor (none aligned), fp32 sums into bf16
        dict(name="clip-block-odd", kind="clip", layout="block", D=777, depth=1, g="f32", out="bf16", packed=True),
        # eight blocks' gradients
        dict(name="clip-blocks", kind="clip", layout="block", D=1280, depth=8, g="f32", out="f32", packed=False),
        # tuning the gains and shifts of a model alone: 128 small tensors
        dict(name="adamw-gains", kind="adamw", layout="gains", D=1024, depth=32, g="f32", packed=False, ema=False,
             copy=False, norm=False),
        # the end of a training step of a whole model: norm, update, averaged weights, bf16 copy; the largest
        dict(name="adamw-model", kind="adamw", layout="block", D=1024, depth=32, g="f32", packed=False, ema=True,
             copy=True, norm=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice([256, 768, 1024, 1280, rng.randint(64, 1400), 8 * rng.randint(8, 180)])


def draw(rng):
    kind = rng.choice(["join", "join", "join", "join_grad", "join_grad", "join_grad", "norm", "clip", "adamw", "adamw"])
    if kind in ("join", "join_grad"):
        c = dict(kind=kind, M=_log(rng, 1, 40960), D=_width(rng), post=rng.choice(["none", "none", "layer", "rms"]),
                 pre=rng.choice(["layer", "layer", "rms"]), group=rng.choice([0, 1, 320, _log(rng, 1, 2000)]),
                 mod=rng.choice(["f32", "bf16"]), gate=rng.random() < 0.8, scale=rng.random() < 0.6,
                 post_g=rng.random() < 0.4, pre_g=rng.random() < 0.4, res=rng.choice([1.0, 1.0, 0.8]),
                 pad=rng.choice([0, 0, 0, 8, rng.randint(1, 40)]))
        if kind == "join":
            h, h8 = rng.choice([("bf16", False), ("f32", False), ("", True), ("bf16", True)])
            c.update(x=rng.choice(["f32", "f32", "bf16"]), y=rng.choice(["bf16", "bf16", "f32", "block8"]),
                     z=rng.choice(["f32", "f32", "bf16"]), h=h, h8=h8, z8=rng.random() < 0.4, y8=rng.random() < 0.3)
        else:
            c.update(dh=rng.choice(["bf16", "bf16", "f32"]), dz=rng.choice(["f32", "f32", "bf16", ""]),
                     z=rng.choice(["f32", "bf16", "block8", "block8"]), y=rng.choice(["bf16", "f32", "block8"]),
                     dx=rng.choice(["f32", "f32", "bf16"]), dy=rng.choice(["bf16", "bf16", "f32"]),
                     dy8=rng.random() < 0.4)
        return c
    layout = rng.choice(["mlp", "block", "block", "gains"])
    D = rng.choice([256, 768, 1024, 1280, _log(rng, 64, 1400)])
    one = sum(_sizes(dict(layout=layout, D=D, depth=1)))
    c = dict(kind=kind, layout=layout, D=D, depth=_log(rng, 1, max(1, min(40, MOST // one))),
             g=rng.choice(["f32", "f32", "bf16"]), packed=rng.random() < 0.3)
    if kind == "clip":
        c.update(out=rng.choice(["f32", "bf16"]))
    if kind == "adamw":
        c.update(ema=rng.random() < 0.5, copy=rng.random() < 0.6, norm=rng.random() < 0.5)
    return c


def _sizes(case):
    """Elements of each tensor of a list."""
    D = case["D"]
    H = 4 * D
    one = {"gains": [D, D, D, D],
           "mlp": [D, D, H * D, H, D * H, D],
           "block": [D, D, 3 * D * D, 3 * D, D * D, D, D, D, H * D, H, D * H, D]}[case["layout"]]
    return one * case["depth"]


# ---------------------------------------------------------------------------
# The 8-bit format, in torch operations
# ---------------------------------------------------------------------------
def _exponent(amax):
    """The smallest e >= -126 with amax <= 448 2^e (448 = 0.875 2^9)."""
    m, e = torch.frexp(amax)
    return (e.int() - 9 + (m > 0.875).int()).clamp(min=-126)


def _power(e):
    """2^e as fp32, exactly, -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _pack(x):
    """x [M, D] fp32 -> E4M3 values [M, D] (float8) and exponent bytes [blocks of 128, M]."""
    M, D = x.shape
    nb = -(-D // 128)
    p = torch.nn.functional.pad(x, (0, nb * 128 - D)).view(M, nb, 128)
    e = _exponent(p.abs().amax(-1))
    q = (p * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return q.view(M, nb * 128)[:, :D], (e + 127).to(torch.uint8).t().contiguous()


def _held(q, scale):
    """An 8-bit tensor as a program keeps it: rows on 16-byte boundaries."""
    M, D = q.shape
    buf = torch.zeros((M, -(-D // 16) * 16), dtype=torch.uint8, device=DEV)
    buf[:, :D] = q.view(torch.uint8)
    return buf, scale


def _empty8(M, D):
    return (torch.zeros((M, -(-D // 16) * 16), dtype=torch.uint8, device=DEV),
            torch.zeros((-(-D // 128), M), dtype=torch.uint8, device=DEV))


def _e4m3(held, D):
    """The bytes of a held tensor as E4M3 values, and its scales as the powers of two that they stand for."""
    return dict(q=held[0][:, :D].view(torch.float8_e4m3fn), scale=held[1].view(torch.float8_e8m0fnu))


def _values(held, D):
    """The fp32 values of a held tensor."""
    s = _power(held[1].int() - 127).t().repeat_interleave(128, 1)
    return held[0][:, :D].view(torch.float8_e4m3fn).float() * s[:, :D]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _groups(c):
    """Rows that share a modulation, and how many such groups there are."""
    group = c["group"] or c["M"]
    return group, -(-c["M"] // group)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    c, kind = dict(case), case["kind"]
    s = dict(case=c)
    if kind in ("join", "join_grad"):
        M, D, pad = c["M"], c["D"], c["pad"]
        G = _groups(c)[1]

        def rows(std, dtype):
            """Rows of different size, some columns much larger, as activations and their gradients have them."""
            x = normal(M, D) * torch.exp(0.5 * normal(M, 1)) * torch.exp(0.7 * normal(1, D)) * std
            if dtype == "block8":
                return _held(*_pack(x))
            buf = torch.zeros((M, D + pad), dtype=TORCH[dtype], device=DEV)
            buf[:, :D] = x
            return buf[:, :D]

        def empty(n, dtype, more=pad):
            return torch.empty((n, D + more), dtype=TORCH[dtype], device=DEV)[:, :D] if dtype else None

        # shift, scale and gate as the modulation's linear layer gives them: side by side
        mod = (0.3 * normal(G, 3 * D)).to(TORCH[c["mod"]])
        s["shift"], s["scale"] = (mod[:, :D], mod[:, D:2 * D]) if c["scale"] else (None, None)
        s["gate"] = mod[:, 2 * D:] if c["gate"] else None
        s["post_g"], s["post_b"] = (1 + 0.1 * normal(D), 0.02 * normal(D)) if c["post_g"] else (None, None)
        s["pre_g"], s["pre_b"] = (1 + 0.1 * normal(D), 0.02 * normal(D)) if c["pre_g"] else (None, None)
        s["stats"] = torch.empty((4, M), device=DEV)  # mean and 1 / deviation of y, then of z
    if kind == "join":
        s["x"], s["y"] = rows(1.0, c["x"]), rows(0.5, c["y"])
        s["z"], s["h"] = empty(M, c["z"]), empty(M, c["h"])
        s["h8"], s["z8"], s["y8"] = (_empty8(M, D) if c[k] else None for k in ("h8", "z8", "y8"))
    elif kind == "join_grad":
        s["z"], s["y"] = rows(1.0, c["z"]), rows(0.5, c["y"])
        s["dh"] = rows(1e-3, c["dh"])
        s["dz"] = rows(1e-3, c["dz"]) if c["dz"] else None
        for at, name, norm in ((0, "y", c["post"]), (2, "z", c["pre"])):
            v = _values(s[name], D) if c[name] == "block8" else s[name].float()
            mean = v.mean(1) if norm == "layer" else torch.zeros(M, device=DEV)
            s["stats"][at] = mean
            s["stats"][at + 1] = torch.rsqrt((v - mean[:, None]).square().mean(1) + EPS)
        s["dx"], s["dy"] = empty(M, c["dx"]), empty(M, c["dy"])
        s["dy8"] = _empty8(M, D) if c["dy8"] else None
        dmod = torch.empty((G, 3 * D), dtype=TORCH[c["mod"]], device=DEV)
        s["dshift"], s["dscale"] = (dmod[:, :D], dmod[:, D:2 * D]) if c["scale"] else (None, None)
        s["dgate"] = dmod[:, 2 * D:] if c["gate"] else None
        s["dpost_g"], s["dpost_b"] = (torch.empty(D, device=DEV) for _ in range(2)) if c["post_g"] else (None, None)
        s["dpre_g"], s["dpre_b"] = (torch.empty(D, device=DEV) for _ in range(2)) if c["pre_g"] else (None, None)
    if kind in ("join", "join_grad"):
        return s

    # a list: each kind of tensor in one buffer, the tensors as views of it, on boundaries of 64 elements or packed
    sizes = _sizes(c)
    room = sizes if c["packed"] else [-(-n // 64) * 64 for n in sizes]
    at = [0]
    for n in room:
        at.append(at[-1] + n)

    def views(flat):
        return [flat[a:a + n] for a, n in zip(at, sizes)]

    def zero_gaps(flat):
        for a, n, r in zip(at, sizes, room):
            if r > n:
                flat[a + n:a + r] = 0
        return flat

    total = at[-1]
    s["sizes"], s["room"] = sizes, torch.tensor(room, device=DEV)
    # a model's gradients: small, of different size from tensor to tensor
    size = torch.exp(0.7 * normal(len(sizes))) * 1e-3
    grad = normal(total)
    grad *= torch.repeat_interleave(size, s["room"], output_size=total)
    s["g"] = zero_gaps(grad.to(TORCH[c["g"]]))
    del grad
    lists = dict(g=views(s["g"]))
    # norm, factor, and (as bits of whole numbers) steps taken and skipped
    s["state"] = torch.tensor([0.0, 0.37, 0.0, 0.0], device=DEV)
    s["state"].view(torch.int32)[2] = 0 if c.get("norm") else 137
    if kind == "clip":
        s["out"] = torch.zeros(total, dtype=TORCH[c["out"]], device=DEV)
        lists["out"] = views(s["out"])
    if kind == "adamw":
        s["p"] = zero_gaps(0.02 * normal(total))
        s["m"] = s["g"].float() * 0.3 + zero_gaps(1e-4 * normal(total))
        s["v"] = zero_gaps(1e-6 * normal(total).square() + 1e-9)
        for k in ("p", "m", "v"):
            lists[k] = views(s[k])
        if c["ema"]:
            s["ema"] = zero_gaps(s["p"] + 1e-3 * normal(total))
            lists["ema"] = views(s["ema"])
        if c["copy"]:
            s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
            lists["copy"] = views(s["copy"])
        # matrices decay, gains and biases do not
        s["decay"] = [DECAY if n > 4 * c["D"] else 0.0 for n in sizes]
        s["decay_of"] = torch.tensor(s["decay"], device=DEV)
    s["lists"] = lists
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _norm(x, kind):
    """(normalised x, mean, 1 / deviation)"""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    d = x - mean
    rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
    return d * rstd, mean, rstd


def _norm_grad(d, n, rstd, kind):
    d = d - n * (d * n).mean(1, keepdim=True) - (d.mean(1, keepdim=True) if kind == "layer" else 0.0)
    return d * rstd


def _out8(x):
    q, scale = _pack(x)
    return dict(q=q, scale=scale.view(torch.float8_e8m0fnu))


def _group_sums(x, group, G):
    M, D = x.shape
    if G == M:
        return x
    return torch.nn.functional.pad(x, (0, 0, 0, G * group - M)).view(G, group, D).sum(1)


def _wide(t, c, kind):
    return _values(t, c["D"]) if kind == "block8" else t.float()


def _plain_join(s):
    c = s["case"]
    of = torch.arange(c["M"], device=DEV) // _groups(c)[0]
    x, y = s["x"].float(), _wide(s["y"], c, c["y"])
    out = {}
    u = y
    if c["post"] != "none":
        u, mean, rstd = _norm(y, c["post"])
        out["y_mean"], out["y_rstd"] = mean[:, 0], rstd[:, 0]
    if c["post_g"]:
        u = u * s["post_g"] + s["post_b"]
    if c["gate"]:
        u = u * s["gate"].float()[of]
    z = x * c["res"] + u
    n, mean, rstd = _norm(z, c["pre"])
    out["z_mean"], out["z_rstd"] = mean[:, 0], rstd[:, 0]
    h = n * s["pre_g"] + s["pre_b"] if c["pre_g"] else n
    if c["scale"]:
        h = h * (1 + s["scale"].float()[of]) + s["shift"].float()[of]
    out.update(z=z.to(TORCH[c["z"]]), h=h.to(TORCH[c["h"]]) if c["h"] else None, h8=_out8(h) if c["h8"] else None,
               z8=_out8(z) if c["z8"] else None, y8=_out8(y) if c["y8"] else None)
    return out


def _plain_join_grad(s):
    c = s["case"]
    group, G = _groups(c)
    of = torch.arange(c["M"], device=DEV) // group
    y, z = _wide(s["y"], c, c["y"]), _wide(s["z"], c, c["z"])
    dh = s["dh"].float()
    ym, yr, zm, zr = (v[:, None] for v in s["stats"])
    n = (z - zm) * zr
    t = n * s["pre_g"] + s["pre_b"] if c["pre_g"] else n
    out = {}
    dt = dh
    if c["scale"]:
        out["dshift"] = _group_sums(dh, group, G).to(TORCH[c["mod"]])
        out["dscale"] = _group_sums(dh * t, group, G).to(TORCH[c["mod"]])
        dt = dh * (1 + s["scale"].float()[of])
    dn = dt
    if c["pre_g"]:
        out["dpre_g"], out["dpre_b"] = (dt * n).sum(0), dt.sum(0)
        dn = dt * s["pre_g"]
    dz = _norm_grad(dn, n, zr, c["pre"])
    if c["dz"]:
        dz = dz + s["dz"].float()
    u = (y - ym) * yr if c["post"] != "none" else y
    dv = dz
    if c["gate"]:
        v = u * s["post_g"] + s["post_b"] if c["post_g"] else u
        out["dgate"] = _group_sums(dz * v, group, G).to(TORCH[c["mod"]])
        dv = dz * s["gate"].float()[of]
    du = dv
    if c["post_g"]:
        out["dpost_g"], out["dpost_b"] = (dv * u).sum(0), dv.sum(0)
        du = dv * s["post_g"]
    dy = du if c["post"] == "none" else _norm_grad(du, u, yr, c["post"])
    out.update(dx=(dz * c["res"]).to(TORCH[c["dx"]]), dy=dy.to(TORCH[c["dy"]]), dy8=_out8(dy) if c["dy8"] else None)
    return out


MAX_NORM = 1.0


def _plain_norm(s):
    norm = s["g"].float().square().sum(dtype=torch.float64).sqrt().float()
    s["state"][0] = norm
    s["state"][1] = (MAX_NORM / norm).clamp(max=1.0)
    s["state"].view(torch.int32)[2] += 1


def _plain_adamw(s):
    c = s["case"]
    steps, factor = s["state"].view(torch.int32)[2].double(), s["state"][1]
    g = s["g"].float() * factor
    s["m"] += (g - s["m"]) * (1 - BETA1)
    s["v"] += (g * g - s["v"]) * (1 - BETA2)
    step = s["m"] / (1 - BETA1 ** steps).float()
    step /= (s["v"] / (1 - BETA2 ** steps).float()).sqrt() + ADAM_EPS
    decay = torch.repeat_interleave(s["decay_of"], s["room"], output_size=s["p"].numel())
    s["p"] -= LR * (step + decay * s["p"])
    if c["ema"]:
        s["ema"] += (s["p"] - s["ema"]) * (1 - EMA)
    if c["copy"]:
        s["copy"].copy_(s["p"])


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "join":
        return _plain_join(s)
    if kind == "join_grad":
        return _plain_join_grad(s)
    if kind == "norm":
        _plain_norm(s)
    elif kind == "clip":
        s["out"].copy_(s["g"].float() * s["state"][1])
    else:
        if s["case"]["norm"]:
            _plain_norm(s)
        _plain_adamw(s)
    return _state_out(s)


def _state_out(s):
    """The buffers that a pass over a list has written."""
    c, kind = s["case"], s["case"]["kind"]
    out = {}
    if kind == "norm" or c.get("norm"):
        out.update(norm=s["state"][0], factor=s["state"][1])
    if kind == "clip":
        out["out"] = s["out"]
    if kind == "adamw":
        out.update(p=s["p"], m=s["m"], v=s["v"], ema=s.get("ema"), copy=s.get("copy"))
    return out


def _plan(s):
    """What a program keeps between calls: descriptors of its buffers, a workspace, the handle of its list."""
    from paper_2503_12450_gb300 import lazymar as lm

    c, kind = s["case"], s["case"]["kind"]
    if kind in ("join", "join_grad"):
        def rows(t):
            return None if t is None else lm.lazymar_rows(*t) if isinstance(t, tuple) else lm.lazymar_rows(t)
        norms = {"none": lm.LAZYMAR_NORM_NONE, "layer": lm.LAZYMAR_NORM_LAYER, "rms": lm.LAZYMAR_NORM_RMS}
        same = dict(M=c["M"], D=c["D"], group=c["group"], post=norms[c["post"]], pre=norms[c["pre"]], res=c["res"],
                    gate=rows(s["gate"]), scale=rows(s["scale"]))
        same.update({k: s[k] for k in ("post_g", "post_b", "pre_g", "pre_b")})
        if c["post"] != "none":
            same.update(y_mean=s["stats"][0], y_rstd=s["stats"][1])
        same.update(z_mean=s["stats"][2], z_rstd=s["stats"][3])
        if kind == "join":
            more = {k: rows(s[k]) for k in ("x", "y", "z", "h", "h8", "z8", "y8", "shift")}
            return lm, lm.lazymar_join_args(eps=EPS, **same, **more)
        size = lm.lazymar_join_grad_workspace(c["M"], c["D"], c["group"])
        more = {k: rows(s[k]) for k in ("dh", "dz", "z", "y", "dx", "dy", "dy8", "dgate", "dscale", "dshift")}
        more.update({k: s[k] for k in ("dpost_g", "dpost_b", "dpre_g", "dpre_b")})
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        return lm, lm.lazymar_join_grad_args(workspace=ws, **same, **more)
    keys = [k for k in ("g", "out", "p", "m", "v", "ema", "copy") if k in s["lists"]]
    entries = [dict(zip(keys, t)) for t in zip(*(s["lists"][k] for k in keys))]
    if kind == "adamw":
        entries = [dict(e, weight_decay=d) for e, d in zip(entries, s["decay"])]
    return lm, lm.lazymar_params_create(entries)


def _own(s):
    c, kind = s["case"], s["case"]["kind"]
    if "plan" not in s:
        s["plan"] = _plan(s)
    lm, plan = s["plan"]
    if kind == "join":
        lm.lazymar_join(plan)
        out = dict(z=s["z"], h=s["h"], z_mean=s["stats"][2], z_rstd=s["stats"][3])
        if c["post"] != "none":
            out.update(y_mean=s["stats"][0], y_rstd=s["stats"][1])
        out.update({k: _e4m3(s[k], c["D"]) for k in ("h8", "z8", "y8") if c[k]})
        return out
    if kind == "join_grad":
        lm.lazymar_join_grad(plan)
        out = {k: s[k] for k in ("dx", "dy", "dgate", "dscale", "dshift", "dpost_g", "dpost_b", "dpre_g", "dpre_b")}
        return dict(out, dy8=_e4m3(s["dy8"], c["D"])) if c["dy8"] else out
    if kind == "norm" or c.get("norm"):
        lm.lazymar_grad_norm(plan, s["state"], MAX_NORM)
    if kind == "clip":
        lm.lazymar_clip_grads(plan, s["state"])
    elif kind == "adamw":
        lm.lazymar_adamw(plan, s["state"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS,
                         ema_decay=EMA if c["ema"] else 0.0)
    return _state_out(s)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "bf16": 2, "block8": 1 + 1 / 128, "": 0}
    e8 = size["block8"]
    c, kind = case, case["kind"]
    if kind in ("join", "join_grad"):
        M, D = c["M"], c["D"]
        n, mods = M * D, _groups(c)[1] * D * size[c["mod"]]
        params = 8 * D * (c["post_g"] + c["pre_g"])
        if kind == "join":
            each = size[c["x"]] + size[c["y"]] + size[c["z"]] + size[c["h"]] + e8 * (c["h8"] + c["z8"] + c["y8"])
            return dict(bytes=n * each + mods * (c["gate"] + 2 * c["scale"]) + params + 8 * M * (1 + (c["post"] != "none")),
                        flops=30 * n)
        reads_y = c["gate"] or c["post_g"] or c["post"] != "none"  # a bare addition passes its gradient on
        each = (size[c["dh"]] + size[c["dz"]] + size[c["z"]] + size[c["y"]] * reads_y + size[c["dx"]] + size[c["dy"]]
                + e8 * c["dy8"])
        return dict(bytes=n * each + mods * (2 * c["gate"] + 3 * c["scale"]) + 2 * params
                    + 8 * M * (1 + (c["post"] != "none")), flops=40 * n)
    n = sum(_sizes(c))
    if kind == "norm":
        return dict(bytes=n * size[c["g"]], flops=2 * n)
    if kind == "clip":
        return dict(bytes=n * (size[c["g"]] + size[c["out"]]), flops=n)
    return dict(bytes=n * (size[c["g"]] + 24 + 8 * c["ema"] + 2 * c["copy"]), flops=20 * n)


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(t, kind, D):
    if kind != "block8":
        return t.double()
    b, block = t[0][:, :D].int(), torch.arange(D, device=DEV) // 128
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * _two(e - 7)) * (1 - 2 * (b >> 7).double())
    return v * _two(t[1].int() - 127)[block].t()


def _exact8(x):
    """x in 64 bits rounded to 8: the E4M3 values and the scales."""
    M, D = x.shape
    nb = (D + 127) // 128
    big = torch.stack([x[:, 128 * j:128 * j + 128].abs().amax(1) for j in range(nb)], 1)
    e = torch.ceil(torch.log2(big.clamp(min=2.0 ** -200) / 448)) - 1  # or one more: log2 rounds
    e = torch.where(big <= 448 * _two(e), e, e + 1).clamp(min=-126)
    v = x / _two(e)[:, torch.arange(D, device=DEV) // 128]
    step = _two(torch.frexp(v.abs().clamp(min=2.0 ** -6))[1] - 4)  # of three mantissa bits
    return dict(q=torch.round(v / step) * step, scale=_two(e).t())


def _exact_mod(t, case):
    """A row of t for each row of the tensors."""
    group, G = _groups(case)
    return t.double().repeat_interleave(group, 0)[:case["M"]]


def _exact_sums(x, case):
    group, G = _groups(case)
    if G == 1:
        return x.sum(0, keepdim=True)
    return torch.stack([part.sum(0) for part in x.split(group)]) if group > 1 else x


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "join":
        D = c["D"]
        y = _exact_rows(s["y"], c["y"], D)
        out, u = {}, y
        if c["post"] != "none":
            mean = y.sum(1) / D if c["post"] == "layer" else torch.zeros(c["M"], dtype=torch.float64, device=DEV)
            rstd = 1 / torch.sqrt(((y - mean[:, None]) ** 2).sum(1) / D + EPS)
            u = (y - mean[:, None]) * rstd[:, None]
            out.update(y_mean=mean, y_rstd=rstd)
        v = u * s["post_g"].double() + s["post_b"].double() if c["post_g"] else u
        z = s["x"].double() * c["res"] + (_exact_mod(s["gate"], c) * v if c["gate"] else v)
        mean = z.sum(1) / D if c["pre"] == "layer" else torch.zeros(c["M"], dtype=torch.float64, device=DEV)
        rstd = 1 / torch.sqrt(((z - mean[:, None]) ** 2).sum(1) / D + EPS)
        h = (z - mean[:, None]) * rstd[:, None]
        if c["pre_g"]:
            h = h * s["pre_g"].double() + s["pre_b"].double()
        if c["scale"]:
            h = h * (1 + _exact_mod(s["scale"], c)) + _exact_mod(s["shift"], c)
        out.update(z_mean=mean, z_rstd=rstd, z=z, h=h if c["h"] else None, h8=_exact8(h) if c["h8"] else None,
                   z8=_exact8(z) if c["z8"] else None, y8=_exact8(y) if c["y8"] else None)
        return out
    if kind == "join_grad":
        D = c["D"]
        stats = s["stats"].double()
        one = torch.ones(D, dtype=torch.float64, device=DEV)
        n = (_exact_rows(s["z"], c["z"], D) - stats[2][:, None]) * stats[3][:, None]
        u = _exact_rows(s["y"], c["y"], D)
        if c["post"] != "none":
            u = (u - stats[0][:, None]) * stats[1][:, None]
        pre_g, pre_b = (s["pre_g"].double(), s["pre_b"].double()) if c["pre_g"] else (one, 0 * one)
        post_g, post_b = (s["post_g"].double(), s["post_b"].double()) if c["post_g"] else (one, 0 * one)
        dh, out = s["dh"].double(), {}
        more = 1 + _exact_mod(s["scale"], c) if c["scale"] else 1.0
        if c["scale"]:
            out.update(dshift=_exact_sums(dh, c), dscale=_exact_sums(dh * (n * pre_g + pre_b), c))
        if c["pre_g"]:
            out.update(dpre_g=(dh * more * n).sum(0), dpre_b=(dh * more).sum(0))
        d = dh * more * pre_g
        m1 = d.sum(1, keepdim=True) / D if c["pre"] == "layer" else 0.0
        dz = stats[3][:, None] * (d - m1 - n * ((d * n).sum(1, keepdim=True) / D))
        if c["dz"]:
            dz = dz + s["dz"].double()
        gate = _exact_mod(s["gate"], c) if c["gate"] else 1.0
        if c["gate"]:
            out["dgate"] = _exact_sums(dz * (u * post_g + post_b), c)
        if c["post_g"]:
            out.update(dpost_g=(dz * gate * u).sum(0), dpost_b=(dz * gate).sum(0))
        d = dz * gate * post_g
        if c["post"] != "none":
            m1 = d.sum(1, keepdim=True) / D if c["post"] == "layer" else 0.0
            d = stats[1][:, None] * (d - m1 - u * ((d * u).sum(1, keepdim=True) / D))
        out.update(dx=dz * c["res"], dy=d, dy8=_exact8(d) if c["dy8"] else None)
        return out
    out = {}
    factor, steps = s["state"][1].double(), int(s["state"].view(torch.int32)[2])
    if kind == "norm" or c.get("norm"):
        norm = torch.sqrt(sum((g.double() ** 2).sum() for g in s["lists"]["g"]))
        factor, steps = torch.clamp(MAX_NORM / norm, max=1.0), steps + 1
        out.update(norm=norm, factor=factor)
    if kind == "clip":
        out["out"] = s["g"].double() * factor
    if kind == "adamw":
        g = s["g"].double() * factor
        m = BETA1 * s["m"].double() + (1 - BETA1) * g
        v = BETA2 * s["v"].double() + (1 - BETA2) * g * g
        del g
        p = s["p"].double()
        at = 0
        for n, r, decay in zip(s["sizes"], s["room"].tolist(), s["decay"]):
            p[at:at + n] *= 1 - LR * decay
            at += r
        p -= LR * (m / (1 - BETA1 ** steps)) / (torch.sqrt(v / (1 - BETA2 ** steps)) + ADAM_EPS)
        out.update(p=p, m=m, v=v, copy=p if c["copy"] else None)
        if c["ema"]:
            out["ema"] = EMA * s["ema"].double() + (1 - EMA) * p
    return out
