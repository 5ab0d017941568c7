"""Workloads by which the speed of the training operators is judged.

The operators train and serve a block whose activations are kept in 8 bits
("block8": E4M3 bytes with one power-of-two scale for each row and 128 columns;
weights one for each 128 x 128 block):

  ln_fwd    LayerNorm with statistics, its output in bf16 or as the 8-bit operand
            of the next product, and an 8-bit checkpoint of its input
  ln_bwd    LayerNorm's gradient from the statistics and the (checkpointed) input,
            with the gradients of gain and shift
  save      an activation into its 8-bit checkpoint
  load      the checkpoint back into bf16 or fp32
  gelu_bwd  the gradient through GELU from the 8-bit checkpoint of its input, also
            as 8-bit operand of the next product, with the bias gradient
  linear    the 8-bit product with its fused outputs: bias, GELU (8-bit output and
            checkpoint, or bf16), residual addition in fp32
  wgrad     the weight gradient from the output's gradient and the checkpoint

Widths and row counts are those of the repository's configurations (synth/inputs.py:
widths 768, 1024 and 1280 with MLPs four times as wide, 320 or 1088 tokens for each of
up to 128 rows), and odd ones of the same ranges. `own` chooses between the plain form
of torch operations in fp32 and the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token's LayerNorm in front of a projection: the smallest call
        dict(name="ln-forward-token", kind="ln_fwd", M=1, D=1024, x="f32", y="bf16", y8=False, x8=False, pad=0),
        # a training step's LayerNorm over 128 rows of 320 tokens: 8-bit operand, checkpoint, statistics
        dict(name="ln-forward-train", kind="ln_fwd", M=40960, D=1024, x="f32", y="", y8=True, x8=True, pad=0),
        # gradient at an odd width in rows that are not aligned, bf16 throughout
        dict(name="ln-backward-odd", kind="ln_bwd", M=4801, D=777, x="bf16", dy="bf16", dres=False, dx="bf16", pad=0),
        # a training step's LayerNorm gradient, input from its checkpoint, added to the residual stream's gradient
        dict(name="ln-backward-train", kind="ln_bwd", M=40960, D=1280, x="block8", dy="bf16", dres=True, dx="f32",
             pad=0),
        # an MLP activation of 64 rows of 320 tokens into its checkpoint
        dict(name="save-mlp", kind="save", M=20480, D=4096, x="bf16", pad=0),
        # GELU's gradient on the recomputed tokens of a few rows, ragged
        dict(name="gelu-backward-ragged", kind="gelu_bwd", M=1111, D=5000, da="bf16", du="bf16", du8=True, pad=8),
        # GELU's gradient of a training step
        dict(name="gelu-backward-train", kind="gelu_bwd", M=40960, D=4096, da="bf16", du="bf16", du8=True, pad=0),
        # the MLP's up-projection of two tokens: latency and the weights' bytes
        dict(name="linear-token", kind="linear", epi="gelu", M=2, N=4096, K=1024, out="bf16", u8=False),
        # the MLP's up-projection of a training step: 8-bit output and checkpoint of GELU's input
        dict(name="linear-gelu-train", kind="linear", epi="gelu", M=20480, N=5120, K=1280, out="block8", u8=True),
        # the MLP's down-projection into the fp32 residual stream: the largest
        dict(name="linear-residual-train", kind="linear", epi="residual", M=40960, N=1024, K=4096, out="f32",
             u8=False),
        # weight gradient of ragged sizes: few tiles, a long sum
        dict(name="wgrad-ragged", kind="wgrad", M=3211, N=1000, K=776),
        # weight gradient of the up-projection of a training step
        dict(name="wgrad-train", kind="wgrad", M=20480, N=4096, K=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice([256, 768, 1024, 1280, rng.randint(64, 1400), 8 * rng.randint(8, 180)])


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_fwd", "ln_bwd", "ln_bwd", "save", "load", "gelu_bwd", "gelu_bwd", "linear",
                       "linear", "linear", "linear", "wgrad", "wgrad"])
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 40)])
    M = _log(rng, 1, 40960)
    if kind == "ln_fwd":
        y8, y = rng.choice([(False, "bf16"), (False, "f32"), (True, ""), (True, "bf16")])
        return dict(kind=kind, M=M, D=_width(rng), x=rng.choice(["f32", "bf16"]), y=y, y8=y8,
                    x8=rng.random() < 0.5, pad=pad)
    if kind == "ln_bwd":
        return dict(kind=kind, M=M, D=_width(rng), x=rng.choice(["f32", "bf16", "block8", "block8"]),
                    dy=rng.choice(["f32", "bf16", "bf16"]), dres=rng.random() < 0.5, dx=rng.choice(["f32", "bf16"]),
                    pad=pad)
    if kind == "save" or kind == "load":
        return dict(kind=kind, M=M, D=_log(rng, 64, 5120), x=rng.choice(["f32", "bf16"]), pad=pad)
    if kind == "gelu_bwd":
        du, du8 = rng.choice([("bf16", True), ("bf16", True), ("f32", False), ("", True)])
        return dict(kind=kind, M=M, D=_log(rng, 256, 5120), da=rng.choice(["bf16", "bf16", "f32"]), du=du, du8=du8,
                    pad=pad)
    D = rng.choice([256, 768, 1024, 1280, rng.randint(64, 1280)])
    H = rng.choice([1024, 4096, 5120, rng.randint(300, 5120)])
    N, K = (D, H) if rng.random() < 0.5 else (H, D)
    if kind == "linear":
        M = _log(rng, 1, max(2, min(40960, int(171e9 / (N * K)))))
        epi = rng.choice(["bias", "gelu", "gelu", "residual"])
        out = {"bias": rng.choice(["bf16", "f32", "block8"]), "gelu": rng.choice(["block8", "bf16"]),
               "residual": "f32"}[epi]
        return dict(kind=kind, epi=epi, M=M, N=N, K=K, out=out, u8=epi == "gelu" and rng.random() < 0.6)
    return dict(kind=kind, M=_log(rng, 64, max(65, min(40960, int(86e9 / (N * K))))), N=8 * ((N + 7) // 8), K=K)


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
    e = _exponent(torch.where(p.isfinite(), p.abs(), 0.0).amax(-1))
    q = (p * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return q.view(M, nb * 128)[:, :D], (e + 127).to(torch.uint8).t().contiguous()


def _pack_weight(w):
    """w [N, K] fp32 -> E4M3 values [N, K] and exponent bytes [blocks of K, blocks of N]."""
    N, K = w.shape
    nn, nk = -(-N // 128), -(-K // 128)
    p = torch.nn.functional.pad(w, (0, nk * 128 - K, 0, nn * 128 - N)).view(nn, 128, nk, 128)
    e = _exponent(p.abs().amax(dim=(1, 3)))
    q = (p * _power(-e)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(nn * 128, nk * 128)[:N, :K], (e + 127).to(torch.uint8).t().contiguous()


def _values(q, scale):
    """The fp32 values of a block8 tensor [M, D]."""
    s = _power(scale.int() - 127).t().repeat_interleave(128, 1)
    return q.float() * s[:, :q.shape[1]]


def _weight_values(q, scale):
    s = _power(scale.int() - 127).t().repeat_interleave(128, 0).repeat_interleave(128, 1)
    return q.float() * s[:q.shape[0], :q.shape[1]]


def _held(q, scale):
    """A block8 tensor as a program keeps it: rows on 16-byte boundaries."""
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


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    def rows(M, D, std, dtype, pad=0):
        """Rows of different size, some columns much larger, as activations and their gradients have them."""
        buf = torch.zeros((M, D + pad), dtype=TORCH[dtype], device=DEV)
        x = normal(M, D) * torch.exp(0.5 * normal(M, 1)) * torch.exp(0.7 * normal(1, D)) * std
        buf[:, :D] = x
        return buf[:, :D]

    def empty(M, D, dtype, pad=0):
        return torch.empty((M, D + pad), dtype=TORCH[dtype], device=DEV)[:, :D]

    c, kind, M = dict(case), case["kind"], case["M"]
    s = dict(case=c, held={})
    D, pad = case.get("D"), case.get("pad", 0)
    if kind in ("ln_fwd", "ln_bwd"):
        s["g"], s["b"] = 1 + 0.1 * normal(D), 0.02 * normal(D)
        s["mean"], s["rstd"] = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    if kind == "ln_fwd":
        s["x"] = rows(M, D, 1.0, c["x"], pad)
        s["y"] = empty(M, D, c["y"], pad) if c["y"] else None
        s["y8"] = _empty8(M, D) if c["y8"] else None
        s["x8"] = _empty8(M, D) if c["x8"] else None
    elif kind == "ln_bwd":
        x = rows(M, D, 1.0, "bf16" if c["x"] == "bf16" else "f32", pad)
        mean = x.float().mean(1)
        s["mean"] = mean
        s["rstd"] = torch.rsqrt((x.float() - mean[:, None]).square().mean(1) + EPS)
        s["x"], s["x8"] = (x, None) if c["x"] != "block8" else (None, _held(*_pack(x)))
        s["dy"] = rows(M, D, 1e-3, c["dy"], pad)
        s["dres"] = rows(M, D, 1e-3, "f32") if c["dres"] else None
        s["dx"] = empty(M, D, c["dx"], pad)
        s["dg"], s["db"] = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    elif kind == "save":
        s["x"], s["x8"] = rows(M, D, 1.0, c["x"], pad), _empty8(M, D)
    elif kind == "load":
        s["x8"], s["x"] = _held(*_pack(rows(M, D, 1.0, "f32"))), empty(M, D, c["x"], pad)
    elif kind == "gelu_bwd":
        s["da"] = rows(M, D, 1e-3, c["da"], pad)
        s["u8"] = _held(*_pack(rows(M, D, 0.7, "f32")))
        s["du"] = empty(M, D, c["du"], pad) if c["du"] else None
        s["du8"] = _empty8(M, D) if c["du8"] else None
        s["db"] = torch.empty(D, device=DEV)
    elif kind == "linear":
        N, K = c["N"], c["K"]
        s["a8"] = _held(*_pack(rows(M, K, 0.5, "f32")))
        s["w8"] = _held(*_pack_weight(0.02 * normal(N, K)))
        s["bias"] = 0.02 * normal(N)
        s["residual"] = rows(M, N, 1.0, "f32") if c["epi"] == "residual" else None
        s["out"] = empty(M, N, c["out"]) if c["out"] != "block8" else None
        s["out8"] = _empty8(M, N) if c["out"] == "block8" else None
        s["u8"] = _empty8(M, N) if c["u8"] else None
    else:
        N, K = c["N"], c["K"]
        s["dy"] = rows(M, N, 1e-3, "bf16")
        s["x8"] = _held(*_pack(rows(M, K, 1.0, "f32")))
        s["dw"] = torch.empty((N, K), device=DEV)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _gelu(x):
    return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))


def _gelu_grad(x):
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))


def _out8(x):
    q, scale = _pack(x)
    return dict(q=q, scale=scale.view(torch.float8_e8m0fnu))


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
        y = d * rstd * s["g"] + s["b"]
        return dict(y=y.to(TORCH[c["y"]]) if c["y"] else None, y8=_out8(y) if c["y8"] else None,
                    x8=_out8(x) if c["x8"] else None, mean=mean[:, 0], rstd=rstd[:, 0])
    if kind == "ln_bwd":
        D = c["D"]
        x = s["x"].float() if s["x"] is not None else _values(s["x8"][0][:, :D].view(torch.float8_e4m3fn), s["x8"][1])
        dy = s["dy"].float()
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        a = dy * s["g"]
        dx = (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["dres"] is not None:
            dx = dx + s["dres"]
        return dict(dx=dx.to(TORCH[c["dx"]]), dg=(dy * xh).sum(0), db=dy.sum(0))
    if kind == "save":
        return _out8(s["x"].float())
    if kind == "load":
        return _values(s["x8"][0][:, :c["D"]].view(torch.float8_e4m3fn), s["x8"][1]).to(TORCH[c["x"]])
    if kind == "gelu_bwd":
        u = _values(s["u8"][0][:, :c["D"]].view(torch.float8_e4m3fn), s["u8"][1])
        du = s["da"].float() * _gelu_grad(u)
        return dict(du=du.to(TORCH[c["du"]]) if c["du"] else None, du8=_out8(du) if c["du8"] else None, db=du.sum(0))
    if kind == "linear":
        a = _values(s["a8"][0][:, :c["K"]].view(torch.float8_e4m3fn), s["a8"][1])
        w = _weight_values(s["w8"][0][:, :c["K"]].view(torch.float8_e4m3fn), s["w8"][1])
        u = a @ w.t() + s["bias"]
        y = _gelu(u) if c["epi"] == "gelu" else u + s["residual"] if c["epi"] == "residual" else u
        return dict(out=_out8(y) if c["out"] == "block8" else y.to(TORCH[c["out"]]), u8=_out8(u) if c["u8"] else None)
    x = _values(s["x8"][0][:, :c["K"]].view(torch.float8_e4m3fn), s["x8"][1])
    return dict(dw=s["dy"].float().t() @ x)


LM_EPI = {"bias": "LAZYMAR_EPI_BIAS", "gelu": "LAZYMAR_EPI_GELU", "residual": "LAZYMAR_EPI_RESIDUAL"}


def _plan(s):
    """What a program keeps between calls: descriptors of its 8-bit buffers and a workspace."""
    from paper_2503_12450_gb300 import lazymar as lm

    c, kind = s["case"], s["case"]["kind"]
    p = dict(lm=lm)
    for k in ("x8", "y8", "u8", "du8", "a8", "w8", "out8"):
        p[k] = lm.lazymar_block8(*s[k]) if s.get(k) is not None else None
    size = 0
    if kind == "ln_bwd":
        size = lm.lazymar_layernorm_backward_workspace(c["M"], c["D"])
    elif kind == "gelu_bwd":
        size = lm.lazymar_block8_gelu_backward_workspace(c["M"], c["D"])
    elif kind == "wgrad":
        size = lm.lazymar_block8_wgrad_workspace(c["M"], c["N"], c["K"])
    p["ws"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
    for k in ("x", "y", "dy", "dx", "da", "du"):
        if c.get(k) in TORCH:
            p[k] = {"f32": lm.LAZYMAR_F32, "bf16": lm.LAZYMAR_BF16}[c[k]]
    p["out"] = lm.LAZYMAR_BF16 if c.get("out") == "bf16" else lm.LAZYMAR_F32
    p["epi"] = getattr(lm, LM_EPI[c["epi"]]) if "epi" in c else 0
    return p


def _ld(t):
    return t.stride(0) if t is not None else 0


def _own(s):
    c, kind = s["case"], s["case"]["kind"]
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    lm, M = p["lm"], c["M"]
    if kind == "ln_fwd":
        x, y = s["x"], s["y"]
        lm.lazymar_layernorm_forward(p["x"], x, _ld(x), s["g"], s["b"], p.get("y", 0), y, _ld(y), p["y8"], p["x8"],
                                     s["mean"], s["rstd"], M, c["D"], EPS)
        return dict(y=y, y8=_e4m3(s["y8"], c["D"]) if c["y8"] else None, x8=_e4m3(s["x8"], c["D"]) if c["x8"] else None,
                    mean=s["mean"], rstd=s["rstd"])
    if kind == "ln_bwd":
        x, dy, dx, dres = s["x"], s["dy"], s["dx"], s["dres"]
        lm.lazymar_layernorm_backward(p["dy"], dy, _ld(dy), p.get("x", 0), x, _ld(x), p["x8"], s["mean"], s["rstd"],
                                      s["g"], dres, _ld(dres), p["dx"], dx, _ld(dx), s["dg"], s["db"], False, M,
                                      c["D"], p["ws"], p["ws"].numel())
        return dict(dx=dx, dg=s["dg"], db=s["db"])
    if kind == "save":
        lm.lazymar_block8_pack(p["x"], s["x"], _ld(s["x"]), p["x8"], M, c["D"])
        return _e4m3(s["x8"], c["D"])
    if kind == "load":
        lm.lazymar_block8_unpack(p["x8"], p["x"], s["x"], _ld(s["x"]), M, c["D"])
        return s["x"]
    if kind == "gelu_bwd":
        da, du = s["da"], s["du"]
        lm.lazymar_block8_gelu_backward(p["da"], da, _ld(da), p["u8"], p.get("du", 0), du, _ld(du), p["du8"], s["db"],
                                        False, M, c["D"], p["ws"], p["ws"].numel())
        return dict(du=du, du8=_e4m3(s["du8"], c["D"]) if c["du8"] else None, db=s["db"])
    if kind == "linear":
        out, res = s["out"], s["residual"]
        lm.lazymar_block8_linear(p["epi"], p["a8"], p["w8"], s["bias"], res, _ld(res), p["out"], out, _ld(out),
                                 p["out8"], p["u8"], M, c["N"], c["K"])
        return dict(out=_e4m3(s["out8"], c["N"]) if c["out"] == "block8" else out,
                    u8=_e4m3(s["u8"], c["N"]) if c["u8"] else None)
    lm.lazymar_block8_wgrad(s["dy"], _ld(s["dy"]), p["x8"], s["dw"], c["K"], False, M, c["N"], c["K"], p["ws"],
                            p["ws"].numel())
    return dict(dw=s["dw"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "bf16": 2, "block8": 1 + 1 / 128, "": 0}
    c, kind, M = case, case["kind"], case["M"]
    e8 = size["block8"]
    if kind == "ln_fwd":
        n = M * c["D"]
        return dict(bytes=n * (size[c["x"]] + size[c["y"]] + e8 * (c["y8"] + c["x8"])) + 8 * M + 8 * c["D"],
                    flops=8 * n)
    if kind == "ln_bwd":
        n = M * c["D"]
        return dict(bytes=n * (size[c["x"]] + size[c["dy"]] + size[c["dx"]] + 4 * c["dres"]) + 8 * M + 12 * c["D"],
                    flops=14 * n)
    if kind == "save" or kind == "load":
        n = M * c["D"]
        return dict(bytes=n * (size[c["x"]] + e8), flops=2 * n)
    if kind == "gelu_bwd":
        n = M * c["D"]
        return dict(bytes=n * (size[c["da"]] + e8 + size[c["du"]] + e8 * c["du8"]) + 4 * c["D"], flops=20 * n)
    N, K = c["N"], c["K"]
    if kind == "linear":
        out = M * N * (size[c["out"]] + e8 * c["u8"] + 4 * (c["epi"] == "residual"))
        return dict(bytes=M * K * e8 + N * K + out + 4 * N, flops=2.0 * M * N * K)
    return dict(bytes=2 * M * N + M * K * e8 + 4 * N * K, flops=2.0 * M * N * K)


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _wide(held, D):
    """A held tensor's values from its bytes: sign, four exponent and three mantissa bits, and the block's scale."""
    b = held[0][:, :D].int()
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * _two(e - 7))
    v = torch.where((b & 0x7F) == 0x7F, float("nan"), v) * (1 - 2 * (b >> 7).double())
    block = torch.arange(D, device=DEV) // 128
    return v, block


def _exact_rows(held, D):
    v, block = _wide(held, D)
    return v * _two(held[1].int() - 127)[block].t()


def _exact_weight(held, K):
    v, block = _wide(held, K)
    rows = torch.arange(v.shape[0], device=DEV) // 128
    return v * _two(held[1].int() - 127)[block][:, rows].t()


def _exact8(x):
    """x in 64 bits rounded to block8: the E4M3 values and the scales."""
    M, D = x.shape
    nb = (D + 127) // 128
    big = torch.stack([x[:, 128 * j:128 * j + 128].abs().amax(1) for j in range(nb)], 1)
    e = torch.ceil(torch.log2(big.clamp(min=2.0 ** -200) / 448)) - 1  # or one more: log2 rounds
    e = torch.where(big <= 448 * _two(e), e, e + 1).clamp(min=-126)
    v = x / _two(e)[:, torch.arange(D, device=DEV) // 128]
    step = _two(torch.frexp(v.abs().clamp(min=2.0 ** -6))[1] - 4)  # of three mantissa bits
    return dict(q=torch.round(v / step) * step, scale=_two(e).t())


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "ln_fwd":
        x = s["x"].double()
        mean = x.sum(1) / c["D"]
        rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / c["D"] + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * s["g"].double() + s["b"].double()
        return dict(y=y if c["y"] else None, y8=_exact8(y) if c["y8"] else None, x8=_exact8(x) if c["x8"] else None,
                    mean=mean, rstd=rstd)
    if kind == "ln_bwd":
        x = s["x"].double() if s["x"] is not None else _exact_rows(s["x8"], c["D"])
        dy, g = s["dy"].double(), s["g"].double()
        xh = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        m1 = (dy * g).sum(1, keepdim=True) / c["D"]
        m2 = (dy * g * xh).sum(1, keepdim=True) / c["D"]
        dx = s["rstd"].double()[:, None] * (dy * g - m1 - xh * m2)
        return dict(dx=dx + s["dres"].double() if s["dres"] is not None else dx, dg=(dy * xh).sum(0), db=dy.sum(0))
    if kind == "save":
        return _exact8(s["x"].double())
    if kind == "load":
        return _exact_rows(s["x8"], c["D"])
    if kind == "gelu_bwd":
        u = _exact_rows(s["u8"], c["D"])
        phi = torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
        du = s["da"].double() * (0.5 * torch.erfc(-u / math.sqrt(2)) + u * phi)
        return dict(du=du if c["du"] else None, du8=_exact8(du) if c["du8"] else None, db=du.sum(0))
    if kind == "linear":
        u = _exact_rows(s["a8"], c["K"]) @ _exact_weight(s["w8"], c["K"]).t() + s["bias"].double()
        y = u
        if c["epi"] == "gelu":
            y = 0.5 * u * torch.erfc(-u / math.sqrt(2))
        elif c["epi"] == "residual":
            y = s["residual"].double() + u
        return dict(out=_exact8(y) if c["out"] == "block8" else y, u8=_exact8(u) if c["u8"] else None)
    return dict(dw=s["dy"].double().t() @ _exact_rows(s["x8"], c["K"]))
