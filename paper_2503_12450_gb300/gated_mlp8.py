"""A stack of modulated, gated MLP blocks with 8-bit activations, for training and serving:

    x <- x + gate (W2 GELU(W1 (LN(x) (1 + scale) + shift) + b1) + b2)

with a shift, a scale and a gate for each block, given for each row or for each group of rows (the form of the
diffusion head's blocks and of transformers whose norms a condition modulates). What stands between two products of
neighbouring blocks, the gate, the residual addition and the next block's modulated norm, is one pass over the rows
(lazymar_join, lazymar_join_grad). Kept for the backward pass are four 8-bit tensors a block and row: the stream and the
branch's output behind it, and GELU's input and output; and the norm's output in front.
"""
import torch

from . import lazymar as lm
from . import mlp_block8
from .mlp_block8 import BF16, F32, Tensor8, _row_stride

LAYER = lm.LAZYMAR_NORM_LAYER


class GatedMlpStack8:
    """blocks: a list of dicts of fp32 tensors w1 [H, D], b1 [H], w2 [D, H], b2 [D], the same
    H and D in all, used where they are if they are contiguous.
    `p` and `grads` hold them all under names "0.w1" and so on. One stream at a time. Buffers are those of one number of
    rows; another number replaces them, except for those that a captured pass has used, which the object keeps."""

    def __init__(self, blocks, eps=1e-6):
        if not blocks or blocks[0]["w1"].dim() != 2:
            raise lm.LazymarError(1, "blocks: one at least, w1 [H, D]")
        H, D = blocks[0]["w1"].shape
        for i, b in enumerate(blocks):
            for k, shape in (("w1", (H, D)), ("b1", (H,)), ("w2", (D, H)), ("b2", (D,))):
                if tuple(b[k].shape) != shape:
                    raise lm.LazymarError(1, "blocks: %d.%s %s required, as the first block's w1 says" % (i, k, list(shape)))
        self.p = {"%d.%s" % (i, k): b[k].detach().float().contiguous() for i, b in enumerate(blocks) for k in ("w1", "b1", "w2", "b2")}
        self.grads = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.depth, self.eps = len(blocks), eps
        self.H, self.D = H, D
        dev = self.p["0.w1"].device
        self.w8 = [dict(w1=Tensor8(self.H, self.D, dev, True), w1t=Tensor8(self.D, self.H, dev, True),
                        w2=Tensor8(self.D, self.H, dev, True), w2t=Tensor8(self.H, self.D, dev, True)) for _ in blocks]
        self.kept = None  # rows, group and modulation of the forward pass that backward() belongs to
        self.rows = self.serving_rows = None
        self.captured = []  # buffers that graphs write to
        self.pack()

    def pack(self):
        """The weights' 8-bit copies, after the weights have changed."""
        for i, w in enumerate(self.w8):
            lm.lazymar_block8_pack_weight(F32, self.p["%d.w1" % i], self.D, w["w1"].d, w["w1t"].d, self.H, self.D)
            lm.lazymar_block8_pack_weight(F32, self.p["%d.w2" % i], self.H, w["w2"].d, w["w2t"].d, self.D, self.H)

    def _modulation(self, mod, M, group):
        """Views (shift, scale, gate) of each block of mod [rows of it, 3 D depth], fp32 or bf16."""
        D, rows = self.D, (-(-M // group) if group else 1)
        if mod.dim() != 2 or tuple(mod.shape) != (rows, 3 * D * self.depth):
            raise lm.LazymarError(1, "mod: [%d, %d] required" % (rows, 3 * D * self.depth))
        return [tuple(mod[:, (3 * i + j) * D:(3 * i + j + 1) * D] for j in range(3)) for i in range(self.depth)]

    def _keep(self, M, dev):
        if M == self.rows:
            return
        D, H = self.D, self.H
        self.x8 = Tensor8(M, D, dev)
        self.k = [dict(h=Tensor8(M, D, dev), u=Tensor8(M, H, dev), a=Tensor8(M, H, dev), y=Tensor8(M, D, dev), z=Tensor8(M, D, dev),
                       mean=torch.empty(M, device=dev), rstd=torch.empty(M, device=dev)) for _ in range(self.depth)]
        self.dy8, self.du8 = Tensor8(M, D, dev), Tensor8(M, H, dev)
        self.rows = M

    def _serve(self, M, dev):
        if M != self.serving_rows:
            self.hs, self.a_s = Tensor8(M, self.D, dev), Tensor8(M, self.H, dev)
            self.serving_rows = M

    def _hold(self, x, train):
        """Keeps the buffers of a captured pass."""
        if mlp_block8.capturing(x):
            self.captured.append((self.x8, self.k, self.dy8, self.du8) if train else (self.hs, self.a_s))

    def forward(self, x, mod, group=0, train=True):
        """x [M, D] fp32; mod [ceil(M / group), 3 D depth] (group 0: one row for all), each block's shift, scale and gate in
        turn. Returns the stream after the last block, [M, D] fp32. Without `train` nothing is kept."""
        _row_stride(x, self.D, "x")
        M, D, H, dev = x.shape[0], self.D, self.H, x.device
        parts = self._modulation(mod, M, group)
        z = torch.empty((M, D), device=dev)
        y = torch.empty((M, -(-D // 8) * 8), dtype=torch.bfloat16, device=dev)
        if train:
            self.kept = None
            self._keep(M, dev)
        else:
            self._serve(M, dev)
        rows = lambda t: lm.lazymar_rows(t.q, t.scale)  # noqa: E731
        stream = x
        for i in range(self.depth + 1):
            # behind block i - 1 and in front of block i
            a = dict(group=group)
            if i > 0:
                a.update(y=y[:, :D], gate=parts[i - 1][2], z=z)
                if train:
                    a.update(y8=rows(self.k[i - 1]["y"]), z8=rows(self.k[i - 1]["z"]))
            elif train:
                a.update(z8=rows(self.x8))
            if i < self.depth:
                h8 = self.k[i]["h"] if train else self.hs
                a.update(pre=LAYER, eps=self.eps, shift=parts[i][0], scale=parts[i][1], h8=rows(h8))
                if train:
                    a.update(z_mean=self.k[i]["mean"], z_rstd=self.k[i]["rstd"])
            lm.lazymar_join(lm.lazymar_join_args(M, D, stream, **a))
            if i == self.depth:
                break
            stream = z if i > 0 else x
            a8, w = (self.k[i]["a"] if train else self.a_s), self.w8[i]
            lm.lazymar_block8_linear(lm.LAZYMAR_EPI_GELU, h8.d, w["w1"].d, self.p["%d.b1" % i], None, 0, F32, None, 0, a8.d,
                                     self.k[i]["u"].d if train else None, M, H, D)
            lm.lazymar_block8_linear(lm.LAZYMAR_EPI_BIAS, a8.d, w["w2"].d, self.p["%d.b2" % i], None, 0, BF16, y, y.stride(0), None,
                                     None, M, D, H)
        if train:
            self.kept = (M, group, mod)
        self._hold(x, train)
        return z

    def backward(self, dz, accumulate=False):
        """dz [M, D] fp32, of the last forward pass with `train`. Returns dx [M, D] fp32 and the modulation's gradient in
        mod's shape and type, and leaves (or adds) the parameters' gradients."""
        if self.kept is None:
            raise lm.LazymarError(1, "backward() needs a forward pass with train=True")
        M, group, mod = self.kept
        if tuple(dz.shape) != (M, self.D):
            raise lm.LazymarError(1, "dz: [%d, %d], as the forward pass's rows" % (M, self.D))
        _row_stride(dz, self.D, "dz")
        self._hold(dz, True)
        D, H, dev, g = self.D, self.H, dz.device, self.grads
        parts, dmod = self._modulation(mod, M, group), torch.empty_like(mod, memory_format=torch.contiguous_format)
        dparts = self._modulation(dmod, M, group)
        size = max([lm.lazymar_join_grad_workspace(M, D, group), lm.lazymar_join_grad_workspace(M, D, 0),
                    lm.lazymar_block8_gelu_backward_workspace(M, H),
                    lm.lazymar_block8_wgrad_workspace(M, H, D), lm.lazymar_block8_wgrad_workspace(M, D, H), 16])
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
        wide = lambda n: torch.empty((M, -(-n // 8) * 8), dtype=torch.bfloat16, device=dev)  # noqa: E731
        dy, da, dh = wide(D), wide(H), wide(D)
        ldd, ldh = dy.stride(0), da.stride(0)
        dx = torch.empty((M, D), device=dev)
        rows = lambda t: lm.lazymar_rows(t.q, t.scale)  # noqa: E731
        for i in range(self.depth, -1, -1):
            # through what stands behind block i - 1 and in front of block i
            a = dict(group=group, workspace=ws, dz=dz if i == self.depth else dx, dx=dx)
            if i < self.depth:
                a.update(pre=LAYER, dh=dh[:, :D], z=rows(self.k[i - 1]["z"] if i > 0 else self.x8), scale=parts[i][1],
                         z_mean=self.k[i]["mean"], z_rstd=self.k[i]["rstd"], dshift=dparts[i][0], dscale=dparts[i][1])
            if i > 0:
                a.update(y=rows(self.k[i - 1]["y"]), gate=parts[i - 1][2], dgate=dparts[i - 1][2], dy=dy[:, :D], dy8=rows(self.dy8))
            lm.lazymar_join_grad(lm.lazymar_join_grad_args(M, D, **a))
            if i == 0:
                break
            b, k, w, n = i - 1, self.k[i - 1], self.w8[i - 1], ws.numel()
            # the bias gradient in a call of its own, because `accumulate` is for the parameters and not for dmod
            lm.lazymar_join_grad(lm.lazymar_join_grad_args(M, D, dz=dy[:, :D], dpost_b=g["%d.b2" % b], accumulate=accumulate,
                                                           workspace=ws))
            lm.lazymar_block8_wgrad(dy, ldd, k["a"].d, g["%d.w2" % b], H, accumulate, M, D, H, ws, n)
            lm.lazymar_block8_linear(lm.LAZYMAR_EPI_BIAS, self.dy8.d, w["w2t"].d, None, None, 0, BF16, da, ldh, None, None, M, H, D)
            lm.lazymar_block8_gelu_backward(BF16, da, ldh, k["u"].d, BF16, da, ldh, self.du8.d, g["%d.b1" % b], accumulate, M, H, ws, n)
            lm.lazymar_block8_wgrad(da, ldh, k["h"].d, g["%d.w1" % b], D, accumulate, M, H, D, ws, n)
            lm.lazymar_block8_linear(lm.LAZYMAR_EPI_BIAS, self.du8.d, w["w1t"].d, None, None, 0, BF16, dh, ldd, None, None, M, D, H)
        return dx, dmod
