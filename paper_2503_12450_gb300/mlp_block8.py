"""The MLP half of a transformer block with 8-bit activations, for training and
serving: y = x + W2 GELU(W1 LN(x) + b1) + b2 on the library's training operators.

Kept for the backward pass are the block's input, the LayerNorm's output and
GELU's input and output, each as E4M3 bytes with one scale per 128 columns: 2 D +
2 H bytes a token instead of 4 D + 4 H in bf16. Weights are fp32; their 8-bit copies
(and the transposed ones that the input gradients need) are packed after each
update by pack(). PyTorch holds the memory; adamw.AdamW or one of its optimizers updates the
weights. Every product and row-wise pass runs in liblazymar.so.
"""
import torch

from . import lazymar as lm

F32, BF16 = lm.LAZYMAR_F32, lm.LAZYMAR_BF16


class Tensor8:
    """An 8-bit tensor [rows, cols] with a scale for each row and 128 columns (weight: for each 128 x 128 block)."""

    def __init__(self, rows, cols, device, weight=False):
        self.q = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device)
        self.scale = torch.empty((-(-cols // 128), -(-rows // 128) if weight else rows), dtype=torch.uint8, device=device)
        self.d = lm.lazymar_block8(self.q, self.scale)

    def bytes(self):
        return self.q.numel() + self.scale.numel()


def capturing(x):
    """Whether a pass over x is being captured into a graph."""
    return x.is_cuda and torch.cuda.is_current_stream_capturing()


def _row_stride(t, cols, name):
    """The stride of fp32 rows of `cols` consecutive elements; refuses anything else."""
    if t.dim() != 2 or t.shape[1] != cols or t.dtype != torch.float32 or (cols > 1 and t.stride(1) != 1):
        raise lm.LazymarError(1, "%s: fp32 [rows, %d] with consecutive columns required" % (name, cols))
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), cols)


class MlpBlock8:
    """Parameters and gradients: dicts of fp32 tensors ln_g, ln_b [D], w1 [H, D], b1 [H], w2 [D, H], b2 [D]. Contiguous
    fp32 parameters are used where they are, not copied: an optimizer over them, or over `p`, updates both. An object
    has one workspace and belongs to one stream at a time. Buffers are those of one number of rows; another number
    replaces them, except for those that a captured pass has used, which the object keeps."""

    def __init__(self, params, eps=1e-6):
        self.p = {k: v.detach().float().contiguous() for k, v in params.items()}
        self.H, self.D = self.p["w1"].shape
        self.eps = eps
        dev = self.p["w1"].device
        self.grads = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.w1, self.w1t = Tensor8(self.H, self.D, dev, True), Tensor8(self.D, self.H, dev, True)
        self.w2, self.w2t = Tensor8(self.D, self.H, dev, True), Tensor8(self.H, self.D, dev, True)
        self.rows = self.serving_rows = None  # of the buffers for training, for serving
        self.captured = []  # buffers that graphs write to
        self.kept = False  # whether a forward pass has left what backward() reads
        self.pack()

    def pack(self):
        """The weights' 8-bit copies, after the weights have changed."""
        D, H = self.D, self.H
        lm.lazymar_block8_pack_weight(F32, self.p["w1"], D, self.w1.d, self.w1t.d, H, D)
        lm.lazymar_block8_pack_weight(F32, self.p["w2"], H, self.w2.d, self.w2t.d, D, H)

    def _serving_buffers(self, M, dev):
        if M != self.serving_rows:
            self.h8s, self.a8s = Tensor8(M, self.D, dev), Tensor8(M, self.H, dev)
            self.serving_rows = M

    def _buffers(self, M, dev):
        if M == self.rows:
            return
        D, H = self.D, self.H
        self.x8, self.h8, self.dy8 = Tensor8(M, D, dev), Tensor8(M, D, dev), Tensor8(M, D, dev)
        self.u8, self.a8, self.du8 = Tensor8(M, H, dev), Tensor8(M, H, dev), Tensor8(M, H, dev)
        self.mean, self.rstd = torch.empty(M, device=dev), torch.empty(M, device=dev)
        size = max(lm.lazymar_layernorm_backward_workspace(M, D), lm.lazymar_block8_gelu_backward_workspace(M, H),
                   lm.lazymar_block8_gelu_backward_workspace(M, D), lm.lazymar_block8_wgrad_workspace(M, H, D),
                   lm.lazymar_block8_wgrad_workspace(M, D, H), 16)
        self.ws = torch.empty(size, dtype=torch.uint8, device=dev)
        self.rows = M

    def _hold(self, x, train):
        """Keeps the buffers of a captured pass."""
        if capturing(x):
            self.captured.append((self.x8, self.h8, self.dy8, self.u8, self.a8, self.du8, self.mean, self.rstd, self.ws) if train
                                 else (self.h8s, self.a8s))

    def saved_bytes(self):
        return sum(t.bytes() for t in (self.x8, self.h8, self.u8, self.a8))

    def forward(self, x, train=True):
        """x [M, D] fp32, the residual stream. Returns y [M, D] fp32. Without `train` nothing is kept, and what an
        earlier pass has kept stays."""
        ldx = _row_stride(x, self.D, "x")
        M, D, H = x.shape[0], self.D, self.H
        p, y = self.p, torch.empty((M, D), device=x.device)
        if train:
            self.kept = False
            self._buffers(M, x.device)
            h8, a8 = self.h8, self.a8
        else:
            self._serving_buffers(M, x.device)
            h8, a8 = self.h8s, self.a8s
        lm.lazymar_layernorm_forward(F32, x, ldx, p["ln_g"], p["ln_b"], F32, None, 0, h8.d,
                                     self.x8.d if train else None, self.mean if train else None,
                                     self.rstd if train else None, M, D, self.eps)
        lm.lazymar_block8_linear(lm.LAZYMAR_EPI_GELU, h8.d, self.w1.d, p["b1"], None, 0, F32, None, 0, a8.d,
                                 self.u8.d if train else None, M, H, D)
        lm.lazymar_block8_linear(lm.LAZYMAR_EPI_RESIDUAL, a8.d, self.w2.d, p["b2"], x, ldx, F32, y, D, None, None, M,
                                 D, H)
        self.kept = self.kept or train
        self._hold(x, train)
        return y

    def backward(self, dy, accumulate=False):
        """dy [M, D] fp32, of the last forward pass with `train`. Returns dx [M, D] fp32 and leaves (or adds) the
        parameters' gradients."""
        if not self.kept:
            raise lm.LazymarError(1, "backward() needs a forward pass with train=True")
        if tuple(dy.shape) != (self.rows, self.D):
            raise lm.LazymarError(1, "dy: [%d, %d], as the forward pass's rows" % (self.rows, self.D))
        lddy = _row_stride(dy, self.D, "dy")
        self._hold(dy, True)
        M, D, H = dy.shape[0], self.D, self.H
        g, ws, n, dev = self.grads, self.ws, self.ws.numel(), dy.device
        dyb = torch.empty((M, -(-D // 8) * 8), dtype=torch.bfloat16, device=dev)
        da = torch.empty((M, -(-H // 8) * 8), dtype=torch.bfloat16, device=dev)
        dh, dx = torch.empty_like(dyb), torch.empty((M, D), device=dev)
        ldd, ldh = dyb.stride(0), da.stride(0)
        lm.lazymar_block8_gelu_backward(F32, dy, lddy, None, BF16, dyb, ldd, self.dy8.d, g["b2"], accumulate, M,
                                        D, ws, n)
        lm.lazymar_block8_wgrad(dyb, ldd, self.a8.d, g["w2"], H, accumulate, M, D, H, ws, n)
        lm.lazymar_block8_linear(lm.LAZYMAR_EPI_BIAS, self.dy8.d, self.w2t.d, None, None, 0, BF16, da, ldh, None, None, M,
                                 H, D)
        lm.lazymar_block8_gelu_backward(BF16, da, ldh, self.u8.d, BF16, da, ldh, self.du8.d, g["b1"], accumulate, M, H, ws,
                                        n)
        lm.lazymar_block8_wgrad(da, ldh, self.h8.d, g["w1"], D, accumulate, M, H, D, ws, n)
        lm.lazymar_block8_linear(lm.LAZYMAR_EPI_BIAS, self.du8.d, self.w1t.d, None, None, 0, BF16, dh, ldd, None, None, M,
                                 D, H)
        lm.lazymar_layernorm_backward(BF16, dh, ldd, F32, None, 0, self.x8.d, self.mean, self.rstd, self.p["ln_g"], dy,
                                      lddy, F32, dx, D, g["ln_g"], g["ln_b"], accumulate, M, D, ws, n)
        return dx
