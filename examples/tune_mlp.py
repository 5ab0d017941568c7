"""Tunes the MLP half of a transformer block with 8-bit activations: a student
whose weights were disturbed learns a teacher's outputs again.

    python examples/tune_mlp.py [--width 1024] [--rows 20480] [--steps 30]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_12450_gb300 import lazymar as lm  # noqa: E402
from paper_2503_12450_gb300.mlp_block8 import MlpBlock8  # noqa: E402


def random_params(D, H, seed, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    n = lambda *s: torch.randn(s, device=device, generator=g)  # noqa: E731
    return dict(ln_g=1 + 0.1 * n(D), ln_b=0.02 * n(D), w1=n(H, D) / D ** 0.5, b1=0.02 * n(H), w2=n(D, H) / H ** 0.5,
                b2=0.02 * n(D))


def tune(width, rows, steps, mlp_ratio=4, seed=0):
    """Returns the losses, the student and the milliseconds of a step."""
    lr = 0.03 / width ** 0.5  # a tenth of the disturbance
    teacher = MlpBlock8(random_params(width, mlp_ratio * width, seed))
    noise = random_params(width, mlp_ratio * width, seed + 1)
    student = MlpBlock8({k: v + 0.3 * noise[k] if k.startswith("w") else v.clone() for k, v in teacher.p.items()})
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    opt = torch.optim.Adam(list(student.p.values()), lr=lr)
    for k, v in student.p.items():
        v.grad = student.grads[k]
    losses, a, b = [], torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i in range(steps):
        x = torch.randn((rows, width), device="cuda", generator=g)
        target = teacher.forward(x, train=False)
        if i == steps - 1:
            a.record()
        y = student.forward(x)
        d = y - target
        losses.append((d * d).mean())
        student.backward(d * (1.0 / rows))
        opt.step()
        student.pack()
        if i == steps - 1:
            b.record()
    torch.cuda.synchronize()
    lm.lazymar_device_check()
    return [float(v) for v in losses], student, a.elapsed_time(b)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--rows", type=int, default=20480)
    ap.add_argument("--steps", type=int, default=30)
    c = ap.parse_args()
    losses, student, ms = tune(c.width, c.rows, c.steps)
    for i in range(0, c.steps, max(1, c.steps // 10)):
        print("step %3d  loss %.5f" % (i, losses[i]))
    print("step %3d  loss %.5f  %.2f ms a step" % (c.steps - 1, losses[-1], ms))
    kept = student.saved_bytes()
    print("kept for the backward pass: %.1f MB in 8 bits (bf16: %.1f MB)" % (
        kept / 1e6, 4 * c.rows * (student.D + student.H) / 1e6))


if __name__ == "__main__":
    main()
