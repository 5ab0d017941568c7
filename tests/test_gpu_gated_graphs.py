"""Captured passes of the MLP classes beside eager ones of another number of rows."""
import pytest

from _gpu import torch_cuda
from test_gpu_gated_stack import _blocks, _inputs, _stack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False])
def test_a_captured_step_outlives_passes_of_other_rows(gated):
    """Replayed after eager passes with other numbers of rows, and after the memory that these left was taken by others,
    a captured step gives what it gave, and leaves the others' memory alone."""
    torch = torch_cuda()
    D, H, M, group = 128, 512, 300, 50
    x, dz, mod = (torch.from_numpy(a).cuda() for a in _inputs(1, M, D, group, 20))
    other = [tuple(torch.from_numpy(a).cuda() for a in _inputs(1, n, D, group, 21)) for n in (500, 130)]
    if gated:
        s = _stack(_blocks(1, D, H, 22))
        forward = lambda x, mod, train=True: s.forward(x, mod, group, train)  # noqa: E731
    else:
        from paper_2503_12450_gb300.mlp_block8 import MlpBlock8
        b = {k: torch.from_numpy(v).cuda() for k, v in _blocks(1, D, H, 22)[0].items()}
        s = MlpBlock8(dict(b, ln_g=torch.ones(D, device="cuda"), ln_b=torch.zeros(D, device="cuda")))
        forward = lambda x, mod, train=True: s.forward(x, train)  # noqa: E731

    def step():
        forward(x, mod)
        return forward(x, mod, False), s.backward(dz)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            z, d = step()
        graph.replay()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    outputs = lambda: [z] + list(d if isinstance(d, tuple) else [d]) + list(s.grads.values())  # noqa: E731
    want = [t.clone() for t in outputs()]
    for x2, dz2, mod2 in other:
        forward(x2, mod2)
        forward(x2, mod2, False)
        s.backward(dz2)
    torch.cuda.synchronize()
    taken = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in (M * D, M * H, M * 4, M * 2 * D, 512) for _ in range(24)]
    for _ in range(3):
        for t in outputs():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    assert all((t == 0x5A).all() for t in taken)
