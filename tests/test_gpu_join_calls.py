"""Calls of the residual join and its gradient that their documentation allows and that leave the usual
allocations: workspaces inside another, outputs that choose another kernel."""
import pytest

from paper_2503_12450_gb300 import lazymar as lm
from _gpu import torch_cuda
from test_gpu_join import Grad
from test_gpu_train import sync

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D,group", [(40, 8, 3), (700, 256, 5), (1000, 1280, 320), (500, 1024, 7), (300, 4096, 20), (90, 6000, 30),
                                       (300, 777, 9), (600, 512, 0), (600, 512, 1)])
def test_join_grad_in_a_workspace_between_boundaries_of_32_bytes(M, D, group):
    """A workspace may start on any boundary of 16 bytes: the same bits as on one of 256, nothing written around it."""
    torch = torch_cuda()
    g = Grad(M, D, group, "rms", "layer", seed=40).check()
    want = {k: t.clone() for k, t in g.o.items()}
    n = lm.lazymar_join_grad_workspace(M, D, group)
    for at in (16, 32, 48):
        room = torch.full((n + 256,), 0xC3, dtype=torch.uint8, device="cuda")
        assert room.data_ptr() % 64 == 0
        for t in g.o.values():
            t.fill_(float("nan"))
        lm.lazymar_join_grad(g.args(workspace=room[at:at + n]))
        sync()
        for k, t in g.o.items():
            assert torch.equal(t, want[k]), (at, k)
        assert (room[:at] == 0xC3).all() and (room[at + n:] == 0xC3).all()
