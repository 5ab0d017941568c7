"""The stack of gated MLP blocks without a GPU: what it refuses, against a library that is not called."""
import pytest

from paper_2503_12450_gb300 import lazymar as lm
from test_optim_host import calls  # noqa: F401

torch = pytest.importorskip("torch")


def _block(D=16, H=32, **other):
    b = dict(w1=torch.zeros(H, D), b1=torch.zeros(H), w2=torch.zeros(D, H), b2=torch.zeros(D))
    return dict(b, **{k: torch.zeros(s) for k, s in other.items()})


def test_blocks_of_other_sizes_are_refused(calls):  # noqa: F811
    """They would be read beyond their ends, under the first block's sizes."""
    from paper_2503_12450_gb300.gated_mlp8 import GatedMlpStack8
    good = _block()
    for bad in (_block(H=24), _block(D=8), _block(b1=(31,)), _block(b2=(8,)), _block(w2=(32, 16)), _block(b1=(32, 1))):
        with pytest.raises(lm.LazymarError, match="blocks"):
            GatedMlpStack8([good, bad])
    for bad in (_block(w1=(32,)), _block(w2=(16, 31)), _block(b1=(16,))):
        with pytest.raises(lm.LazymarError, match="blocks"):
            GatedMlpStack8([bad])
    with pytest.raises(lm.LazymarError, match="blocks"):
        GatedMlpStack8([])
    assert not calls
    s = GatedMlpStack8([good, _block()])
    assert (s.D, s.H, s.depth) == (16, 32, 2) and calls == ["lazymar_block8_pack_weight"] * 4


@pytest.mark.parametrize("gated", [True, False])
def test_buffers_of_a_captured_pass_live_on(calls, monkeypatch, gated):  # noqa: F811
    """A graph writes to the buffers of its own number of rows; a pass with another number must not give them back to the
    allocator while the object lives."""
    import gc
    import weakref

    from paper_2503_12450_gb300 import gated_mlp8, mlp_block8
    if gated:
        s, mod = gated_mlp8.GatedMlpStack8([_block(), _block()]), torch.zeros(1, 3 * 16 * 2)
        forward = lambda M, train: s.forward(torch.zeros(M, 16), mod, train=train)  # noqa: E731
        kept = lambda: [s.x8.q, s.k[1]["z"].q, s.k[0]["mean"], s.dy8.q, s.du8.scale]  # noqa: E731
        served = lambda: [s.hs.q, s.a_s.scale]  # noqa: E731
    else:
        s = mlp_block8.MlpBlock8(dict(_block(), ln_g=torch.ones(16), ln_b=torch.zeros(16)))
        forward = lambda M, train: s.forward(torch.zeros(M, 16), train=train)  # noqa: E731
        kept = lambda: [s.x8.q, s.a8.scale, s.mean, s.ws, s.du8.q]  # noqa: E731
        served = lambda: [s.h8s.q, s.a8s.scale]  # noqa: E731
    for train, of, captured, step in ((True, kept, False, forward), (True, kept, True, forward), (False, served, False, forward),
                                      (False, served, True, forward), (True, kept, True, lambda M, train: s.backward(torch.zeros(M, 16)))):
        monkeypatch.setattr(mlp_block8, "capturing", lambda x: False)
        forward(4, train)
        monkeypatch.setattr(mlp_block8, "capturing", lambda x: captured)
        step(4, train)
        old = [weakref.ref(t) for t in of()]
        monkeypatch.setattr(mlp_block8, "capturing", lambda x: False)
        forward(6, train)
        gc.collect()
        assert all((r() is not None) == captured for r in old)
