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
