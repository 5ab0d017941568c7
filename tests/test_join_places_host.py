"""Outputs of the residual join in the place of others, or of inputs, by their 8-bit tensors' scales: refused before the device
is touched."""
import pytest

from paper_2503_12450_gb300 import lazymar as lm
from test_join_host import GRAD, JOIN, JOIN_GRAD, LAYER, RMS, X, _rows, lib  # noqa: F401

E8 = lambda p, scale, ld=16, lds=8: _rows(p, 2, ld, lds, scale)  # noqa: E731

JOINS = [
    (dict(y=_rows(256), y8=E8(512, 640), z8=E8(768, 640), **X), "one place"),
    (dict(pre=LAYER, h8=E8(512, 640), z8=E8(768, 640), **X), "one place"),
    (dict(pre=LAYER, h8=E8(512, 640), h=_rows(640), **X), "one place"),
    (dict(pre=LAYER, z8=E8(512, 640), z_mean=640, **X), "one place"),
    (dict(pre=LAYER, z8=E8(512, 512), **X), "one place"),
    (dict(y=E8(256, 640), y8=E8(512, 640), **X), "in place"),
    (dict(pre=LAYER, y=E8(256, 640), h8=E8(512, 640, lds=16), **X), "in place"),
    (dict(y=E8(256, 640), y8=E8(256, 640, lds=16), **X), "in place"),
    (dict(y=E8(256, 640), x=_rows(64), z=_rows(640)), "in place"),
    (dict(pre=LAYER, y=E8(256, 640), z_mean=640, **X), "in place"),
    (dict(y=_rows(256), gate=_rows(640), y8=E8(512, 640), **X), "in place"),
    (dict(pre=RMS, pre_g=640, h8=E8(512, 640), **X), "in place"),
    (dict(z8=E8(512, 64), **X), "in place"),
    (dict(y=E8(256, 640), z8=E8(512, 256), **X), "in place"),
]
GRADS = [
    (dict(y=E8(512, 640), dy8=E8(768, 640)), "in place"),
    (dict(z=E8(512, 640), dy8=E8(768, 640)), "in place"),
    (dict(y=E8(512, 640), dy8=E8(512, 640, lds=16)), "in place"),
    (dict(y=E8(512, 640), dy=_rows(640)), "in place"),
    (dict(z=E8(512, 640), dshift=_rows(640)), "in place"),
    (dict(dy8=E8(512, 256)), "one place"),
    (dict(dy8=E8(512, 640), dpre_g=640), "one place"),
    (dict(dy8=E8(512, 64)), "in place"),
    (dict(dy8=E8(512, 16)), "in place"),
    (dict(scale=_rows(768), dy8=E8(512, 768)), "in place"),
]


@pytest.mark.parametrize("fields,word", JOINS)
def test_join_scales_in_place_of_others(lib, fields, word):  # noqa: F811
    d = lm._filled(lm.lazymar_join_desc(), dict(dict(M=4, D=8, res=1.0, eps=1e-6), **fields))
    assert lib.lazymar_join(d.addr, None) == 1
    assert word in lib.lazymar_last_error().decode()


@pytest.mark.parametrize("fields,word", GRADS)
def test_join_grad_scales_in_place_of_others(lib, fields, word):  # noqa: F811
    d = lm._filled(lm.lazymar_join_grad_desc(), dict(dict(M=4, D=8, res=1.0, **GRAD), **fields))
    assert lib.lazymar_join_grad(d.addr, None) == 1
    assert word in lib.lazymar_last_error().decode()


@pytest.mark.parametrize("fields", [dict(y=E8(256, 640), y8=E8(256, 640), **X), dict(pre=LAYER, y=E8(256, 640), h8=E8(256, 640), **X),
                                    dict(y=E8(256, 640), y8=E8(256, 768), **X), dict(x=_rows(64, scale=640), z=_rows(128, scale=640)),
                                    dict(y=E8(256, 640), y8=E8(512, 768), z8=E8(1024, 1280), **X)])
def test_join_places_that_are_allowed(lib, fields):  # noqa: F811
    """An 8-bit output over y itself, bytes over y's with scales of their own, and a scale that no 8-bit tensor has."""
    d = lm._filled(lm.lazymar_join_desc(), dict(dict(M=4, D=8, res=1.0, eps=1e-6), **fields))
    assert lib.lazymar_join(d.addr, None) == 1  # (no device memory)
    assert "place" not in lib.lazymar_last_error().decode()
