"""The residual join and the end of a training step without a GPU: the oracle's
gradients against differences, exports, and the argument checks that need no device."""
import ctypes
import math

import numpy as np
import pytest

from oracle import training as T
from paper_2503_12450_gb300 import build
from paper_2503_12450_gb300 import lazymar as lm

NONE, LAYER, RMS = lm.LAZYMAR_NORM_NONE, lm.LAZYMAR_NORM_LAYER, lm.LAZYMAR_NORM_RMS


@pytest.fixture(scope="module")
def lib():
    build.build()
    return lm.lib()


# --------------------------------------------------------------------------
# Oracle
# --------------------------------------------------------------------------

def _difference(f, x, h=1e-5):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        d[i] = (f(a) - f(b)) / (2 * h)
    return d


@pytest.mark.parametrize("post,pre,group", [("none", "layer", 2), ("layer", "rms", 0), ("rms", "layer", 1),
                                            ("layer", "none", 3), ("none", "rms", 5)])
def test_join_gradient_against_differences(post, pre, group):
    """Central differences of step 1e-5: an error of the third derivative times 1e-10 and of rounding 1e-16 / 1e-5."""
    r = np.random.default_rng(3)
    M, D = 5, 6
    G = -(-M // group) if group else 1
    n = r.standard_normal
    a = dict(x=n((M, D)), y=n((M, D)), gate=n((G, D)), post_g=1 + 0.1 * n(D), post_b=n(D))
    if pre != "none":
        a.update(scale=n((G, D)), shift=n((G, D)), pre_g=1 + 0.1 * n(D), pre_b=n(D))
    dh, dz = n((M, D)), n((M, D))
    kw = dict(post=post, pre=pre, group=group, res=0.7)

    def loss(a):
        o = T.join(**a, **kw)
        return float((o["z"] * dz).sum() + ((o["h"] * dh).sum() if pre != "none" else 0.0))
    o = T.join(**a, **kw)
    got = T.join_grad(dh if pre != "none" else None, dz, o["z"], a["y"], gate=a["gate"], scale=a.get("scale"),
                      post_g=a["post_g"], post_b=a["post_b"], pre_g=a.get("pre_g"), pre_b=a.get("pre_b"),
                      **{k: o.get(k) for k in ("y_mean", "y_rstd", "z_mean", "z_rstd")}, **kw)
    for k in a:
        want = _difference(lambda v: loss(dict(a, **{k: v})), a[k])
        np.testing.assert_allclose(got["d" + k], want, atol=2e-7, err_msg=k)


def test_join_with_nothing_is_the_residual_addition_and_a_layernorm():
    r = np.random.default_rng(4)
    x, y, g, b = r.standard_normal((3, 8)), r.standard_normal((3, 8)), r.standard_normal(8), r.standard_normal(8)
    o = T.join(x, y, pre="layer", pre_g=g, pre_b=b)
    np.testing.assert_array_equal(o["z"], x + y)
    np.testing.assert_allclose(o["h"], T.layernorm(x + y, g, b, 1e-6)[0], atol=1e-14)
    o = T.join(x, None, pre="rms")
    np.testing.assert_allclose((o["h"] ** 2).mean(1), 1.0, atol=1e-5)


def test_clip_factor_and_adamw_by_hand():
    assert T.clip_factor([[3.0], [4.0]], 1.0, 10.0) == (5.0, 1.0)
    assert T.clip_factor([[3.0], [4.0]], 1.0, 1.0) == (5.0, 0.2)
    assert T.clip_factor([[3.0], [4.0]], 2.0, 5.0) == (10.0, 1.0)
    assert T.clip_factor([[0.0]], 0.5, 1.0) == (0.0, 0.5)
    assert T.clip_factor([[np.inf]], 1.0, 1.0)[1] == 0.0 and T.clip_factor([[np.nan]], 1.0, 1.0)[1] == 0.0
    # the first step moves by lr whatever the gradient's size, and decays
    p, m, v = T.adamw([1e-3, -5.0], [1.0, 2.0], [0.0, 0.0], [0.0, 0.0], 1, 1.0, 0.01, 0.9, 0.99, 1e-12, 0.1)
    np.testing.assert_allclose(p, [1.0 - 0.001 - 0.01, 2.0 - 0.002 + 0.01], atol=1e-9)
    np.testing.assert_allclose(m, [1e-4, -0.5])
    np.testing.assert_allclose(v, [1e-8, 0.25])


# --------------------------------------------------------------------------
# Library
# --------------------------------------------------------------------------

def test_structs_have_the_layout_of_the_header(tmp_path):
    """Sizes and offsets of the binding's structs and of the compiler's."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pairs = [("lazymar_rows", lm.lazymar_rows_desc), ("lazymar_join_args", lm.lazymar_join_desc),
             ("lazymar_join_grad_args", lm.lazymar_join_grad_desc), ("lazymar_param", lm.lazymar_param),
             ("lazymar_adamw_args", lm.lazymar_adamw_desc)]
    body = "".join('printf("%%zu\\n", sizeof(%s));' % n + "".join(
        'printf("%%zu\\n", offsetof(%s, %s));' % (n, f) for f, _ in t._fields_) for n, t in pairs)
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stdio.h>\n#include "lazymar.h"\nint main(void) { %s return 0; }\n' % body)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)],
                   check=True, timeout=120)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, t in pairs:
        want += [ctypes.sizeof(t)] + [getattr(t, f).offset for f, _ in t._fields_]
    assert got == want


def _rows(p=64, dtype=0, ld=8, lds=8, scale=None):
    return lm.lazymar_rows_desc(p, scale, dtype, ld, lds)


X = dict(x=_rows(64), z=_rows(128))
JOIN = [
    (dict(M=-1, **X), 1, "M >= 0"),
    (dict(D=0, **X), 1, "D >= 1"),
    (dict(group=-1, **X), 1, "group"),
    (dict(post=3, **X), 1, "post and pre"),
    (dict(pre=-1, **X), 1, "post and pre"),
    (dict(eps=0.0, **X), 1, "eps"),
    (dict(eps=math.inf, **X), 1, "eps"),
    (dict(res=math.nan, **X), 1, "res"),
    (dict(D=8193, x=_rows(ld=8193), z=_rows(128, ld=8193)), 6, "8192"),
    (dict(M=(1 << 30) + 1, **X), 6, "2^30"),
    (dict(x=_rows()), 1, "no output"),
    (dict(z=_rows()), 1, "x:"),
    (dict(post=LAYER, **X), 1, "need y"),
    (dict(gate=_rows(256), **X), 1, "need y"),
    (dict(post_g=256, **X), 1, "need y"),
    (dict(y8=_rows(256, 2, 16, 8, 512), **X), 1, "need y"),
    (dict(y=_rows(256), y_mean=512, **X), 1, "need post"),
    (dict(h=_rows(256), **X), 1, "need pre"),
    (dict(scale=_rows(256), **X), 1, "need pre"),
    (dict(pre_b=256, **X), 1, "need pre"),
    (dict(z_rstd=256, **X), 1, "need pre"),
    (dict(pre=RMS, x=_rows(64), z=_rows(128), h=_rows(128)), 1, "one place"),
    (dict(y=_rows(256), y8=_rows(512, 2, 16, 8, 640), z8=_rows(512, 2, 16, 8, 640), **X), 1, "one place"),
    (dict(pre=LAYER, z_mean=256, z_rstd=256, **X), 1, "one place"),
    (dict(pre=LAYER, y=_rows(96, 2, 16, 8, 512), h8=_rows(96, 2, 32, 8, 512), **X), 1, "in place"),
    (dict(x=_rows(64), z=_rows(64, 1)), 1, "in place"),
    (dict(x=_rows(64), z=_rows(64, 0, 16)), 1, "in place"),
    (dict(x=_rows(64), y=_rows(96, 1), pre=RMS, h=_rows(96, 0)), 1, "in place"),
    (dict(x=_rows(64), y=_rows(96, 2, 16, 8, 512), z=_rows(96, 1, 16)), 1, "in place"),
    (dict(y=_rows(96, 2, 16, 8, 512), y8=_rows(96, 2, 16, 16, 512), **X), 1, "in place"),
    (dict(y=_rows(96), gate=_rows(128), **X), 1, "in place"),
    (dict(pre=LAYER, pre_g=256, x=_rows(64), h=_rows(256)), 1, "in place"),
    (dict(pre=LAYER, x=_rows(64), z_rstd=64), 1, "in place"),
    (dict(x=_rows(64, 2, 16, 8, 512), z=_rows(128)), 1, "x:"),
    (dict(x=_rows(64, 0, 7), z=_rows(128)), 1, "x:"),
    (dict(x=_rows(66), z=_rows(128)), 1, "x:"),
    (dict(**X), 1, "x:"),  # no device memory
]


@pytest.mark.parametrize("fields,status,word", JOIN)
def test_join_refusals_before_touching_the_device(lib, fields, status, word):
    d = lm._filled(lm.lazymar_join_desc(), dict(dict(M=4, D=8, res=1.0, eps=1e-6), **fields))
    assert lib.lazymar_join(d.addr, None) == status
    assert word in lib.lazymar_last_error().decode()


GRAD = dict(pre=LAYER, dh=_rows(64), z=_rows(128), z_mean=16, z_rstd=32, dx=_rows(256))
JOIN_GRAD = [
    (dict(M=-1), 1, "M >= 0"),
    (dict(D=8193), 6, "8192"),
    (dict(M=(1 << 30) + 1), 6, "2^30"),
    (dict(post=5), 1, "post and pre"),
    (dict(res=math.inf), 1, "res"),
    (dict(dx=_rows(0)), 1, "no output"),
    (dict(dh=_rows(0)), 1, "exactly with pre"),
    (dict(pre=NONE), 1, "exactly with pre"),
    (dict(pre=NONE, dh=_rows(0)), 1, "dh or dz"),
    (dict(pre=NONE, dh=_rows(0), dz=_rows(64), dshift=_rows(512)), 1, "need pre"),
    (dict(pre=NONE, dh=_rows(0), dz=_rows(64), scale=_rows(512)), 1, "need pre"),
    (dict(z=_rows(0)), 1, "pre needs z"),
    (dict(z_mean=0), 1, "pre needs z"),
    (dict(z_rstd=0), 1, "pre needs z"),
    (dict(post=RMS, y_rstd=16), 1, "need y"),
    (dict(dgate=_rows(512)), 1, "need y"),
    (dict(post=LAYER, y=_rows(512), y_rstd=16), 1, "y's statistics"),
    (dict(dy=_rows(256)), 1, "one place"),
    (dict(dscale=_rows(512), dshift=_rows(512)), 1, "one place"),
    (dict(dpre_g=512, dpre_b=512), 1, "one place"),
    (dict(y=_rows(512, 2, 16, 8, 640), dy8=_rows(512, 2, 32, 8, 640)), 1, "in place"),
    (dict(dx=_rows(64, 1)), 1, "in place"),
    (dict(dx=_rows(64, 0, 16)), 1, "in place"),
    (dict(dy=_rows(128, 0, 16)), 1, "in place"),
    (dict(scale=_rows(512), dscale=_rows(512)), 1, "in place"),
    (dict(gate=_rows(512), y=_rows(640), dshift=_rows(512)), 1, "in place"),
    (dict(scale=_rows(256)), 1, "in place"),
    (dict(pre_g=512, dpre_g=512), 1, "in place"),
    (dict(dshift=_rows(64)), 1, "in place"),
    (dict(dpre_b=16), 1, "in place"),
    (dict(y=_rows(512, 2, 16, 8, 640), dy8=_rows(512, 2, 16, 16, 640)), 1, "in place"),
    (dict(dh=_rows(64, 2, 16, 8, 512)), 1, "dh:"),
    (dict(dh=_rows(64, 0, 4)), 1, "dh:"),
]


@pytest.mark.parametrize("fields,status,word", JOIN_GRAD)
def test_join_grad_refusals_before_touching_the_device(lib, fields, status, word):
    d = lm._filled(lm.lazymar_join_grad_desc(), dict(dict(M=4, D=8, res=1.0, **GRAD), **fields))
    assert lib.lazymar_join_grad(d.addr, None) == status
    assert word in lib.lazymar_last_error().decode()


def test_join_null_arguments_and_no_rows(lib):
    assert lib.lazymar_join(None, None) == 1 and lib.lazymar_join_grad(None, None) == 1
    d = lm._filled(lm.lazymar_join_desc(), dict(M=0, D=8, res=1.0, eps=1e-6))
    assert lib.lazymar_join(d.addr, None) == 0
    d = lm._filled(lm.lazymar_join_grad_desc(), dict(M=0, D=8, res=1.0, pre=LAYER))
    assert lib.lazymar_join_grad(d.addr, None) == 0


def test_join_workspace(lib):
    assert lm.lazymar_join_grad_workspace(0, 768, 0) == 0
    assert lm.lazymar_join_grad_workspace(1, 768, 1) >= 4 * 768 * 4
    for group in (0, 1, 320):
        for M, D in ((40960, 1280), (1 << 30, 8192), (40960, 64)):
            assert 0 < lm.lazymar_join_grad_workspace(M, D, group) <= 96 << 20


def test_binding_refuses_what_it_cannot_describe():
    torch = pytest.importorskip("torch")
    t = torch.zeros((4, 8))
    r = lm.lazymar_rows(t)
    assert (r.dtype, r.ld) == (lm.LAZYMAR_F32, 8) and lm.lazymar_rows(t[:1, 2:5]).ld == 8
    assert lm.lazymar_rows(t[:, 2:5].bfloat16()).dtype == lm.LAZYMAR_BF16
    for other in (t.double(), t[0], t.t(), t[:, ::2]):
        with pytest.raises(lm.LazymarError, match="rows"):
            lm.lazymar_rows(other)
    with pytest.raises(TypeError, match="gates"):
        lm.lazymar_join_args(4, 8, t, gates=t)
    for other in (t[0].double(), t[:, 0], t[0].bfloat16()):
        with pytest.raises(lm.LazymarError, match="post_g"):
            lm.lazymar_join_args(4, 8, t, post_g=other)


# --------------------------------------------------------------------------
# Lists
# --------------------------------------------------------------------------

def _param(**kw):
    return lm.lazymar_param(**dict(dict(n=8, g=64, g_dtype=0, lr_scale=1.0), **kw))


@pytest.mark.parametrize("param,word", [
    (_param(n=-1), "2^40"),
    (_param(n=(1 << 40) + 1), "2^40"),
    (_param(g_dtype=2), "g_dtype"),
    (_param(out=128, out_dtype=2), "out_dtype"),
    (_param(out=64, out_dtype=1), "in place"),
    (_param(lr_scale=math.nan), "finite"),
    (_param(weight_decay=math.inf), "finite"),
    (_param(p=64), "all or none"),
    (_param(p=64, m=64), "all or none"),
    (_param(m=64, v=64), "all or none"),
    (_param(ema=64), "need p"),
    (_param(copy=64), "need p"),
    (_param(p=64, m=64, v=66), "fp32 device"),
    (_param(), "g must"),
    (_param(g=0), "g must"),
])
def test_list_refusals_before_touching_the_device(lib, param, word):
    h = ctypes.c_void_p(1)
    one = (lm.lazymar_param * 1)(param)
    assert lib.lazymar_params_create(one, 1, ctypes.byref(h)) == 1
    assert word in lib.lazymar_last_error().decode() and not h.value


def test_list_and_call_arguments(lib):
    h = ctypes.c_void_p()
    one = (lm.lazymar_param * 1)(_param())
    assert lib.lazymar_params_create(one, -1, ctypes.byref(h)) == 1
    assert lib.lazymar_params_create(None, 1, ctypes.byref(h)) == 1
    assert lib.lazymar_params_create(one, 1, None) == 1
    assert lib.lazymar_params_create(one, (1 << 20) + 1, ctypes.byref(h)) == 6
    lib.lazymar_params_destroy(None)
    for scale, most in ((0.0, 1.0), (-1.0, 1.0), (math.inf, 1.0), (math.nan, 1.0), (1.0, 0.0), (1.0, math.nan)):
        assert lib.lazymar_grad_norm(None, scale, most, 16, None) == 1
        assert "max_norm" in lib.lazymar_last_error().decode()
    assert lib.lazymar_grad_norm(None, 1.0, 1.0, 16, None) == 1 and "list" in lib.lazymar_last_error().decode()
    assert lib.lazymar_clip_grads(None, 16, None) == 1 and "list" in lib.lazymar_last_error().decode()
    assert lib.lazymar_adamw(None, None, 16, None) == 1

    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, ema_decay=0.5, factor=1.0, steps=1)
    for bad, state, word in ((dict(beta1=1.0), 16, "beta"), (dict(beta2=-0.1), 16, "beta"), (dict(beta1=math.nan), 16, "beta"),
                             (dict(eps=0.0), 16, "eps"), (dict(eps=1e-60), 16, "eps"), (dict(lr=math.inf), 16, "lr"),
                             (dict(lr=1e60), 16, "lr"), (dict(ema_decay=1.5), 16, "ema"), (dict(steps=0), None, "steps"),
                             (dict(factor=0.0), None, "factor"), (dict(factor=math.nan), None, "factor"), (dict(), 16, "list")):
        a = lm.lazymar_adamw_desc(**dict(good, **bad))
        assert lib.lazymar_adamw(None, ctypes.byref(a), state, None) == 1
        assert word in lib.lazymar_last_error().decode()


def test_binding_refuses_lists_that_do_not_match():
    torch = pytest.importorskip("torch")
    g = torch.zeros(8)
    for e, word in ((dict(g=g, p=torch.zeros(7), m=g, v=g), "p:"), (dict(g=g.double()), "g:"), (dict(g=torch.zeros(16)[::2]), "g:"),
                    (dict(g=g, p=g.bfloat16(), m=g, v=g), "p:"), (dict(g=g, p=g, m=g, v=g, copy=g), "copy:")):
        with pytest.raises(lm.LazymarError, match=word):
            lm.lazymar_params_create([e])
