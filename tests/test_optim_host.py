"""The end of a training step without a GPU: what the binding and AdamW refuse, against a library that is not called."""
import pytest

from paper_2503_12450_gb300 import lazymar as lm

torch = pytest.importorskip("torch")


class Handle:
    ptr = 16


@pytest.fixture
def calls(monkeypatch):
    """Stands in for the library: counts the calls that reach it."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0
    monkeypatch.setattr(lm, "lib", lambda: Library())
    return made


def test_a_learning_rate_of_another_type_is_refused(calls):
    """Its bytes would be read as fp32: a rate of 1e-3 in fp64 as 2.4e-13."""
    for lr in (torch.tensor(1e-3, dtype=torch.float64), torch.tensor([1e-3], dtype=torch.bfloat16), torch.tensor([1]),
               torch.tensor([1], dtype=torch.int32), torch.tensor([1e-3, 1e-3]), torch.empty(0)):
        with pytest.raises(lm.LazymarError, match="lr_device"):
            lm.lazymar_adamw(Handle, torch.zeros(4), 0.0, lr_device=lr)
    assert not calls
    for lr in (torch.tensor(1e-3), torch.tensor([1e-3]), torch.tensor([[1e-3]]), None, 4096):
        lm.lazymar_adamw(Handle, torch.zeros(4), 0.0, lr_device=lr)
    assert calls == ["lazymar_adamw"] * 5


def test_a_state_of_another_type_or_size_is_refused(calls):
    ways = [lambda s: lm.lazymar_grad_norm(Handle, s, 1.0), lambda s: lm.lazymar_clip_grads(Handle, s),
            lambda s: lm.lazymar_adamw(Handle, s, 1e-3)]
    for f in ways:
        for s in (torch.zeros(4, dtype=torch.float64), torch.zeros(2), torch.zeros(4, dtype=torch.bfloat16), torch.zeros(8)[::2],
                  torch.zeros(2, dtype=torch.int64), torch.zeros(15, dtype=torch.uint8)):
            with pytest.raises(lm.LazymarError, match="state"):
                f(s)
    assert not calls
    for f in ways:
        for s in (torch.zeros(4), torch.zeros(4, dtype=torch.int32), torch.zeros(16, dtype=torch.uint8), torch.zeros((1, 4)), 4096):
            f(s)
    assert len(calls) == 15
    lm.lazymar_adamw(Handle, None, 1e-3, steps=1)


# --------------------------------------------------------------------------
# AdamW
# --------------------------------------------------------------------------
def _adamw(calls, shapes=dict(w=(4, 3), b=(3,)), **kw):
    from paper_2503_12450_gb300.adamw import AdamW
    g = torch.Generator().manual_seed(1)
    p = {k: torch.randn(s, generator=g) for k, s in shapes.items()}
    return AdamW(p, {k: torch.zeros_like(v) for k, v in p.items()}, 1e-3, **kw)


def test_averages_of_parameters_that_ask_for_gradients_have_no_graph(calls):
    import copy

    from paper_2503_12450_gb300.adamw import AdamW
    p = {"w": torch.nn.Parameter(torch.ones(4, 3))}
    opt = AdamW(p, {"w": torch.zeros(4, 3)}, 1e-3, ema_decay=0.9)
    assert not opt.ema["w"].requires_grad and opt.ema["w"].is_leaf
    d = copy.deepcopy(opt.state_dict())
    opt.load_state_dict(d)
    assert torch.equal(opt.ema["w"], torch.ones(4, 3)) and not opt.ema["w"].requires_grad


def test_a_state_that_does_not_fit_is_refused_and_changes_nothing(calls):
    """Not spread over the tensors, and not loaded in part."""
    opt = _adamw(calls, ema_decay=0.9)
    good = opt.state_dict()
    for k in ("m", "v", "ema"):
        for t in good[k].values():
            t.fill_(2.0)
    good["state"].fill_(3.0)
    before = {k: [t.clone() for t in ([v] if k == "state" else v.values())] for k, v in opt.state_dict().items()}
    bad = [dict(good, state=torch.zeros(1)), dict(good, state=torch.zeros(4, dtype=torch.float64)),
           {k: v for k, v in good.items() if k != "ema"}, {k: v for k, v in good.items() if k != "m"}]
    for k in ("m", "v", "ema"):
        bad += [dict(good, **{k: dict(good[k], w=torch.zeros(3))}), dict(good, **{k: dict(good[k], w=torch.zeros(3, 4))}),
                dict(good, **{k: {"w": good[k]["w"]}}), dict(good, **{k: dict(good[k], other=torch.zeros(1))})]
    for d in bad:
        with pytest.raises(lm.LazymarError, match="state"):
            opt.load_state_dict(d)
        now = opt.state_dict()
        assert all(torch.equal(a, b) for k, w in before.items() for a, b in zip([now[k]] if k == "state" else now[k].values(), w))
    with pytest.raises(lm.LazymarError, match="no averaged weights"):
        opt.load_state_dict(_adamw(calls).state_dict())
    opt.load_state_dict(good)
    assert all((t == 2.0).all() for k in ("m", "v", "ema") for t in getattr(opt, k).values()) and (opt.state == 3.0).all()
    plain = _adamw(calls)
    plain.load_state_dict(good)  # averages that it does not keep are not looked at
    assert (plain.m["w"] == 2.0).all()


def test_copies_of_weights_that_are_not_there_are_refused(calls):
    with pytest.raises(lm.LazymarError, match="copies"):
        _adamw(calls, copies={"w": torch.zeros((4, 3), dtype=torch.bfloat16), "weight": torch.zeros(3, dtype=torch.bfloat16)})
    assert not calls
    _adamw(calls, copies={"w": torch.zeros((4, 3), dtype=torch.bfloat16)})
