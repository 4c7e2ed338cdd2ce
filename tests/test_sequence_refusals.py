"""What is no tensor, or none where one is needed, is a ValueError or TypeError from every
argument of the calls that take tensors; on a host without a GPU, with host tensors taken for the
GPU's and nothing launched."""
import numpy as np
import pytest
import torch

import paper_2509_02197_amd as adst
from paper_2509_02197_amd import sequence

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only")


@pytest.fixture(autouse=True)
def host_tensors(monkeypatch):
    real = sequence._code

    def code(name, t):
        if isinstance(t, torch.Tensor) and t.dtype in sequence._codes():
            return sequence._codes()[t.dtype]
        return real(name, t)

    def call(*args):
        raise AssertionError("a call was made")

    monkeypatch.setattr(sequence, "_code", code)
    monkeypatch.setattr(sequence, "_call", call)


T = torch.zeros
CALLS = {
    "recurrence": (adst.recurrence, dict(a=T(2, 3, 4), u=T(2, 3, 4), h0=T(2, 4),
                                         lens=T(2, dtype=torch.int32)), ("a", "u")),
    "recurrence_vjp": (adst.recurrence_vjp,
                       dict(a=T(2, 3, 4), u=T(2, 3, 4), dh=T(2, 3, 4), h0=T(2, 4),
                            lens=T(2, dtype=torch.int32), dhT=T(2, 4),
                            ck=T(32, dtype=torch.uint8)), ("a", "u", "dh")),
    "recurrence_step": (adst.recurrence_step,
                        dict(a=T(2, 4), u=T(2, 4), state=T(3, 4), slots=T(2, dtype=torch.int32)),
                        ("a", "u", "state")),
    "layer_norm": (adst.layer_norm, dict(x=T(2, 4), w=T(4), b=T(4)), ("x",)),
    "layer_norm_vjp": (adst.layer_norm_vjp,
                       dict(x=T(2, 4), dy=T(2, 4), mean=T(2), rstd=T(2), w=T(4)),
                       ("x", "dy", "mean", "rstd")),
}
WRONG = {"a number": 3.0, "a text": "x", "a list": [1.0, 2.0], "an array": np.zeros((2, 4)),
         "a scalar": T(()), "no axes but one": T(1), "many axes": T(1, 1, 1, 1, 1)}
CASES = [(name, arg, kind) for name, (_, args, _) in CALLS.items() for arg in args
         for kind in WRONG] + \
        [(name, arg, "none") for name, (_, _, needed) in CALLS.items() for arg in needed]


@pytest.mark.parametrize("name", CALLS)
def test_the_right_arguments_reach_the_call(name):
    f, args, _ = CALLS[name]
    with pytest.raises(AssertionError, match="a call was made"):
        f(**args)


@pytest.mark.parametrize("name,arg,kind", CASES)
def test_arguments_that_are_no_tensors(name, arg, kind):
    f, args, _ = CALLS[name]
    with pytest.raises((ValueError, TypeError)):
        f(**{**args, arg: WRONG.get(kind)})


def optimizer():
    return adst.AdamW([T(5), T(4, 3)], copies=[T(5), T(4, 3)])


@pytest.mark.parametrize("wrong", [None, 3.0, "x", [1.0], np.zeros(5)])
@pytest.mark.parametrize("where", [0, 1])
def test_adamw_lists(wrong, where):
    good = [T(5), T(4, 3)]
    bad = list(good)
    bad[where] = wrong
    state = {"m": good, "v": good}
    for make in (lambda: adst.AdamW(bad), lambda: adst.AdamW(good, copies=bad),
                 lambda: adst.AdamW(good, state=dict(state, m=bad)),
                 lambda: adst.AdamW(good, state=dict(state, v=bad)),
                 lambda: optimizer().step(bad)):
        with pytest.raises((ValueError, TypeError)):
            make()
    for name in ("params", "copies", "m", "v"):
        opt = optimizer()
        setattr(opt, name, bad)
        with pytest.raises((ValueError, TypeError)):
            opt.step(good)


@pytest.mark.parametrize("wrong", [3.0, "x", [1.0], np.zeros(1), T(2), T(1, dtype=torch.int32)])
def test_adamw_scale(wrong):
    with pytest.raises((ValueError, TypeError)):
        optimizer().step([T(5), T(4, 3)], grad_scale=wrong)


@pytest.mark.parametrize("make", [
    lambda: adst.AdamW(None), lambda: adst.AdamW(3), lambda: adst.AdamW([T(5)], copies=3),
    lambda: adst.AdamW([T(5)], state={"m": [T(5)]}), lambda: adst.AdamW([T(5)], state=[T(5)]),
    lambda: adst.AdamW([T(5)], lr="x"), lambda: adst.AdamW([T(5)], betas=0.9),
    lambda: adst.AdamW([T(5)], eps=None), lambda: optimizer().step(None),
    lambda: optimizer().step(T(5)), lambda: optimizer().step(3),
    lambda: optimizer().step([T(5), T(4, 3)], t="x"),
    lambda: optimizer().step([T(5), T(4, 3)], t=1.5)])
def test_adamw_arguments(make):
    with pytest.raises((ValueError, TypeError)):
        make()
