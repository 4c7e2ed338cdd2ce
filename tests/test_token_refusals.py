"""What is no tensor, or none where one is needed, or of another shape, type or layout, is a
ValueError or TypeError from every argument of the token operators' calls; on a host without a GPU,
with host tensors taken for the GPU's and nothing launched."""
import numpy as np
import pytest
import torch

import paper_2509_02197_amd as adst
from paper_2509_02197_amd import sequence, tokens

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

    monkeypatch.setattr(tokens, "_code", code)
    monkeypatch.setattr(tokens, "_call", call)


def T(*shape, kind=torch.float32):
    return torch.zeros(*shape, dtype=kind)


I32 = torch.int32
CONV = dict(x=T(2, 3, 6), w=T(4, 6), b=T(6), x0=T(2, 3, 6), lens=T(2, kind=I32))
SCAN = dict(x=T(2, 3, 6), delta=T(2, 3, 6), A=T(6, 4), B=T(2, 3, 2, 4), C=T(2, 3, 2, 4), D=T(6),
            z=T(2, 3, 6), delta_bias=T(6), h0=T(2, 6, 4), lens=T(2, kind=I32))
XENT = dict(x=T(5, 4), w=T(7, 4), labels=T(5, kind=I32))
CK = 2 * 6 * 4 * 4  # one checkpoint of [2, 6, 4] float32
CALLS = {
    "causal_conv": (adst.causal_conv, CONV, ("x", "w")),
    "causal_conv_vjp": (adst.causal_conv_vjp, dict(CONV, dy=T(2, 3, 6), dxT=T(2, 3, 6)),
                        ("x", "dy", "w")),
    "causal_conv_step": (adst.causal_conv_step,
                         dict(x=T(2, 6), w=T(4, 6), window=T(5, 3, 6), b=T(6),
                              slots=T(2, kind=I32)), ("x", "w", "window")),
    "selective_scan": (adst.selective_scan, SCAN, ("x", "delta", "A", "B", "C")),
    "selective_scan_vjp": (adst.selective_scan_vjp,
                           dict(SCAN, dy=T(2, 3, 6), dhT=T(2, 6, 4), ck=T(CK, kind=torch.uint8)),
                           ("x", "delta", "A", "B", "C", "dy")),
    "selective_scan_step": (adst.selective_scan_step,
                            dict(x=T(2, 6), delta=T(2, 6), A=T(6, 4), B=T(2, 2, 4), C=T(2, 2, 4),
                                 state=T(5, 6, 4), D=T(6), z=T(2, 6), delta_bias=T(6),
                                 slots=T(2, kind=I32)), ("x", "delta", "A", "B", "C", "state")),
    "linear_cross_entropy": (adst.linear_cross_entropy, XENT, ("x", "w", "labels")),
    "linear_cross_entropy_vjp": (adst.linear_cross_entropy_vjp, dict(XENT, lse=T(5), dloss=T(5)),
                                 ("x", "w", "labels", "lse")),
}
WRONG = {"a number": 3.0, "a text": "x", "a list": [1.0, 2.0], "an array": np.zeros((2, 4)),
         "a scalar": T(()), "no axes but one": T(1), "many axes": T(1, 1, 1, 1, 1)}


def of_another(kind, t):
    """t as it may not be."""
    if kind == "type":
        return t.to(torch.int64 if t.dtype == I32 else torch.int16)
    if kind == "layout":  # every second of twice as many
        return torch.cat([t, t], -1)[..., ::2]
    return torch.cat([t, t[..., :1]], -1)  # one more along the last axis


def cases():
    for name, (_, args, needed) in CALLS.items():
        for arg in args:
            for kind in WRONG:
                yield name, arg, kind
            for kind in ("type", "layout", "shape"):
                if not (arg == "x" and kind != "layout"):  # x gives the others' shape and type
                    yield name, arg, kind
        for arg in needed:
            yield name, arg, "none"


@pytest.mark.parametrize("name", CALLS)
def test_the_right_arguments_reach_the_call(name):
    f, args, _ = CALLS[name]
    with pytest.raises(AssertionError, match="a call was made"):
        f(**args)


@pytest.mark.parametrize("name,arg,kind", cases())
def test_wrong_arguments(name, arg, kind):
    f, args, _ = CALLS[name]
    value = None if kind == "none" else WRONG[kind] if kind in WRONG else of_another(kind, args[arg])
    with pytest.raises((ValueError, TypeError)):
        f(**{**args, arg: value})


@pytest.mark.parametrize("kw", [
    dict(B=T(2, 3, 4)), dict(C=T(2, 3, 4)), dict(B=T(2, 3, 4, 4), C=T(2, 3, 4, 4)),
    dict(B=T(2, 3, 4, 4)[:, :, ::2]), dict(A=T(6, 5)), dict(A=T(6, 0)),
    dict(B=T(2, 3, 2, 4, kind=torch.bfloat16)), dict(D=T(6, kind=torch.float64))])
def test_groups_and_types_of_the_scan(kw):
    with pytest.raises((ValueError, TypeError)):
        adst.selective_scan(**{**SCAN, **kw})


def test_coefficients_without_the_groups_axis():
    one = dict(SCAN, B=T(2, 3, 4), C=T(2, 3, 1, 4))
    with pytest.raises(AssertionError, match="a call was made"):
        adst.selective_scan(**one)


@pytest.mark.parametrize("w", [T(0, 6), T(9, 6), T(4, 5), T(4, 6, kind=torch.bfloat16)])
def test_taps(w):
    with pytest.raises((ValueError, TypeError)):
        adst.causal_conv(CONV["x"], w)


@pytest.mark.parametrize("act", [1 << 31, 1 << 32, (1 << 32) + 1, -(1 << 32), 0.5, None, "silu"])
@pytest.mark.parametrize("name", ["causal_conv", "causal_conv_vjp", "causal_conv_step"])
def test_activations(name, act):
    """A number beyond 32 bits is not cut to one of the two; others are the C call's to refuse."""
    f, args, _ = CALLS[name]
    with pytest.raises((ValueError, TypeError)):
        f(**args, act=act)
