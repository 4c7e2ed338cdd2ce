"""AdamW's object where what it holds has changed, on a host without a GPU: the native call and
the C call are replaced by ones that record, and the checks between are the object's own."""
import ctypes

import pytest
import torch

import paper_2509_02197_amd as adst
from paper_2509_02197_amd import sequence

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only")


class Calls:
    """In place of the library and the binding: the C calls' descriptors, and what the native
    call answers."""

    def __init__(self):
        self.made = []
        self.problems = []
        self.used = []  # what each call records on its stream
        self.native = None

    def adst_adamw(self, prob, rows, n, handle):
        self.problems.append({k: getattr(prob, k) for k, _ in prob._fields_})
        self.made.append([{k: getattr(r, k) for k, _ in r._fields_} for r in rows])
        return adst.ADST_OK

    def adamw_step(self, *args):
        return self.native


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(sequence, "lib", lambda: c)
    monkeypatch.setattr(sequence, "_binding", lambda: c)
    monkeypatch.setattr(sequence, "_code", lambda name, t: sequence._codes()[t.dtype])

    def call(device, stream, used, body):
        c.used.append(used)
        return body(0)

    monkeypatch.setattr(sequence, "_call", call)
    return c


def make(bits=32, copies=True):
    params = [torch.zeros(1000), torch.zeros(4, 6)]
    held = [torch.zeros(p.shape, dtype=torch.bfloat16) for p in params] if copies else None
    return adst.AdamW(params, bits=bits, copies=held), [torch.zeros(1000), torch.zeros(4, 6)]


CHANGES = {
    "fewer values": lambda t: torch.zeros(10, dtype=t.dtype),
    "another type": lambda t: torch.zeros(t.shape, dtype=torch.float16),
    "another order": lambda t: t.t() if t.dim() > 1 else torch.zeros(2 * len(t),
                                                                    dtype=t.dtype)[::2],
    "another shape": lambda t: t.reshape(2, -1),
    "another device": lambda t: torch.empty_like(t, device="meta")}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("name", ["params", "copies", "m", "v"])
@pytest.mark.parametrize("change", CHANGES)
def test_tensors_that_are_not_what_they_were(calls, change, name, which, bits):
    opt, grads = make(bits)
    opt.step(grads)
    assert len(calls.made) == 1 and opt.t == 1
    held = list(getattr(opt, name))
    held[which] = CHANGES[change](held[which])
    setattr(opt, name, tuple(held))
    with pytest.raises(ValueError, match=name):
        opt.step(grads)
    assert len(calls.made) == 1 and opt.t == 1


@pytest.mark.parametrize("name", ["params", "copies"])
def test_data_that_was_replaced(calls, name):
    """By a module's conversion, say: all of them."""
    opt, grads = make()
    for t in getattr(opt, name):
        t.data = t.data.to(torch.float16)
    with pytest.raises(ValueError, match=name):
        opt.step(grads)
    opt, grads = make()
    getattr(opt, name)[0].data = torch.zeros(10, dtype=getattr(opt, name)[0].dtype)
    with pytest.raises(ValueError, match=name):
        opt.step(grads)
    assert not calls.made


def test_other_memory_of_the_same_kind_is_followed(calls):
    opt, grads = make()
    opt.params[0].data = torch.ones(1000)
    opt.step(grads)
    assert calls.made[0][0]["p"] == opt.params[0].data_ptr()


@pytest.mark.parametrize("name", ["params", "copies"])
def test_lists_of_another_length(calls, name):
    opt, grads = make()
    setattr(opt, name, getattr(opt, name)[:1])
    with pytest.raises(ValueError):
        opt.step(grads)
    assert not calls.made


@pytest.mark.parametrize("copies", [True, False])
@pytest.mark.parametrize("bits", [32, 8])
def test_everything_that_a_call_touches_is_recorded_on_its_stream(calls, bits, copies):
    """Else memory that the step still writes could be given to others when its owner goes."""
    opt, grads = make(bits, copies)
    scale = torch.ones(1)
    opt.step(grads, grad_scale=scale, stream=7)
    names = ["params", "m", "v"] + (["m_scale", "v_scale"] if bits == 8 else []) + \
        (["copies"] if copies else [])
    expected = [scale, *grads] + [t for n in names for t in getattr(opt, n)]
    assert {id(t) for t in calls.used[0]} == {id(t) for t in expected}


@pytest.mark.parametrize("name", ["m", "v", "m_scale", "v_scale"])
@pytest.mark.parametrize("how", ["list", "tuple", "data"])
def test_states_that_were_replaced_are_followed(calls, name, how):
    opt, grads = make(8)
    loaded = [torch.zeros_like(t) for t in getattr(opt, name)]
    if how == "data":
        for t, new in zip(getattr(opt, name), loaded):
            t.data = new
    else:
        setattr(opt, name, loaded if how == "list" else tuple(loaded))
    opt.step(grads)
    assert [r[name] for r in calls.made[0]] == [t.data_ptr() for t in loaded]


def test_copies_that_were_dropped_are_not_written(calls):
    opt, grads = make()
    opt.step(grads)
    opt.copies = None
    opt.step(grads)
    assert calls.made[0][0]["copy"] and calls.made[1][0]["copy"] is None
    other, _ = make(copies=False)
    other.copies = opt.params
    with pytest.raises(ValueError, match="copies"):
        other.step(grads)


@pytest.mark.parametrize("name", ["m_scale", "v_scale"])
def test_scales_that_are_not_what_they_were(calls, name):
    for new in (lambda t: t[:-1], lambda t: t.double(), lambda t: t.repeat(2)[::2]):
        opt, grads = make(8)
        held = list(getattr(opt, name))
        held[0] = new(held[0])
        setattr(opt, name, held)
        with pytest.raises(ValueError, match=name):
            opt.step(grads)
    assert not calls.made


def test_rates_that_are_assigned_take_effect(calls):
    opt, grads = make()
    opt.lr, opt.weight_decay, opt.betas, opt.eps = 0.5, [0.25, 0.125], (0.5, 0.75), 1e-3
    assert (opt.lr, opt.weight_decay, opt.betas, opt.eps) == (0.5, [0.25, 0.125], (0.5, 0.75), 1e-3)
    opt.step(grads)
    assert [r["lr"] for r in calls.made[0]] == [0.5, 0.5]
    assert [r["weight_decay"] for r in calls.made[0]] == [0.25, 0.125]
    p = calls.problems[0]
    assert (p["beta1"], p["beta2"], p["eps"]) == (0.5, 0.75, 1e-3)
    opt.step(grads, lr=2.0)
    assert opt.lr == 2.0 and calls.made[1][1]["lr"] == 2.0
    with pytest.raises(ValueError, match="lr"):
        opt.lr = [1.0]
    with pytest.raises((TypeError, ValueError)):
        opt.betas = (0.5,)
    with pytest.raises(AttributeError):
        opt.bits = 8
    assert opt.lr == 2.0 and opt.betas == (0.5, 0.75) and opt.bits == 32


@pytest.mark.parametrize("bits", [32, 8])
def test_the_tensors_versions_rise(calls, bits):
    """Autograd's check of saved tensors sees the step."""
    opt, grads = make(bits)
    names = ["params", "m", "v", "copies"] + (["m_scale", "v_scale"] if bits == 8 else [])
    before = {n: [t._version for t in getattr(opt, n)] for n in names}
    opt.step(grads)
    for n in names:
        assert all(t._version > v for t, v in zip(getattr(opt, n), before[n]))


def test_a_tensor_twice_is_refused(calls):
    """Its two updates would race."""
    p, q = torch.zeros(600), torch.zeros(600)
    state = {"m": [torch.zeros(600) for _ in range(2)], "v": [torch.zeros(600) for _ in range(2)]}
    for make in (lambda: adst.AdamW([p, p]), lambda: adst.AdamW([p, p.view(600)]),
                 lambda: adst.AdamW([p, q], copies=[p.half()] * 2),
                 lambda: adst.AdamW([p, q], state=dict(state, m=state["m"][:1] * 2)),
                 lambda: adst.AdamW([p, q], state=dict(state, v=state["v"][:1] * 2))):
        with pytest.raises(ValueError, match="twice"):
            make()
    empty = torch.zeros(0)
    adst.AdamW([p, q, empty, torch.zeros(0)])  # nothing to update twice
