"""AdamW's object where what it holds has changed between steps: refused before anything is
launched, or followed."""
import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(bits=32, copies=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    shapes = [(1000,), (40, 60)]
    params = [torch.randn(*s, generator=g).cuda() for s in shapes]
    held = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    return (adst.AdamW(params, bits=bits, copies=held if copies else None),
            [torch.randn(*s, generator=g).cuda() for s in shapes])


def bits_of(opt):
    names = ["params", "m", "v"] + (["m_scale", "v_scale"] if opt.bits == 8 else []) + \
        (["copies"] if opt.copies is not None else [])
    return [t.detach().float().cpu().clone() for n in names for t in getattr(opt, n)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


CHANGES = {
    "fewer values": lambda t: t.new_zeros(10),
    "another type": lambda t: t.to(torch.float16),
    "another order": lambda t: t.t(),
    "another shape": lambda t: t.t().contiguous(),
    "on the host": lambda t: t.cpu()}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("name", ["params", "copies"])
@pytest.mark.parametrize("change", CHANGES)
def test_data_that_was_replaced(change, name, bits):
    opt, grads = make(bits)
    opt.step(grads)
    tensors = getattr(opt, name)
    was = [t.data for t in tensors]
    for i in ([0, 1] if change == "another type" else [1]):
        tensors[i].data = CHANGES[change](tensors[i].data)
    with pytest.raises(ValueError, match=name):
        opt.step(grads)
    for t, d in zip(tensors, was):
        t.data = d
    opt.step(grads)
    other, _ = make(bits)
    other.step(grads)
    other.step(grads)
    assert opt.t == 2 and equal(bits_of(opt), bits_of(other))


@pytest.mark.parametrize("bits", [32, 8])
def test_other_memory_of_the_same_kind_is_followed(bits):
    opt, grads = make(bits)
    other, _ = make(bits)
    opt.step(grads)
    other.step(grads)
    old = opt.params[0].data
    kept = old.clone()
    opt.params[0].data = old.clone()
    opt.step(grads)
    other.step(grads)
    assert equal(bits_of(opt), bits_of(other)) and torch.equal(old, kept)


@pytest.mark.parametrize("how", ["list", "tuple", "data"])
@pytest.mark.parametrize("bits", [32, 8])
def test_states_that_were_replaced_are_followed(bits, how):
    opt, grads = make(bits)
    other, _ = make(bits)
    opt.step(grads)
    other.step(grads)
    names = ["m", "v"] + (["m_scale", "v_scale"] if bits == 8 else []) + ["copies"]
    old = {n: [t.data for t in getattr(opt, n)] for n in names}
    kept = {n: [t.clone() for t in old[n]] for n in names}
    for n in names:
        new = [t.clone() for t in old[n]]
        if how == "data":
            for t, d in zip(getattr(opt, n), new):
                t.data = d
        else:
            setattr(opt, n, new if how == "list" else tuple(new))
    for x in (opt, other):
        x.step(grads)
    assert equal(bits_of(opt), bits_of(other))
    assert all(torch.equal(x.float(), y.float()) for n in names for x, y in zip(old[n], kept[n]))


def test_copies_that_were_dropped_are_not_written():
    opt, grads = make()
    opt.step(grads)
    old = opt.copies
    kept = [t.clone() for t in old]
    opt.copies = None
    opt.step(grads)
    assert equal(old, kept)


@pytest.mark.parametrize("name", ["m", "v", "m_scale", "v_scale"])
def test_states_that_are_not_what_they_were(name):
    opt, grads = make(8)
    opt.step(grads)
    before = bits_of(opt)
    held = getattr(opt, name)
    for new in (lambda t: t[:-1], lambda t: t.float().double(), lambda t: t.cpu(), lambda t: None):
        setattr(opt, name, tuple(new(t) for t in held))
        with pytest.raises(ValueError, match=name):
            opt.step(grads)
    setattr(opt, name, held)
    assert equal(bits_of(opt), before)


def test_rates_that_are_assigned_take_effect():
    opt, grads = make()
    opt.lr, opt.weight_decay, opt.betas, opt.eps = 0.5, 0.25, (0.5, 0.75), 1e-3
    other = adst.AdamW(make()[0].params, copies=make()[0].copies, lr=0.5, weight_decay=0.25,
                       betas=(0.5, 0.75), eps=1e-3)
    for x in (opt, other):
        x.step(grads)
    assert equal(bits_of(opt), bits_of(other))


@pytest.mark.parametrize("stream", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_the_tensors_versions_rise(bits, stream):
    """Autograd's check of saved tensors sees the step."""
    on = torch.cuda.Stream() if stream else None
    opt, grads = make(bits)
    names = ["params", "m", "v", "copies"] + (["m_scale", "v_scale"] if bits == 8 else [])
    before = {n: [t._version for t in getattr(opt, n)] for n in names}
    w = opt.params[0].requires_grad_()
    loss = (w * w).sum()
    opt.step(grads, stream=on)
    torch.cuda.synchronize()
    for n in names:
        assert all(t._version > v for t, v in zip(getattr(opt, n), before[n]))
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()


@pytest.mark.parametrize("stream", [False, True])
def test_a_pools_version_rises(stream):
    on = torch.cuda.Stream() if stream else None
    a, u, state = (torch.randn(4, 40, device="cuda") for _ in range(3))
    torch.cuda.synchronize()
    before = state._version
    adst.recurrence_step(a, u, state, stream=on)
    torch.cuda.synchronize()
    assert state._version > before
    with torch.inference_mode():
        pool = torch.zeros(4, 40, device="cuda")
    torch.cuda.synchronize()
    adst.recurrence_step(a, u, pool, stream=on)
    torch.cuda.synchronize()
    assert bool((pool != 0).any())
