"""AdamW over many tensors against the formula in 64 bits on the host. One step
rounds each of its values a few times (16 roundings bound them); an 8-bit state
adds one rounding to e4m3 (relative 2^-4, and half the smallest code's step
near zero) times its block's scale."""
import math

import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util as ref

pytestmark = pytest.mark.gpu
BLOCK = adst.ADST_STATE_BLOCK
SHAPES = [(1,), (7,), (255,), (256,), (257,), (33, 65), (0,), (1000,), (4, 5, 6), (3, 2048),
          (70001,)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(shapes, dtype=torch.float32, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(*s, generator=g, dtype=torch.float64) * std).to(dtype).cuda()
            for s in shapes]


def values(opt, name, i):
    """A state's values in float64: of "v" with 8 bits the square root, as it is held."""
    x = getattr(opt, name)[i].double().cpu().reshape(-1)
    if opt.bits == 8:
        s = getattr(opt, name + "_scale")[i].double().cpu()
        x = x * s.repeat_interleave(BLOCK)[:x.numel()]
    return x


def expected(p, g, m, v, t, lr, wd, betas, eps, scale=1.0):
    """m, v and p after the step, and their bounds, by the formula in float64."""
    b1, b2 = betas
    u = 2.0 ** -24 if p.dtype == torch.float32 else 2.0 ** -53
    p, g = p.double().cpu().reshape(-1), g.double().cpu().reshape(-1) * scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    mE = 16 * u * (b1 * m.abs() + (1 - b1) * g.abs())
    vE = 16 * u * v1
    denominator = torch.sqrt(v1 / (1 - b2 ** t)) + eps
    update = m1 / (1 - b1 ** t) / denominator
    updateE = mE / (1 - b1 ** t) / denominator + 16 * u * update.abs()
    p1 = p * (1 - lr * wd) - lr * update
    return (m1, mE + 1e-40), (v1, vE + 1e-40), (p1, 16 * u * (p.abs() + lr * update.abs())
                                               + lr * updateE)


def near(got, want, bound):
    got = got.double().cpu().reshape(-1)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def check_step(opt, grads, t=None, scale=1.0, **over):
    """One step against the formula from the state before it."""
    before = [(p.clone(), values(opt, "m", i), values(opt, "v", i))
              for i, p in enumerate(opt.params)]
    opt.step(grads, t=t, **over)
    lrs, wds = (x if isinstance(x, list) else [x] * len(grads) for x in (opt.lr, opt.weight_decay))
    for i, (p, m, v) in enumerate(before):
        v = v * v if opt.bits == 8 else v
        M, V, P = expected(p, grads[i], m, v, opt.t, lrs[i], wds[i], opt.betas, opt.eps, scale)
        near(opt.params[i], *P)
        if opt.copies is not None:
            c = opt.copies[i]
            assert torch.equal(c, opt.params[i].to(torch.float32).to(c.dtype))
        if opt.bits == 32:
            near(values(opt, "m", i), *M)
            near(values(opt, "v", i), *V)
            continue
        for name, (x, E) in (("m", M), ("v", (V[0].sqrt(), 16 * 2.0 ** -24 * V[0].sqrt()))):
            pad = torch.zeros(-(-x.numel() // BLOCK) * BLOCK, dtype=torch.float64)
            pad[:x.numel()] = x.abs()
            top = pad.view(-1, BLOCK).amax(1)
            tops = top.repeat_interleave(BLOCK)[:x.numel()]
            got = values(opt, name, i)
            # v's positive values are raised to the smallest code instead of half a step up or down
            step = 2.0 ** -9 if name == "v" else 2.0 ** -10
            near(got, x, 1.001 * (2.0 ** -4 * x.abs() + step * tops / 448) + E)
            near(getattr(opt, name + "_scale")[i], top / 448, 1e-6 * top)
            if name == "v":
                assert bool((got[(x > 0) & (tops > 2.0 ** -99)] > 0).all())


@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_against_the_formula(bits, grad, copy):
    params = make(SHAPES)
    copies = None if copy is None else [torch.empty_like(p, dtype=copy) for p in params]
    opt = adst.AdamW(params, bits=bits, copies=copies, lr=0.01, betas=(0.9, 0.95),
                     weight_decay=0.1)
    for k in range(4):
        check_step(opt, make(SHAPES, grad, seed=k + 1, std=0.1))
    assert opt.t == 4


def test_double_precision():
    opt = adst.AdamW(make(SHAPES, torch.float64), lr=0.01)
    for k in range(3):
        check_step(opt, make(SHAPES, torch.float64, seed=k + 1))


@pytest.mark.parametrize("bits", [32, 8])
def test_each_tensor_has_its_rate_and_decay(bits):
    n = len(SHAPES)
    opt = adst.AdamW(make(SHAPES), bits=bits, lr=[0.01 * (i + 1) for i in range(n)],
                     weight_decay=[0.1 * (i % 3) for i in range(n)])
    check_step(opt, make(SHAPES, seed=1))
    check_step(opt, make(SHAPES, seed=2), lr=0.5)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    g = torch.Generator().manual_seed(3)
    shapes = [(int(n),) for n in torch.randint(1, 900, (523,), generator=g)]
    opt = adst.AdamW(make(shapes), bits=bits)
    check_step(opt, make(shapes, seed=1))


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_at_any_element(bits):
    """Views that start one element into a buffer, beside aligned ones."""
    flats = [torch.randn(5000, device="cuda") for _ in range(2)]
    params = [flats[0][1:2000], flats[0][2001:2007], flats[0][2500:4999]]
    grads = [flats[1][3:2002], flats[1][2100:2106], flats[1][2501:5000]]
    opt = adst.AdamW(params, bits=bits, copies=[torch.zeros(p.numel() + 1, device="cuda",
                                                            dtype=torch.bfloat16)[1:]
                                                for p in params])
    keep = flats[0][2000].item(), flats[0][2007].item(), flats[0][4999].item()
    check_step(opt, grads)
    assert keep == (flats[0][2000].item(), flats[0][2007].item(), flats[0][4999].item())


@pytest.mark.parametrize("bits", [32, 8])
def test_going_on_from_a_state(bits):
    one = adst.AdamW(make(SHAPES), bits=bits)
    for k in range(2):
        one.step(make(SHAPES, seed=k))
    names = ("m", "v", "m_scale", "v_scale") if bits == 8 else ("m", "v")
    two = adst.AdamW([p.clone() for p in one.params], bits=bits,
                     state={k: [t.clone() for t in getattr(one, k)] for k in names})
    for opt in (one, two):
        opt.step(make(SHAPES, seed=9), t=3)
    for k in ("params",) + names:
        for a, b in zip(getattr(one, k), getattr(two, k)):
            assert torch.equal(a.float(), b.float())


@pytest.mark.parametrize("bits", [32, 8])
def test_grad_scale(bits):
    opt = adst.AdamW(make(SHAPES), bits=bits)
    check_step(opt, make(SHAPES, seed=1), scale=0.25,
               grad_scale=torch.tensor(0.25, device="cuda"))
    held = [t.clone() for k in ("params", "m", "v") for t in getattr(opt, k)]
    for bad in (math.nan, math.inf):
        opt.step(make(SHAPES, seed=2), grad_scale=torch.tensor([bad], device="cuda"))
    for a, b in zip(held, [t for k in ("params", "m", "v") for t in getattr(opt, k)]):
        assert torch.equal(a.float(), b.float())
    assert opt.t == 3


@pytest.mark.parametrize("bits", [32, 8])
def test_a_nan_stays_in_its_element_or_block(bits):
    opt, clean = (adst.AdamW(make([(1000,)]), bits=bits) for _ in range(2))
    g = make([(1000,)], seed=1)
    clean.step(g)
    g[0][300] = math.nan
    opt.step(g)
    bad = torch.zeros(1000, dtype=torch.bool)
    bad[300] = True
    assert torch.equal(torch.isnan(opt.params[0]).cpu(), bad)
    assert torch.equal(opt.params[0].cpu()[~bad], clean.params[0].cpu()[~bad])
    if bits == 8:
        bad[256:512] = True
    for name in ("m", "v"):
        assert torch.equal(torch.isnan(values(opt, name, 0)), bad)
        assert torch.equal(values(opt, name, 0)[~bad], values(clean, name, 0)[~bad])


def test_blocks_of_zeros_and_of_tiny_values():
    """No gradient, and one whose states are below the smallest scale: held as zeros, and the
    parameters only decay or move by a finite amount."""
    p = make([(600,)])
    opt = adst.AdamW(p, bits=8, lr=0.1, weight_decay=0.0)
    before = p[0].clone()
    g = torch.zeros(600, device="cuda")
    g[300] = 1e-30
    opt.step([g])
    assert torch.equal(p[0][:300], before[:300])
    assert bool(torch.isfinite(p[0]).all())
    assert all(bool((x[0].float() == 0).all()) for x in (opt.m, opt.v, opt.m_scale, opt.v_scale))


def test_codes_follow_the_block_not_the_tensor():
    """Blocks of very different magnitudes keep their own precision."""
    p = make([(1024,)])
    opt = adst.AdamW(p, bits=8)
    scale = torch.tensor([1e3, 1.0, 1e-3, 1e-6], device="cuda").repeat_interleave(BLOCK)
    check_step(opt, [make([(1024,)], seed=1)[0] * scale])


def test_the_same_bits_each_time_and_on_another_stream():
    def go(stream):
        opt = adst.AdamW(make(SHAPES), bits=8)
        for k in range(3):
            g = make(SHAPES, torch.bfloat16, seed=k)
            torch.cuda.synchronize()
            opt.step(g, stream=stream)
        torch.cuda.synchronize()
        return [t.float() for k in ("params", "m", "v", "m_scale") for t in getattr(opt, k)]

    one = go(None)
    for other in (go(None), go(torch.cuda.Stream())):
        assert all(torch.equal(a, b) for a, b in zip(one, other))


def test_a_large_tensor():
    """More than 2^31 values: the last ones as those of a small tensor."""
    n = (1 << 31) + 1000
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    tail = make([(2000,)], torch.bfloat16)[0]
    p[-2000:], g[-2000:] = 1.0, tail
    opt = adst.AdamW([p], bits=8)
    opt.step([g])
    small = adst.AdamW([p.new_ones(2000)], bits=32)
    small.step([tail])
    assert torch.equal(p[-2000:], small.params[0])
    assert bool((p[:1000] == 0).all())


def test_refusals():
    p = make([(30,), (4, 5)])
    opt = adst.AdamW(p, bits=8)
    g = make([(30,), (4, 5)], seed=1)
    half = torch.bfloat16
    for call in (lambda: opt.step(g[:1]), lambda: opt.step([g[0], g[1].to(half)]),
                 lambda: opt.step([g[0][:9], g[1]]), lambda: opt.step([g[0], g[1].cpu()]),
                 lambda: opt.step([g[0], torch.zeros(5, 8, device="cuda")[:, ::2]]),
                 lambda: opt.step(g, lr=[1.0]),
                 lambda: opt.step(g, grad_scale=torch.ones(2, device="cuda")),
                 lambda: adst.AdamW(p, bits=16),
                 lambda: adst.AdamW([p[0], p[1].t()]),
                 lambda: adst.AdamW(p, copies=[p[0].to(half)]),
                 lambda: adst.AdamW(p, copies=[p[0].to(half), p[0].to(half)]),
                 lambda: adst.AdamW(p, state={"m": p, "v": p[:1]}),
                 lambda: adst.AdamW(p, bits=8, state={"m": p, "v": p, "m_scale": p,
                                                      "v_scale": p})):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: adst.AdamW([x.to(half) for x in p]),
                 lambda: adst.AdamW([x.double() for x in p], bits=8),
                 lambda: opt.step([x.double() for x in g])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: opt.step(g, t=0), lambda: opt.step(g, lr=float("nan"))):
        with pytest.raises(adst.AdstError):
            call()
    assert opt.t == 0
