"""16-bit gates at the ends of their range: a closed gate leaves nothing of the state."""
import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.gpu
SIGMOID = adst.ADST_GATE_SIGMOID
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


@pytest.mark.parametrize("T", [1, 40, 3000])
@pytest.mark.parametrize("a", [-float("inf"), -60000.0, -200.0])
@pytest.mark.parametrize("dtype", HALVES)
def test_a_closed_gate_replaces_the_state(dtype, a, T):
    """exp(a) is beyond the 32-bit range: s = 0 and 1 - s = 1, whatever the state's size."""
    g = torch.Generator().manual_seed(1)
    u, dh = (torch.randn(2, T, 70, generator=g).to(dtype).cuda() for _ in range(2))
    av = torch.randn(2, T, 70, generator=g).to(dtype).cuda()
    t = T // 2
    av[:, t] = a
    h0 = torch.full((2, 70), 1e37, device="cuda")
    f = adst.recurrence(av, u, h0=h0, gate=SIGMOID, want_ck=True)
    assert torch.equal(f["h"][:, t], u[:, t])
    b = adst.recurrence_vjp(av, u, dh, h0=h0, ck=f["ck"], gate=SIGMOID)
    assert bool((b["da"][:, t] == 0).all())
    if t == 0:  # nothing of h0 is left (later it is seen by the steps before)
        assert bool((b["dh0"] == 0).all())
    zeros = torch.zeros_like(h0)
    rest = adst.recurrence(av[:, t:], u[:, t:], h0=zeros, gate=SIGMOID)
    close = (f["h"][:, t:].double() - rest["h"].double()).abs()
    # the same steps, joined in other spans: two roundings to the type and some in 32 bits
    unit = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    assert bool((close <= 2 * unit * rest["h"].double().abs() + 1e-3).all())
    pool = torch.full((2, 70), float("inf"), device="cuda")
    pool[1] = 1e37
    one = adst.recurrence_step(av[1:, t], u[1:, t], pool,
                               slots=torch.tensor([1], dtype=torch.int32, device="cuda"),
                               gate=SIGMOID)
    assert torch.equal(one, u[1:, t]) and torch.equal(pool[1], u[1, t].float())


@pytest.mark.parametrize("dtype", HALVES)
def test_gates_over_the_range(dtype):
    """One step from h0 = 1 with u = 0 is the gate itself, and from h0 = 0 with u = 1 its rest:
    against 64 bits within |a| units of 2^-24 and a few, one rounding, and the smallest normal
    32-bit value."""
    a = torch.cat([torch.linspace(-130, 130, 5200), torch.tensor([float("inf"), -float("inf"),
                                                                   0.0, -0.0])]).to(dtype)
    n = a.numel()
    zero, one = torch.zeros(1, 1, n, dtype=dtype), torch.ones(1, 1, n, dtype=dtype)
    x = a.view(1, 1, n).cuda()
    s = adst.recurrence(x, zero.cuda(), h0=torch.ones(1, n, device="cuda"), gate=SIGMOID)["hT"]
    q = adst.recurrence(x, one.cuda(), h0=torch.zeros(1, n, device="cuda"), gate=SIGMOID)["hT"]
    for got, z in ((s, a.double()), (q, -a.double())):
        want = torch.sigmoid(z)
        bound = (16 + 4 * z.abs().nan_to_num(0, 0, 0)) * 2.0 ** -24 * want + 2.0 ** -126
        assert bool(((got[0].double().cpu() - want).abs() <= bound).all())


def test_a_nan_stays():
    for dtype in HALVES:
        a = torch.tensor([[[float("nan"), 1.0]]], dtype=dtype, device="cuda")
        got = adst.recurrence(a, torch.ones_like(a), gate=SIGMOID)["h"]
        assert torch.isnan(got[0, 0]).tolist() == [True, False]
