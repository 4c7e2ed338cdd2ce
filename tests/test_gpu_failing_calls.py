"""Calls around which HIP reports an error. The error is one that the host makes: an invalid
device number, which HIP refuses and keeps as the thread's last error."""
import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def leave_an_error():
    assert adst.lib().hipSetDevice(9999) != 0


def attempt(call):
    """Whether it raised AdstError."""
    try:
        call()
    except adst.AdstError as e:
        assert e.status == adst.ADST_ERR_HIP
        return True
    finally:
        adst.lib().hipGetLastError()
    return False


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_updates_once(bits):
    g = [torch.randn(n, device="cuda") for n in (5, 1000, 300)]
    one, two = (adst.AdamW([x.clone() for x in g], bits=bits, lr=0.1) for _ in range(2))
    for opt, before in ((one, lambda: None), (two, leave_an_error)):
        opt.step(g)
        before()
        attempt(lambda: opt.step(g))
        torch.cuda.synchronize()
    for name in ("params", "m", "v"):
        for a, b in zip(getattr(one, name), getattr(two, name)):
            assert torch.equal(a.float(), b.float())


def test_a_step_advances_the_states_once():
    a, u, state = (torch.randn(4, 40, device="cuda") for _ in range(3))
    one, two = state.clone(), state.clone()
    adst.recurrence_step(a, u, one)
    adst.recurrence_step(a, u, two)
    adst.recurrence_step(a, u, one)
    leave_an_error()
    attempt(lambda: adst.recurrence_step(a, u, two))
    assert torch.equal(one, two)


def test_an_earlier_error_is_not_a_calls_own():
    """The calls report their own launches, and leave the thread's last error to whom it belongs."""
    L = adst.lib()
    x, y, dx = (torch.randn(6, 300, device="cuda") for _ in range(3))
    w, dw, db = (torch.randn(300, device="cuda") for _ in range(3))
    mean, rstd = (torch.empty(6, device="cuda") for _ in range(2))
    norm = adst.adst_norm_problem(adst.ADST_F32, adst.ADST_F32, 6, 300, 300, 300, 1e-5)
    T = 3000  # several spans: the board is filled by a launch of its own
    rec = adst.adst_recurrence_problem(adst.ADST_F32, adst.ADST_GATE_SIGMOID, 2, T, 70,
                                       *([T * 70, 70] * 3))
    one = adst.adst_recurrence_problem(adst.ADST_F32, adst.ADST_GATE_SIGMOID, 2, 1, 70,
                                       *([T * 70, 70] * 3))
    a, u, h, da, du = (torch.randn(2, T, 70, device="cuda") for _ in range(5))
    info = adst.adst_recurrence_plan(rec)
    ck, ws, nws = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in
                   (info.ck_bytes, info.vjp_workspace_bytes,
                    adst.adst_layer_norm_workspace_bytes(norm)))
    state = torch.zeros(2, 70, device="cuda")
    p, m, v, g = (torch.ones(500, device="cuda") for _ in range(4))
    tensors = (adst.adst_adamw_tensor * 1)(
        adst.adst_adamw_tensor(p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), None, None,
                               None, 500, 0.1, 0.0))
    adamw = adst.adst_adamw_problem(adst.ADST_F32, adst.ADST_F32, adst.ADST_F32, 32, 1, 0.9, 0.99,
                                    1e-8, None)
    for call in (
            lambda: adst.adst_layer_norm_forward(norm, x, w, w, y, mean, rstd),
            lambda: adst.adst_layer_norm_vjp(norm, x, y, w, mean, rstd, dx, dw, db, nws,
                                             nws.numel()),
            lambda: adst.adst_recurrence_forward(rec, a, u, None, None, h, None, ck, ws,
                                                 ws.numel()),
            lambda: adst.adst_recurrence_vjp(rec, a, u, None, None, None, h, None, da, du, None,
                                             ws, ws.numel()),
            lambda: adst.adst_recurrence_step(one, a, u, None, state, 2, y),
            lambda: adst.adst_adamw(adamw, tensors, 1)):
        torch.cuda.current_stream()
        leave_an_error()
        call()
        assert L.hipGetLastError() != 0
        assert L.hipGetLastError() == 0
    assert bool((p < 1).all())
