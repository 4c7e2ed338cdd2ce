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
