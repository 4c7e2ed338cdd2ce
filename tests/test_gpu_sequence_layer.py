"""The operators together: the example's layer, its gradients against
differences, its training, and its one-record form."""
import os
import sys

import pytest
import torch

import paper_2509_02197_amd as adst

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
import sequence_layer as ex  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def test_gradients_against_differences():
    """In float64, with step 1e-6: the truncation is of order 1e-12, the rounding of order
    1e-16 / 1e-6 of the loss."""
    records = ex.probe_records(3, 20, 7).double()
    layer = ex.SequenceLayer(7, 24, dtype=torch.float64)
    loss, grads = layer.loss_and_gradients(records)
    g = torch.Generator().manual_seed(2)
    for name, grad in zip(layer.names, grads):
        p = layer.held[name].view(-1)
        for i in torch.randint(0, p.numel(), (4,), generator=g).tolist():
            keep = p[i].item()
            L = []
            for e in (1e-6, -1e-6):
                p[i] = keep + e
                L.append(float(layer.loss_and_gradients(records)[0]))
            p[i] = keep
            d = (L[0] - L[1]) / 2e-6
            assert abs(d - float(grad.reshape(-1)[i])) <= 1e-8 * (1 + float(loss)), (name, i)


@pytest.mark.parametrize("bits", [32, 8])
def test_training_lowers_the_loss_and_serving_agrees(bits):
    """Outputs are a few times 1 in bfloat16 (one part in 256 each), through two norms and a
    product: a tenth is far above their roundings and far below an error of state."""
    losses, off, y = ex.train(batch=8, steps=64, probes=16, width=96, updates=40, bits=bits)
    assert losses[-1] < 0.7 * losses[0]
    assert off < 0.1 * max(1.0, float(y.abs().max()))


def test_coefficients_are_recovered():
    losses, first, last = ex.fit_coefficients(n=64, steps=30, updates=40)
    assert losses[-1] < 0.2 * losses[0] and last < first
