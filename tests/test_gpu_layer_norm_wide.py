"""Layer norm's VJP over more columns than one launch has groups of, against the definition."""
import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.gpu


def test_more_columns_than_a_launch_of_the_sums_has_groups():
    """dw and db of n >= 2^26 columns. Their values are sums of two rows' products: with 16-bit
    weights each is rounded once (relative 2^-8, to nearest half of it) after a few roundings in
    32 bits, of values below 64."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    n = (1 << 26) + 77
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.empty(2, n, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
             for _ in range(2))
    f = adst.layer_norm(x)
    got = adst.layer_norm_vjp(x, dy, f["mean"], f["rstd"])
    dw = torch.zeros(n, device="cuda")
    db = torch.zeros(n, device="cuda")
    for r in range(2):
        d = dy[r].float()
        dw += d * ((x[r].float() - f["mean"][r]) * f["rstd"][r])
        db += d
    for k, want in (("dw", dw), ("db", db)):
        off = (got[k].float() - want).abs() - (2.0 ** -8 * want.abs() + 1e-5)
        assert bool((off <= 0).all()), (k, float(off.max()))
