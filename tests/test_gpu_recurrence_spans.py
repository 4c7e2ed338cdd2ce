"""The recurrence where rows have dozens to hundreds of spans, in many groups, and where calls
are so large that their accesses are non-temporal: against the definition in 64 bits, within
bounds derived from the roundings (tests/seq_util.py)."""
import pytest
import torch

from tests import seq_util as ref
from tests.test_gpu_recurrence import COEFF, SIGMOID, _gpu, check, make, run  # noqa: F401

pytestmark = pytest.mark.gpu


def held(B, T, D, dtype, seed=0, ragged=False):
    """States that last: coefficients of 1 and inputs of 0, but for one step in some 500 of each
    channel. A state is then carried over whole groups of spans, and the bound stays near it."""
    s = make(B, T, D, dtype, COEFF, seed, ragged=ragged)
    g = torch.Generator().manual_seed(seed + 1)
    rare = (torch.rand(B, T, D, generator=g) < 0.002).cuda()
    s["a"] = torch.where(rare, s["a"], torch.ones_like(s["a"]))
    for k in ("u", "dh"):
        s[k] = torch.where(rare.roll(7, 1), s[k], torch.zeros_like(s[k]))
    return s


# 64 channels: spans of 128 steps (64 in double precision and in the 16-bit types' reverse
# sweep), so up to 1250 spans in 157 groups; a look back reaches 32 groups.
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_states_that_last_over_many_groups(dtype):
    s = held(1, 40000, 64, dtype)
    check(s, COEFF, run(s, COEFF))


# 5 channels: rows of 16 lanes, whose spans are four times as long
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_states_that_last_in_few_channels(dtype):
    s = held(2, 40000, 5, dtype, ragged=True)
    check(s, COEFF, run(s, COEFF))


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_many_spans(dtype, gate):
    s = make(1, 12000, 64, dtype, gate)
    check(s, gate, run(s, gate))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_spans_of_ragged_rows(dtype):
    s = make(4, 9000, 150, dtype, SIGMOID, ragged=True)
    check(s, SIGMOID, run(s, SIGMOID, ck=False))
    s = held(4, 9000, 150, dtype, ragged=True)
    check(s, COEFF, run(s, COEFF))


# More than 128 MiB moved, rows of whole cache lines: several spans, and one of 512 and of 256
# threads. Some channels of a row are compared with the definition, and the row with a call of
# its own, which is small.
LARGE = {torch.float64: [(3, 2048, 1024), (100, 60, 1024), (200, 30, 1024)],
         torch.float32: [(3, 4096, 1024), (100, 120, 1024), (200, 60, 1024)],
         torch.bfloat16: [(6, 4096, 1024), (200, 120, 1024), (400, 60, 1024)],
         torch.float16: [(6, 4096, 1024), (200, 120, 1024), (400, 60, 1024)]}


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_large_calls(dtype, which, gate):
    B, T, D = LARGE[dtype][which]
    size = torch.empty(0, dtype=dtype).element_size()
    assert 3 * B * T * D * size >= 128 << 20 and D * size % 128 == 0
    small = make(2, T, D, dtype, gate, seed=which)  # two rows, repeated
    s = {k: None if v is None else v.repeat(B // 2 + 1, *[1] * (v.dim() - 1))[:B]
         for k, v in small.items()}
    assert all(s[k].data_ptr() % 128 == 0 for k in ("a", "u", "dh"))
    got, one = run(s, gate), run(small, gate)
    for k in one:
        for b in range(B):
            assert torch.equal(got[k][b], one[k][b % 2]), (k, b)
    some = slice(0, 1024, 97)
    part = {k: None if v is None else v[..., some].contiguous() for k, v in small.items()}
    check(part, gate, {k: v[..., some] for k, v in one.items()})
