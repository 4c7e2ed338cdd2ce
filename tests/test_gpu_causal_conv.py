"""The causal convolution, its VJP and its one-step form against the definition in 64 bits on the
host, within bounds derived from the roundings of the accumulation type (tests/token_util.py)."""
import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util
from tests import token_util as ref

pytestmark = pytest.mark.gpu
NONE, SILU = adst.ADST_ACT_NONE, adst.ADST_ACT_SILU


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(B, T, D, K, dtype, wtype=None, seed=0, x0=True, bias=True, ragged=False):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, kind=dtype):
        return torch.randn(*shape, generator=g, dtype=torch.float64).to(kind).cuda()

    wtype = wtype or dtype
    s = {"x": normal(B, T, D), "dy": normal(B, T, D), "w": normal(K, D, kind=wtype),
         "b": normal(D, kind=wtype) if bias else None,
         "x0": normal(B, K - 1, D) if x0 else None, "dxT": normal(B, K - 1, D) if x0 else None,
         "lens": None}
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        n[0], n[-1] = T, (0 if B > 1 else T)
        s["lens"] = n.cuda()
    return s


def run(s, act):
    f = adst.causal_conv(s["x"], s["w"], s["b"], x0=s["x0"], lens=s["lens"], act=act)
    r = adst.causal_conv_vjp(s["x"], s["dy"], s["w"], s["b"], x0=s["x0"], lens=s["lens"],
                             dxT=s["dxT"], act=act)
    return {**f, **r}


def check(s, act, got=None):
    got = got or run(s, act)
    want = ref.conv(s["x"], s["w"], s["b"], s["x0"], s["lens"], act == SILU, s["dy"], s["dxT"])
    t, wt = s["x"].dtype, s["w"].dtype
    ref.check(got, want, t, {"y": t, "xT": t, "dx": t, "dx0": t, "dw": wt, "db": wt})
    return got


@pytest.mark.parametrize("act", [NONE, SILU])
@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("B,T,D,K", [(1, 1, 1, 4), (2, 3, 5, 4), (1, 33, 8, 2), (3, 70, 129, 3),
                                     (2, 64, 64, 1), (1, 130, 31, 8), (5, 35, 260, 5),
                                     (2, 300, 7, 6), (130, 2, 3, 7), (1, 4097, 2, 4)])
def test_against_the_definition(B, T, D, K, dtype, act):
    check(make(B, T, D, K, dtype, seed=B + T + D + K), act)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weights_in_single_precision(dtype):
    check(make(2, 50, 70, 4, dtype, torch.float32), SILU)


@pytest.mark.parametrize("act", [NONE, SILU])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,D,K", [(6, 40, 70, 4), (5, 200, 9, 8), (1, 5, 3, 4), (4, 2, 20, 8)])
def test_ragged_rows_read_nothing_beyond_their_length(B, T, D, K, dtype, act):
    s = make(B, T, D, K, dtype, ragged=True)
    for b, n in enumerate(s["lens"].tolist()):
        s["x"][b, n:] = float("nan")
        s["dy"][b, n:] = float("nan")
    got = check(s, act)
    for b, n in enumerate(s["lens"].tolist()):
        assert bool((got["y"][b, n:] == 0).all()) and bool((got["dx"][b, n:] == 0).all())
        if n == 0:
            assert torch.equal(got["xT"][b], s["x0"][b]) and torch.equal(got["dx0"][b], s["dxT"][b])


def test_lengths_outside_the_steps_are_clamped():
    s = make(3, 40, 20, 4, torch.float32)
    s["lens"] = torch.tensor([-5, 100, 7], dtype=torch.int32, device="cuda")
    check(s, SILU)


def test_without_window_and_bias():
    check(make(2, 50, 40, 4, torch.float32, x0=False, bias=False), SILU)


@pytest.mark.parametrize("B,T,D", [(0, 5, 4), (3, 0, 4), (3, 5, 0)])
def test_empty_extents(B, T, D):
    s = make(B, T, D, 4, torch.float32)
    got = run(s, SILU)
    assert got["y"].shape == (B, T, D) and got["dw"].shape == (4, D)
    assert bool((got["dw"] == 0).all()) and bool((got["db"] == 0).all())
    if T == 0:
        assert torch.equal(got["xT"], s["x0"]) and torch.equal(got["dx0"], s["dxT"])


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("how", ["halves", "steps first", "offset", "repeated"])
def test_strides(how, dtype):
    B, T, D = 3, 90, 77
    s = make(B, T, D, 4, dtype)
    if how == "halves":
        both = torch.cat([s["x"], s["dy"]], 2)
        s["x"], s["dy"] = both[..., :D], both[..., D:]
    elif how == "steps first":
        for k in ("x", "dy"):
            s[k] = s[k].transpose(0, 1).contiguous().transpose(0, 1)
    elif how == "offset":  # rows that start one element into an aligned buffer
        for k in ("x", "dy"):
            flat = torch.zeros(B * T * D + 1, dtype=dtype, device="cuda")
            flat[1:] = s[k].reshape(-1)
            s[k] = flat[1:].view(B, T, D)
    else:
        s["x"] = s["x"][:1, :1].expand(B, T, D)
        s["dy"] = s["dy"][:, :1].expand(B, T, D)
    check(s, SILU)


@pytest.mark.parametrize("dtype", seq_util.TYPES)
def test_pieces_of_a_row_and_steps_are_the_whole_row(dtype):
    """In pieces through windows, and one step at a time on a pool, the same bits; the VJP in
    pieces through dxT gives the whole one's dx."""
    s = make(3, 37, 45, 4, dtype)
    whole = run(s, SILU)
    ys, x0 = [], s["x0"]
    for t in (0, 10, 11):
        e = {0: 10, 10: 11, 11: 37}[t]
        f = adst.causal_conv(s["x"][:, t:e], s["w"], s["b"], x0=x0, act=SILU)
        ys.append(f["y"])
        x0 = f["xT"]
    assert torch.equal(torch.cat(ys, 1), whole["y"]) and torch.equal(x0, whole["xT"])
    pool = torch.zeros(7, 3, 45, dtype=dtype, device="cuda")
    slots = torch.tensor([5, 0, 3], dtype=torch.int32, device="cuda")
    pool[slots.long()] = s["x0"]
    keep = pool.clone()
    y = torch.stack([adst.causal_conv_step(s["x"][:, t], s["w"], pool, s["b"], slots, act=SILU)
                     for t in range(37)], 1)
    assert torch.equal(y, whole["y"]) and torch.equal(pool[slots.long()], whole["xT"])
    rest = [i for i in range(7) if i not in (5, 0, 3)]
    assert torch.equal(pool[rest], keep[rest])


def test_idle_rows_of_a_step():
    x, w = torch.randn(5, 9, device="cuda"), torch.randn(3, 9, device="cuda")
    pool = torch.randn(4, 2, 9, device="cuda")
    keep = pool.clone()
    slots = torch.tensor([-1, 2, 4, 1 << 30, 0], dtype=torch.int32, device="cuda")
    version = pool._version
    y = adst.causal_conv_step(x, w, pool, slots=slots)
    assert pool._version > version
    assert bool((y[[0, 2, 3]] == 0).all()) and torch.equal(pool[[1, 3]], keep[[1, 3]])
    want = keep[2, 0] * w[0] + keep[2, 1] * w[1] + x[1] * w[2]
    torch.testing.assert_close(y[1], want, rtol=1e-5, atol=1e-5)
    assert torch.equal(pool[2], torch.stack([keep[2, 1], x[1]]))


def test_the_same_bits_each_time():
    s = make(4, 700, 300, 4, torch.bfloat16, torch.float32, ragged=True)
    one = run(s, SILU)
    for _ in range(3):
        two = run(s, SILU)
        assert all(torch.equal(one[k], two[k]) for k in one)


def test_gradients_against_differences():
    """In float64 with step 1e-6: the truncation is of order 1e-12, the rounding of order
    1e-16 / 1e-6 of a loss of order 100."""
    s = make(2, 9, 5, 4, torch.float64)

    def loss():
        f = adst.causal_conv(s["x"], s["w"], s["b"], x0=s["x0"], act=SILU)
        return float((f["y"] * s["dy"]).sum() + (f["xT"] * s["dxT"]).sum())

    got = run(s, SILU)
    for name, grad in (("x", "dx"), ("w", "dw"), ("b", "db"), ("x0", "dx0")):
        flat = s[name].view(-1)
        for i in range(0, flat.numel(), 7):
            keep, L = flat[i].item(), []
            for e in (1e-6, -1e-6):
                flat[i] = keep + e
                L.append(loss())
            flat[i] = keep
            assert abs((L[0] - L[1]) / 2e-6 - float(got[grad].view(-1)[i])) < 1e-6, (name, i)


def test_workgroups_sums_are_joined_in_64_bits():
    """A long row's dw and db: one value of 2^26 at its start, one of -2^26 at its end and 62 ones
    in between, 8192 steps apart, where workgroups of their own sum them up exactly. 32 bits lose
    the ones beside 2^26."""
    far, n = 8192, 64
    x = torch.ones(1, far * n, 1, device="cuda")
    dy = torch.zeros_like(x)
    dy[0, ::far, 0] = 1.0
    dy[0, 0, 0], dy[0, -far, 0] = 2.0 ** 26, -2.0 ** 26
    got = adst.causal_conv_vjp(x, dy, torch.ones(1, 1, device="cuda"))
    assert float(got["db"]) == n - 2 and float(got["dw"]) == n - 2
