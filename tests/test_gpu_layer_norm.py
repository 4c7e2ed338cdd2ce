"""Layer norm and its VJP against the definition in 64 bits on the host, within
bounds derived from the roundings of the accumulation type (tests/seq_util.py)."""
import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(rows, n, dtype, wdtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, n, generator=g, dtype=torch.float64) * 1.5 + \
        torch.randn(rows, 1, generator=g, dtype=torch.float64)
    w, b = (torch.randn(n, generator=g, dtype=torch.float64) for _ in range(2))
    dy = torch.randn(rows, n, generator=g, dtype=torch.float64)
    return x.to(dtype).cuda(), w.to(wdtype).cuda(), b.to(wdtype).cuda(), dy.to(dtype).cuda()


def run(x, w, b, dy, eps=EPS):
    f = adst.layer_norm(x, w, b, eps)
    return {**f, **adst.layer_norm_vjp(x, dy, f["mean"], f["rstd"], w)}


def check(x, w, b, dy, got, eps=EPS):
    wdtype = x.dtype if w is None else w.dtype
    for k, (value, bound) in ref.layer_norm(x, w, b, eps, dy).items():
        ref.within(got[k], value, bound,
                   {"dw": wdtype, "db": wdtype, "mean": ref.acc_of(x.dtype),
                    "rstd": ref.acc_of(x.dtype)}.get(k, x.dtype))


SHAPES = [(1, 1), (3, 2), (1, 7), (130, 8), (5, 64), (67, 100), (300, 129), (9, 515), (33, 1024),
          (4, 2047), (17, 4096), (2, 9000), (3, 20011), (2, 40000), (700, 33), (1025, 48)]


@pytest.mark.parametrize("dtype,wdtype", [(t, t) for t in ref.TYPES] +
                         [(torch.bfloat16, torch.float32), (torch.float16, torch.float32)])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_against_the_definition(rows, n, dtype, wdtype):
    s = make(rows, n, dtype, wdtype, rows + n)
    check(*s, run(*s))


@pytest.mark.parametrize("rows,n", [(5, 70), (3, 5000)])
def test_without_weights(rows, n):
    x, _, _, dy = make(rows, n, torch.float32, torch.float32)
    check(x, None, None, dy, run(x, None, None, dy))


def test_constant_rows():
    """No spread: the result is the bias and every gradient is finite."""
    x, w, b, dy = make(4, 300, torch.float32, torch.float32)
    x.fill_(1000.0)
    got = run(x, w, b, dy)
    assert torch.equal(got["y"], b.expand(4, 300))
    assert all(bool(torch.isfinite(v).all()) for v in got.values())


def test_a_large_mean_keeps_its_digits():
    x, w, b, dy = make(6, 1000, torch.float32, torch.float32)
    x += 3000.0
    check(x, w, b, dy, run(x, w, b, dy))


@pytest.mark.parametrize("n", [60, 1000, 20000])
def test_rows_are_independent(n):
    x, w, b, dy = make(9, n, torch.float32, torch.float32)
    one = run(x, w, b, dy)
    x[4, n // 2] = float("inf")
    two = run(x, w, b, dy)
    keep = torch.arange(9) != 4
    for k in ("y", "dx", "mean", "rstd"):
        assert torch.equal(one[k][keep], two[k][keep])
    assert bool(torch.isnan(two["y"][4]).all())
    assert torch.equal(one["db"], two["db"])


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_strides(dtype):
    """Rows apart from each other, and starting at any element."""
    x, w, b, dy = make(40, 77, dtype, dtype)
    one = run(x, w, b, dy)
    wide = torch.zeros(40, 200, dtype=dtype, device="cuda")
    wide[:, 1:78], wide[:, 101:178] = x, dy
    two = run(wide[:, 1:78], w, b, wide[:, 101:178])
    assert all(torch.equal(one[k], two[k]) for k in one)
    three = run(x.view(5, 8, 77), w, b, dy.view(5, 8, 77))
    assert three["y"].shape == (5, 8, 77) and three["mean"].shape == (5, 8)
    assert all(torch.equal(one[k], three[k].view(one[k].shape)) for k in one)
    row = run(x[:1].expand(40, 77), w, b, dy)
    assert bool((row["y"] == row["y"][0]).all())


def test_the_outputs_that_are_asked_for():
    x, w, b, dy = make(50, 300, torch.bfloat16, torch.float32)
    f = adst.layer_norm(x, w, b, EPS)
    every = adst.layer_norm_vjp(x, dy, f["mean"], f["rstd"], w)
    for k in ("dx", "dw", "db"):
        want = {f"want_{o}": o == k for o in ("dx", "dw", "db")}
        got = adst.layer_norm_vjp(x, dy, f["mean"], f["rstd"], w, **want)
        assert torch.equal(got[k], every[k])
        assert all(v is None for o, v in got.items() if o != k)


def test_no_rows():
    x, w, b, dy = make(0, 30, torch.float32, torch.float32)
    got = run(x, w, b, dy)
    assert got["y"].shape == (0, 30) and bool((got["dw"] == 0).all() & (got["db"] == 0).all())


def test_in_place():
    x, w, b, _ = make(30, 200, torch.bfloat16, torch.bfloat16)
    want = adst.layer_norm(x, w, b, EPS)["y"]
    prob = adst.adst_norm_problem(adst.ADST_BF16, adst.ADST_BF16, 30, 200, 200, 200, EPS)
    adst.adst_layer_norm_forward(prob, x, w, b, x, None, None)
    assert torch.equal(x, want)


def test_gradients_against_differences():
    x, w, b, dy = make(3, 19, torch.float64, torch.float64)
    got = run(x, w, b, dy)
    s = {"x": x, "w": w, "b": b}
    size = float((got["y"] * dy).abs().sum())
    g = torch.Generator().manual_seed(5)
    for name in s:
        for _ in range(10):
            i = int(torch.randint(0, s[name].numel(), (1,), generator=g))
            L = []
            for e in (1e-6, -1e-6):
                v = s[name].clone()
                v.view(-1)[i] += e
                a = {**s, name: v}
                L.append(float((adst.layer_norm(a["x"], a["w"], a["b"], EPS)["y"] * dy).sum()))
            d = (L[0] - L[1]) / 2e-6
            assert abs(d - float(got["d" + name].reshape(-1)[i])) <= 1e-9 * (1 + size)


@pytest.mark.parametrize("rows,n", [(3000, 40), (5000, 700), (40, 20000)])
def test_the_same_bits_each_time(rows, n):
    s = make(rows, n, torch.bfloat16, torch.float32)
    one = run(*s)
    for _ in range(3):
        two = run(*s)
        assert all(torch.equal(one[k], two[k]) for k in one)


def test_many_rows():
    """More rows than any workspace holds sums for, and 2^31 values: rows repeat, so each has the
    first one's result and the weights' gradients are the first one's times the rows (a power of
    two of them, and small integers, so that every order of summing is exact)."""
    n, rows = 1024, 1 << 21
    x = torch.randn(1, n, device="cuda").to(torch.bfloat16)
    dy = torch.randint(-2, 3, (1, n), device="cuda").to(torch.bfloat16)
    w = torch.ones(n, device="cuda")
    f = adst.layer_norm(x.expand(rows, n), w, None, EPS)
    one = adst.layer_norm(x, w, None, EPS)
    assert torch.equal(f["y"][-1], one["y"][0]) and torch.equal(f["y"][rows // 2 + 1], one["y"][0])
    b = adst.layer_norm_vjp(x.expand(rows, n), dy.expand(rows, n), f["mean"], f["rstd"], w)
    c = adst.layer_norm_vjp(x, dy, one["mean"], one["rstd"], w)
    assert torch.equal(b["dx"][-1], c["dx"][0])
    assert torch.equal(b["db"], c["db"] * rows)


@pytest.mark.parametrize("dtype,rows,n", [
    (torch.bfloat16, 11003, 2056), (torch.float16, 5501, 4104), (torch.bfloat16, 2801, 8200),
    (torch.bfloat16, 1130, 20000), (torch.float32, 5501, 2060), (torch.float32, 11003, 1032),
    (torch.float32, 2801, 4100), (torch.float32, 701, 16000)])
def test_large_calls(dtype, rows, n):
    """Calls that request their rows ahead of their use: a row's results are those of a small call,
    and the weights' gradients those of rows that start off a 16-byte boundary."""
    g = torch.Generator("cuda").manual_seed(n)
    x, dy = (torch.randn(rows, n, generator=g, device="cuda").to(dtype) for _ in range(2))
    w, b = (torch.randn(n, generator=g, device="cuda").to(dtype) for _ in range(2))
    one = run(x, w, b, dy)
    for r in (slice(0, 40), slice(rows // 2, rows // 2 + 33), slice(rows - 40, rows)):
        few = run(x[r], w, b, dy[r])
        assert all(torch.equal(one[k][r], few[k]) for k in ("y", "mean", "rstd", "dx"))
    wide = torch.zeros(rows, n + 9, dtype=dtype, device="cuda")
    wide[:, 1:n + 1] = x
    off = adst.layer_norm_vjp(wide[:, 1:n + 1], dy, one["mean"], one["rstd"], w)
    assert all(torch.equal(one[k], off[k]) for k in ("dx", "dw", "db"))
    wide = torch.zeros(rows, n + 16, dtype=dtype, device="cuda")
    wide[:, 8:n + 8] = dy
    apart = adst.layer_norm_vjp(x, wide[:, 8:n + 8], one["mean"], one["rstd"], w)
    assert all(torch.equal(one[k], apart[k]) for k in ("dx", "dw", "db"))
    only = adst.layer_norm_vjp(x, dy, one["mean"], one["rstd"], w, want_dx=False)
    assert all(torch.equal(one[k], only[k]) for k in ("dw", "db"))


def test_a_large_call_against_the_definition():
    s = make(11003, 2056, torch.bfloat16, torch.float32, 3)
    check(*s, run(*s))


def test_on_another_stream():
    s = make(2000, 1500, torch.bfloat16, torch.float32)
    one = run(*s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    f = adst.layer_norm(s[0], s[1], s[2], EPS, stream=side)
    b = adst.layer_norm_vjp(s[0], s[3], f["mean"], f["rstd"], s[1], stream=side)
    side.synchronize()
    assert all(torch.equal(one[k], {**f, **b}[k]) for k in one)


def test_in_a_graph():
    s = make(900, 300, torch.bfloat16, torch.float32)
    run(*s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(*s)
    for seed in (1, 2, 3):
        new = make(900, 300, torch.bfloat16, torch.float32, seed)
        for old, v in zip(s, new):
            old.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        want = run(*new)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_refusals():
    x, w, b, dy = make(4, 30, torch.float32, torch.float32)
    f = adst.layer_norm(x, w, b, EPS)
    odd = torch.zeros(4, 60, device="cuda")[:, ::2]
    uneven = torch.zeros(2, 5, 40, device="cuda")[:, :3, :30]
    for call in (lambda: adst.layer_norm(odd), lambda: adst.layer_norm(uneven),
                 lambda: adst.layer_norm(x, w[:9]), lambda: adst.layer_norm(x, w, b.double()),
                 lambda: adst.layer_norm(x, w.to(torch.bfloat16)),
                 lambda: adst.layer_norm(x, w.cpu()),
                 lambda: adst.layer_norm(torch.zeros(3, 0, device="cuda")),
                 lambda: adst.layer_norm_vjp(x, None, f["mean"], f["rstd"], w),
                 lambda: adst.layer_norm_vjp(x, odd, f["mean"], f["rstd"], w),
                 lambda: adst.layer_norm_vjp(x, dy, None, f["rstd"], w),
                 lambda: adst.layer_norm_vjp(x, dy, f["mean"][:2], f["rstd"], w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(adst.AdstError):
        adst.layer_norm(x, w, b, -1.0)
