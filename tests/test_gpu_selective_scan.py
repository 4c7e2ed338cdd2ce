"""The selective scan, its VJP and its one-step form against the definition in 64 bits on the host,
within bounds derived from the roundings of the accumulation type (tests/token_util.py)."""
import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util
from tests import token_util as ref

pytestmark = pytest.mark.gpu
OF_TYPE = ("y", "dx", "ddelta", "dz", "dB", "dC")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(B, T, D, N, dtype, groups=1, seed=0, optional=True, ragged=False):
    g = torch.Generator().manual_seed(seed)
    acc = ref.acc_of(dtype)

    def normal(*shape, kind=dtype, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale + shift).to(kind).cuda()

    s = {"x": normal(B, T, D), "delta": normal(B, T, D, shift=-1.0),
         "A": -normal(D, N, kind=acc, scale=0.7).exp(), "B": normal(B, T, groups, N),
         "C": normal(B, T, groups, N), "dy": normal(B, T, D)}
    more = {"D": None, "z": None, "delta_bias": None, "h0": None, "lens": None, "dhT": None}
    if optional:
        more.update(D=normal(D, kind=acc), z=normal(B, T, D),
                    delta_bias=normal(D, kind=acc, scale=0.5), h0=normal(B, D, N, kind=acc),
                    dhT=normal(B, D, N, kind=acc))
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        n[0], n[-1] = T, (0 if B > 1 else T)
        more["lens"] = n.cuda()
    return s, more


def run(case, ck=True, softplus=True):
    s, more = case
    opt = {k: v for k, v in more.items() if k != "dhT"}
    f = adst.selective_scan(s["x"], s["delta"], s["A"], s["B"], s["C"], want_ck=True,
                            softplus=softplus, **opt)
    r = adst.selective_scan_vjp(s["x"], s["delta"], s["A"], s["B"], s["C"], s["dy"], **more,
                                ck=f["ck"] if ck else None, softplus=softplus)
    return {"y": f["y"], "hT": f["hT"], **r}


def check(case, got=None, softplus=True):
    s, more = case
    got = got or run(case, softplus=softplus)
    want = ref.scan(s["x"], s["delta"], s["A"], s["B"], s["C"], softplus=softplus, dy=s["dy"], **more)
    want = {k: ((v[0].view(got[k].shape), v[1].view(got[k].shape))) for k, v in want.items()}
    ref.check(got, want, s["x"].dtype, OF_TYPE)
    for k, v in got.items():
        assert (v is None) == (k not in want), k
    return got


# states of each layout, chunks and slabs that end unevenly, several segments from 256 steps on
SHAPES = [(1, 1, 1, 1), (2, 3, 5, 3), (1, 17, 33, 4), (3, 16, 64, 8), (2, 40, 31, 16),
          (1, 33, 40, 17), (2, 21, 7, 32), (1, 11, 35, 33), (2, 9, 10, 64), (1, 300, 40, 16),
          (2, 600, 3, 5), (1, 1025, 2, 2), (40, 2, 3, 16)]


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("B,T,D,N", SHAPES)
def test_against_the_definition(B, T, D, N, dtype):
    check(make(B, T, D, N, dtype, seed=B + T + D + N))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D,N", [(7, 33, 65), (20, 5, 128), (270, 2, 100)])
def test_many_states(T, D, N, dtype):
    check(make(2, T, D, N, dtype))


@pytest.mark.parametrize("dtype", [torch.float64, torch.float16])
@pytest.mark.parametrize("groups,D", [(2, 64), (3, 99), (5, 5), (4, 260)])
def test_groups(groups, D, dtype):
    check(make(2, 19, D, 6, dtype, groups=groups))


@pytest.mark.parametrize("dtype", seq_util.TYPES)
def test_nothing_optional_and_plain_steps(dtype):
    case = make(2, 50, 40, 16, dtype, optional=False)
    s = case[0]
    s["delta"] = s["delta"].abs() * 0.2
    check(case, softplus=False)


@pytest.mark.parametrize("left_out", ["D", "z", "delta_bias", "h0", "dhT"])
def test_without_one_of_the_optional_inputs(left_out):
    case = make(2, 37, 40, 16, torch.float32)
    case[1][left_out] = None
    check(case)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,D,N", [(6, 40, 70, 16), (4, 600, 9, 5), (5, 33, 33, 64), (1, 5, 3, 2)])
def test_ragged_rows_read_nothing_beyond_their_length(B, T, D, N, dtype):
    case = make(B, T, D, N, dtype, ragged=True)
    s, more = case
    for b, n in enumerate(more["lens"].tolist()):
        for t in (s["x"], s["delta"], s["B"], s["C"], s["dy"], more["z"]):
            t[b, n:] = float("nan")
    got = check(case)
    for b, n in enumerate(more["lens"].tolist()):
        assert all(bool((got[k][b, n:] == 0).all()) for k in OF_TYPE)
        if n == 0:
            assert torch.equal(got["hT"][b], more["h0"][b])
            assert torch.equal(got["dh0"][b], more["dhT"][b])


def test_lengths_outside_the_steps_are_clamped():
    case = make(3, 40, 20, 16, torch.float32)
    case[1]["lens"] = torch.tensor([-5, 100, 7], dtype=torch.int32, device="cuda")
    check(case)


@pytest.mark.parametrize("B,T,D", [(0, 5, 4), (3, 0, 4), (3, 5, 0)])
def test_empty_extents(B, T, D):
    case = make(B, T, D, 16, torch.float32)
    got = run(case)
    assert got["y"].shape == (B, T, D) and got["dB"].shape == (B, T, 1, 16)
    for k in ("dA", "dD", "ddelta_bias", "dB", "dC"):
        assert bool((got[k] == 0).all()), k
    if T == 0:
        assert torch.equal(got["hT"], case[1]["h0"]) and torch.equal(got["dh0"], case[1]["dhT"])


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("how", ["halves", "steps first", "offset", "repeated", "no groups"])
def test_strides(how, dtype):
    B, T, D, N = 3, 70, 77, 6
    case = make(B, T, D, N, dtype)
    s, more = case
    if how == "halves":
        both = torch.cat([s["x"], more["z"], s["delta"], s["dy"]], 2)
        s["x"], more["z"], s["delta"], s["dy"] = both.split(D, 2)
        bc = torch.cat([s["B"], s["C"]], 3)
        s["B"], s["C"] = bc[..., :N], bc[..., N:]
    elif how == "steps first":
        for d, k in ((s, "x"), (s, "delta"), (s, "dy"), (s, "B"), (s, "C"), (more, "z")):
            d[k] = d[k].transpose(0, 1).contiguous().transpose(0, 1)
    elif how == "offset":
        for d, k in ((s, "x"), (s, "delta"), (s, "dy"), (s, "B"), (s, "C"), (more, "z")):
            flat = torch.zeros(d[k].numel() + 1, dtype=dtype, device="cuda")
            flat[1:] = d[k].reshape(-1)
            d[k] = flat[1:].view(d[k].shape)
    elif how == "repeated":
        s["delta"] = s["delta"][:1, :1].expand(B, T, D)
        s["B"] = s["B"][:, :1].expand(B, T, 1, N)
        s["dy"] = s["dy"][:1].expand(B, T, D)
    else:
        s["B"], s["C"] = s["B"].squeeze(2), s["C"].squeeze(2)
    check(case)


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("T,N", [(50, 16), (2500, 5), (700, 64)])
def test_the_same_bits_each_time_and_without_checkpoints(T, N, dtype):
    case = make(2, T, 50, N, dtype, ragged=True)
    one = run(case)
    for ck in (True, False, True):
        two = run(case, ck=ck)
        assert all(torch.equal(one[k], two[k]) for k in one)


def test_a_nan_stays_in_its_row_and_channel():
    case = make(2, 300, 70, 16, torch.float32)
    one = run(case)
    case[0]["x"][1, 37, 5] = float("nan")
    two = run(case)
    assert bool(torch.isnan(two["y"][1, 37:, 5]).all()) and bool(torch.isnan(two["dA"][5]).all())
    for k in ("y", "dx", "ddelta"):
        bad = torch.isnan(two[k])
        assert not bool(bad[0].any()) and not bool(bad[1, :, :5].any() | bad[1, :, 6:].any()), k
        good = ~bad
        good[1, :, 5] = False
        assert torch.equal(one[k][good], two[k][good]), k
    rest = [i for i in range(70) if i != 5]
    assert torch.equal(one["dA"][rest], two["dA"][rest])
    assert torch.equal(one["dB"][0], two["dB"][0])


def test_far_values_of_the_inputs():
    """Steps from nothing to what forgets a state at once, gates from closed to wide open."""
    case = make(2, 60, 40, 16, torch.float32)
    s, more = case
    s["delta"][:, ::3] *= 12
    more["z"][:, ::5] *= 40
    check(case)


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("N,groups", [(1, 1), (3, 1), (4, 2), (6, 1), (16, 1), (31, 2), (64, 1)])
def test_steps_against_the_definition(N, groups, dtype):
    """Three rows on a pool of six, step after step: each against the definition from the state
    that the step before left."""
    case = make(3, 4, 22, N, dtype, groups=groups)
    s, more = case
    pool = torch.randn(6, 22, N, dtype=ref.acc_of(dtype), device="cuda")
    slots = torch.tensor([4, 0, 3], dtype=torch.int32, device="cuda")
    for t in range(4):
        now = {k: v[:, t:t + 1] for k, v in s.items() if k not in ("A", "dy")}
        h = pool[slots.long()].clone()
        keep = pool.clone()
        want = ref.scan(now["x"], now["delta"], s["A"], now["B"], now["C"], D=more["D"],
                        z=more["z"][:, t:t + 1], delta_bias=more["delta_bias"], h0=h)
        y = adst.selective_scan_step(s["x"][:, t], s["delta"][:, t], s["A"], s["B"][:, t],
                                     s["C"][:, t], pool, D=more["D"], z=more["z"][:, t],
                                     delta_bias=more["delta_bias"], slots=slots, softplus=True)
        ref.within(y.unsqueeze(1), *want["y"], dtype)
        ref.within(pool[slots.long()], *want["hT"], ref.acc_of(dtype))
        assert torch.equal(pool[[1, 2, 5]], keep[[1, 2, 5]])


def test_128_states_in_a_step():
    test_steps_against_the_definition(128, 1, torch.bfloat16)


def test_idle_rows_of_a_step():
    case = make(5, 1, 9, 4, torch.float32)
    s, more = case
    pool = torch.randn(4, 9, 4, device="cuda")
    keep = pool.clone()
    slots = torch.tensor([-1, 2, 4, 1 << 30, 0], dtype=torch.int32, device="cuda")
    version = pool._version
    y = adst.selective_scan_step(s["x"][:, 0], s["delta"][:, 0], s["A"], s["B"][:, 0],
                                 s["C"][:, 0], pool, slots=slots, softplus=True)
    assert pool._version > version
    assert bool((y[[0, 2, 3]] == 0).all()) and torch.equal(pool[[1, 3]], keep[[1, 3]])
    assert not torch.equal(pool[2], keep[2]) and not torch.equal(pool[0], keep[0])


def test_gradients_against_differences():
    """In float64 with step 1e-6: the truncation is of order 1e-12, the rounding of order
    1e-16 / 1e-6 of a loss of order 100."""
    case = make(2, 11, 4, 3, torch.float64, groups=2)
    s, more = case
    opt = {k: v for k, v in more.items() if k != "dhT"}

    def loss():
        f = adst.selective_scan(s["x"], s["delta"], s["A"], s["B"], s["C"], softplus=True, **opt)
        return float((f["y"] * s["dy"]).sum() + (f["hT"] * more["dhT"]).sum())

    got = run(case)
    for name, t in [(k, s[k]) for k in ("x", "delta", "A", "B", "C")] + \
            [(k, more[k]) for k in ("D", "z", "delta_bias", "h0")]:
        flat = t.view(-1)
        for i in range(0, flat.numel(), 5):
            keep, L = flat[i].item(), []
            for e in (1e-6, -1e-6):
                flat[i] = keep + e
                L.append(loss())
            flat[i] = keep
            assert abs((L[0] - L[1]) / 2e-6 - float(got["d" + name].reshape(-1)[i])) < 1e-6, (name, i)


def test_rows_sums_are_joined_in_64_bits():
    """dA, dD and the bias' gradient are each the sum of dy over 64 rows of one step (A is 0, all
    else is 1): 2^26, 62 ones and -2^26, of which 32 bits lose the ones."""
    n = 64
    one = torch.ones(n, 1, 1, device="cuda")
    dy = one.clone()
    dy[0], dy[-1] = 2.0 ** 26, -2.0 ** 26
    got = adst.selective_scan_vjp(one, torch.zeros_like(one), torch.zeros(1, 1, device="cuda"), one,
                                  one, dy, D=torch.ones(1, device="cuda"),
                                  delta_bias=torch.ones(1, device="cuda"), h0=one)
    for k in ("dA", "dD", "ddelta_bias"):
        assert float(got[k]) == n - 2, k
