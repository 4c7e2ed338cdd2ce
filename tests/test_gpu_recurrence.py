"""The gated linear recurrence, its VJP and its one-step form against the
definition in 64 bits on the host, within bounds derived from the roundings of
the accumulation type (tests/seq_util.py)."""
import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util as ref

pytestmark = pytest.mark.gpu
COEFF, SIGMOID = adst.ADST_GATE_COEFF, adst.ADST_GATE_SIGMOID


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(B, T, D, dtype, gate, seed=0, h0=True, ragged=False):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(B, T, D, generator=g, dtype=torch.float64) * 2 + 1
    if gate == COEFF:
        a = torch.tanh(a)  # negative coefficients among them
    u, dh = (torch.randn(B, T, D, generator=g, dtype=torch.float64) for _ in range(2))
    acc = ref.acc_of(dtype)
    s = {"a": a.to(dtype), "u": u.to(dtype), "dh": dh.to(dtype), "h0": None, "dhT": None,
         "lens": None}
    if h0:
        s["h0"], s["dhT"] = (torch.randn(B, D, generator=g, dtype=torch.float64).to(acc)
                             for _ in range(2))
    if ragged:
        s["lens"] = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        s["lens"][0] = T
        s["lens"][-1] = 0 if B > 1 else T
    return {k: None if v is None else v.cuda() for k, v in s.items()}


def run(s, gate, ck=True):
    f = adst.recurrence(s["a"], s["u"], h0=s["h0"], lens=s["lens"], gate=gate, want_ck=True)
    b = adst.recurrence_vjp(s["a"], s["u"], s["dh"], h0=s["h0"], lens=s["lens"], dhT=s["dhT"],
                            ck=f["ck"] if ck else None, gate=gate)
    return {"h": f["h"], "hT": f["hT"], **b}


def check(s, gate, got):
    want = ref.recurrence(s["a"], s["u"], s["h0"], s["lens"], gate == SIGMOID, s["dh"], s["dhT"])
    dtype = s["a"].dtype
    for k, (value, bound) in want.items():
        ref.within(got[k], value, bound, dtype if k in ("h", "da", "du") else ref.acc_of(dtype))


SHAPES = [(1, 1, 1), (2, 3, 5), (1, 15, 8), (3, 16, 64), (2, 17, 129), (5, 33, 31), (1, 300, 128),
          (2, 257, 16), (2, 1025, 7), (1, 3001, 3), (1, 700, 515), (3, 128, 1000), (130, 2, 2)]


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("B,T,D", SHAPES)
def test_against_the_definition(B, T, D, dtype, gate):
    s = make(B, T, D, dtype, gate, seed=B + T + D)
    check(s, gate, run(s, gate))


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
@pytest.mark.parametrize("dtype", [torch.float64, torch.bfloat16])
@pytest.mark.parametrize("B,T,D", [(6, 40, 70), (7, 600, 33), (4, 2100, 9), (1, 50, 3)])
def test_ragged_rows_read_nothing_beyond_their_length(B, T, D, dtype, gate):
    s = make(B, T, D, dtype, gate, ragged=True)
    for b, n in enumerate(s["lens"].tolist()):
        for k in ("a", "u", "dh"):
            s[k][b, n:] = float("nan")
    got = run(s, gate)
    assert all(bool(torch.isfinite(v).all()) for v in got.values())
    check(s, gate, got)
    for b, n in enumerate(s["lens"].tolist()):
        assert all(bool((got[k][b, n:] == 0).all()) for k in ("h", "da", "du"))
        if n == 0:
            assert torch.equal(got["hT"][b], s["h0"][b])
            assert torch.equal(got["dh0"][b], s["dhT"][b])


def test_lengths_outside_the_steps_are_clamped():
    s = make(3, 40, 20, torch.float32, SIGMOID)
    s["lens"] = torch.tensor([-5, 100, 7], dtype=torch.int32, device="cuda")
    check(s, SIGMOID, run(s, SIGMOID))


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
def test_without_initial_state_and_last_gradient(gate):
    s = make(2, 500, 40, torch.float32, gate, h0=False)
    check(s, gate, run(s, gate))


@pytest.mark.parametrize("B,T,D", [(0, 5, 4), (3, 0, 4), (3, 5, 0)])
def test_empty_extents(B, T, D):
    s = make(B, T, D, torch.float32, COEFF)
    got = run(s, COEFF)
    assert got["h"].shape == got["da"].shape == (B, T, D)
    if T == 0:
        assert torch.equal(got["hT"], s["h0"]) and torch.equal(got["dh0"], s["dhT"])


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("how", ["halves", "steps first", "offset", "repeated"])
def test_strides(how, dtype):
    B, T, D = 3, 290, 77
    s = make(B, T, D, dtype, SIGMOID)
    if how == "halves":
        both = torch.cat([s["a"], s["u"], s["dh"]], 2)
        s["a"], s["u"], s["dh"] = both[..., :D], both[..., D:2 * D], both[..., 2 * D:]
    elif how == "steps first":
        for k in ("a", "u", "dh"):
            s[k] = s[k].transpose(0, 1).contiguous().transpose(0, 1)
    elif how == "offset":  # rows that start one element into an aligned buffer
        for k in ("a", "u", "dh"):
            flat = torch.zeros(B * T * D + 1, dtype=dtype, device="cuda")
            flat[1:] = s[k].reshape(-1)
            s[k] = flat[1:].view(B, T, D)
    else:
        s["a"] = s["a"][:1, :1].expand(B, T, D)
        s["dh"] = s["dh"][:, :1].expand(B, T, D)
    check(s, SIGMOID, run(s, SIGMOID))


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_the_same_bits_each_time_and_without_checkpoints(dtype, gate):
    s = make(3, 2500, 150, dtype, gate, ragged=True)
    one = run(s, gate)
    for ck in (True, False, True):
        two = run(s, gate, ck=ck)
        assert all(torch.equal(one[k], two[k]) for k in one)


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
def test_rows_and_channels_are_independent(gate):
    """A NaN stays in its channel from its step on; other values keep their bits."""
    s = make(2, 900, 70, torch.float32, gate)
    one = run(s, gate)
    s["u"][1, 450, 33] = float("nan")
    two = run(s, gate)
    hit = torch.zeros_like(one["h"], dtype=torch.bool)
    hit[1, 450:, 33] = True
    assert torch.equal(torch.isnan(two["h"]), hit)
    assert torch.equal(two["h"][~hit], one["h"][~hit])
    assert torch.equal(two["du"], one["du"])  # G does not depend on u
    hit[1, 450, 33] = gate == SIGMOID  # da reads h_{t-1}, and u_t behind the gate
    assert torch.equal(torch.isnan(two["da"]), hit)
    assert torch.equal(two["da"][~hit], one["da"][~hit])


@pytest.mark.parametrize("B", [3, 4, 5, 9, 33])
def test_a_row_is_the_same_alone(B):
    """Whatever the number of rows, and so of the workgroups' chains and where they run."""
    s = make(B, 900, 250, torch.bfloat16, SIGMOID, seed=B)
    got = run(s, SIGMOID)
    for b in (0, B // 2, B - 1):
        one = run({k: None if v is None else v[b:b + 1] for k, v in s.items()}, SIGMOID)
        assert all(torch.equal(got[k][b:b + 1], one[k]) for k in one)


def test_extreme_gates():
    """Gates at and beyond the type's range: 0 and 1 exactly, no NaN."""
    z = torch.tensor([-1e30, -200.0, -90.0, 0.0, 90.0, 200.0, 1e30, float("inf"), -float("inf")])
    s = make(1, 9, 6, torch.float32, SIGMOID)
    s["a"] = z.view(1, 9, 1).expand(1, 9, 6).contiguous().cuda()
    got = run(s, SIGMOID)
    check(s, SIGMOID, got)
    assert torch.equal(got["h"][:, 0], s["u"][:, 0])      # s = 0: the state is replaced
    assert all(bool(torch.isfinite(v).all()) for v in got.values())


def test_a_zero_coefficient_starts_over():
    s = make(2, 800, 20, torch.float32, COEFF)
    s["a"][:, 400] = 0
    got = run(s, COEFF)
    part = {k: v[:, 400:].contiguous() if v.dim() == 3 else v for k, v in s.items()
            if v is not None}
    check(s, COEFF, got)
    assert torch.equal(got["h"][:, 400], s["u"][:, 400])
    tail = adst.recurrence(part["a"], part["u"])["h"]
    bound = ref.recurrence(part["a"], part["u"], None, None, False)["h"]
    ref.within(tail, bound[0], bound[1], torch.float32)


@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
def test_gradients_against_differences(gate):
    """Central differences of L = <h, W> + <hT, V> in float64: with step 1e-6 their truncation is
    about 1e-12 of the third derivative, their rounding 1e-16 |L| / 1e-6."""
    s = make(2, 37, 3, torch.float64, gate)
    s["lens"] = torch.tensor([37, 30], dtype=torch.int32, device="cuda")
    got = run(s, gate)

    def loss(**over):
        f = adst.recurrence(over.get("a", s["a"]), over.get("u", s["u"]),
                            h0=over.get("h0", s["h0"]), lens=s["lens"], gate=gate)
        return float((f["h"] * s["dh"]).sum() + (f["hT"] * s["dhT"]).sum())

    size = float((got["h"] * s["dh"]).abs().sum() + (got["hT"] * s["dhT"]).abs().sum())
    g = torch.Generator().manual_seed(5)
    for name, grad in (("a", "da"), ("u", "du"), ("h0", "dh0")):
        for _ in range(12):
            i = int(torch.randint(0, s[name].numel(), (1,), generator=g))
            L = []
            for e in (1e-6, -1e-6):
                v = s[name].clone()
                v.view(-1)[i] += e
                L.append(loss(**{name: v}))
            d = (L[0] - L[1]) / 2e-6
            assert abs(d - float(got[grad].reshape(-1)[i])) <= 1e-9 * (1 + size)


def test_gradient_of_a_repeated_input_is_its_uses():
    s = make(4, 60, 10, torch.float64, SIGMOID)
    full = s["a"][:1].expand(4, 60, 10).contiguous()
    one = run({**s, "a": s["a"][:1].expand(4, 60, 10)}, SIGMOID)
    two = run({**s, "a": full}, SIGMOID)
    assert all(torch.equal(one[k], two[k]) for k in one)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("B,D", [(1, 1), (5, 33), (64, 2048), (3, 515)])
@pytest.mark.parametrize("gate", [COEFF, SIGMOID])
def test_steps_are_the_recurrence(B, D, dtype, gate):
    """Tokens one at a time against the definition, the states in a pool."""
    T = 5
    s = make(B, T, D, dtype, gate)
    pool = torch.full((2 * B + 1, D), 7.0, dtype=ref.acc_of(dtype), device="cuda")
    slots = torch.randperm(2 * B + 1)[:B].to(torch.int32).cuda()
    pool[slots.long()] = s["h0"]
    rest = torch.ones(2 * B + 1, dtype=torch.bool, device="cuda")
    rest[slots.long()] = False
    hs = [adst.recurrence_step(s["a"][:, t], s["u"][:, t], pool, slots, gate) for t in range(T)]
    want = ref.recurrence(s["a"], s["u"], s["h0"], None, gate == SIGMOID)
    ref.within(torch.stack(hs, 1), *want["h"], dtype)
    ref.within(pool[slots.long()], *want["hT"], ref.acc_of(dtype))
    assert bool((pool[rest] == 7.0).all())


def test_idle_slots():
    s = make(4, 1, 40, torch.float32, COEFF)
    pool = s["h0"].clone()
    slots = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device="cuda")
    h = adst.recurrence_step(s["a"][:, 0], s["u"][:, 0], pool, slots, COEFF)
    assert bool((h[1:3] == 0).all())
    assert torch.equal(pool[1], s["h0"][1]) and torch.equal(pool[3], s["h0"][3])
    assert torch.equal(pool[2], h[0]) and torch.equal(pool[0], h[3])
    pool = s["h0"].clone()
    h = adst.recurrence_step(s["a"][:, 0], s["u"][:, 0], pool, None, COEFF)
    assert torch.equal(pool, h)


def test_offsets_beyond_32_bits():
    """Outputs of more than 2^31 values; the inputs repeat, so every row has the first one's."""
    B, T, D = 34, 65536, 1000
    s = make(1, T, D, torch.bfloat16, SIGMOID, h0=False)
    a, u, dh = (s[k].expand(B, T, D) for k in ("a", "u", "dh"))
    f = adst.recurrence(a, u, gate=SIGMOID, want_ck=True)
    b = adst.recurrence_vjp(a, u, dh, ck=f["ck"], gate=SIGMOID)
    one = run(s, SIGMOID)
    for row in (0, 17, B - 1):
        for k, v in (("h", f["h"]), ("da", b["da"]), ("du", b["du"])):
            assert torch.equal(v[row], one[k][0]), (k, row)


def test_on_another_stream():
    s = make(4, 3000, 256, torch.float32, SIGMOID)
    one = run(s, SIGMOID)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    f = adst.recurrence(s["a"], s["u"], h0=s["h0"], gate=SIGMOID, want_ck=True, stream=side)
    b = adst.recurrence_vjp(s["a"], s["u"], s["dh"], h0=s["h0"], dhT=s["dhT"], ck=f["ck"],
                            gate=SIGMOID, stream=side)
    side.synchronize()
    for k in one:
        assert torch.equal(one[k], {**f, **b}[k])


def test_in_a_graph():
    """Captured calls, replayed between eager ones, give the eager results each time."""
    s = make(3, 1500, 200, torch.bfloat16, SIGMOID, ragged=True)
    run(s, SIGMOID)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(s, SIGMOID)
    for seed in (1, 2, 3):
        new = make(3, 1500, 200, torch.bfloat16, SIGMOID, seed=seed, ragged=True)
        for k, v in new.items():
            s[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        want = run(new, SIGMOID)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_refusals():
    s = make(2, 6, 4, torch.float32, COEFF)
    a, u, dh = s["a"], s["u"], s["dh"]
    odd = torch.zeros(2, 6, 8, device="cuda")[..., ::2]
    wide = torch.zeros(2, 5, device="cuda")
    lens = torch.zeros(2, dtype=torch.int64, device="cuda")
    for call in (lambda: adst.recurrence(a[0], u[0]), lambda: adst.recurrence(a, u[:, :5]),
                 lambda: adst.recurrence(a, u.double()), lambda: adst.recurrence(odd, u),
                 lambda: adst.recurrence(a, odd), lambda: adst.recurrence(a, u.cpu()),
                 lambda: adst.recurrence(a, u, h0=wide), lambda: adst.recurrence(a, u, lens=lens),
                 lambda: adst.recurrence(a, u, h0=s["h0"].double()),
                 lambda: adst.recurrence_vjp(a, u, None), lambda: adst.recurrence_vjp(a, u, odd),
                 lambda: adst.recurrence_vjp(a, u, dh, dhT=wide),
                 lambda: adst.recurrence_vjp(a, u, dh, ck=torch.zeros(3, device="cuda")),
                 lambda: adst.recurrence_step(a, u, s["h0"]),
                 lambda: adst.recurrence_step(a[:, 0], u[:, 0], wide),
                 lambda: adst.recurrence_step(a[:, 0], u[:, 0], s["h0"].t().contiguous().t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: adst.recurrence(a, u, gate=7),
                 lambda: adst.recurrence_step(a[:, 0], u[:, 0], s["h0"][:1])):
        with pytest.raises(adst.AdstError):
            call()
