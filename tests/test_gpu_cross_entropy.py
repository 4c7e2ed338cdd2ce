"""The vocabulary's cross entropy and its VJP against the definition in 64 bits on the host, within
bounds derived from the roundings of the accumulation type and of g (tests/token_util.py)."""
import pytest
import torch

import paper_2509_02197_amd as adst
from tests import seq_util
from tests import token_util as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


def make(M, K, V, dtype, seed=0, ignored=0.2, mean=True, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g, dtype=torch.float64).to(dtype).cuda()
    w = (torch.randn(V, K, generator=g, dtype=torch.float64) * scale / K ** 0.5).to(dtype).cuda()
    labels = torch.randint(0, V, (M,), generator=g)
    drop = torch.rand(M, generator=g) < ignored
    labels[drop] = torch.tensor([-1, -100, V, 1 << 30])[torch.arange(int(drop.sum())) % 4]
    acc = ref.acc_of(dtype)
    dloss = (torch.full((M,), 0.37) if mean else torch.randn(M, generator=g)).to(acc).cuda()
    return {"x": x, "w": w, "labels": labels.to(torch.int32).cuda(), "dloss": dloss}


def run(s):
    f = adst.linear_cross_entropy(s["x"], s["w"], s["labels"])
    return {**f, **adst.linear_cross_entropy_vjp(s["x"], s["w"], s["labels"], f["lse"], s["dloss"])}


def check(s):
    got = run(s)
    want = ref.xent(s["x"], s["w"], s["labels"], s["dloss"])
    ref.check(got, want, s["x"].dtype, ("dx", "dw"))
    return got


# tiles of every size: few rows, few words, splits of the long axis, whole and odd steps of it
SHAPES = [(1, 1, 1), (3, 5, 7), (64, 64, 64), (65, 63, 66), (17, 200, 1000), (130, 128, 257),
          (300, 33, 2), (2, 70, 3000), (257, 512, 300), (700, 16, 90), (129, 65, 129)]


@pytest.mark.parametrize("mean", [True, False])
@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("M,K,V", SHAPES)
def test_against_the_definition(M, K, V, dtype, mean):
    check(make(M, K, V, dtype, seed=M + K + V, mean=mean))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K,V", [(2048, 128, 6400), (2048, 131, 6401), (3000, 64, 4500)])
def test_large_tiles(M, K, V, dtype):
    check(make(M, K, V, dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_several_pieces_of_the_vocabulary(dtype):
    """More rows than one piece of 128 MB of g has of a vocabulary: the exact values are taken of
    every 64th row and word, and of all words' sums against dx."""
    size = 4 if dtype == torch.float32 else 2
    M, K, V = (128 << 20) // size // 1024, 32, 2100  # 1024 words a piece
    s = make(M, K, V, dtype)
    prob = adst.adst_xent_problem({4: 1, 2: 2}[size], 0, M, K, V, K, K)
    assert adst.adst_linear_cross_entropy_plan(prob).vjp_workspace_bytes < 4 * M * V * size
    got = run(s)
    some = slice(0, None, 64)
    part = {k: s[k][some] for k in ("x", "labels", "dloss")}
    want = ref.xent(part["x"], s["w"], part["labels"], part["dloss"])
    for k in ("loss", "lse", "dx"):
        ref.within(got[k][some], *want[k], dtype if k == "dx" else torch.float32)
    # dw of all rows, on the GPU in 64 bits
    x, w = s["x"].double(), s["w"].double()
    g = torch.softmax(x @ w.T, 1)
    ok = (s["labels"] >= 0) & (s["labels"] < V)
    rows = torch.arange(M, device="cuda")[ok]
    g[rows, s["labels"][ok].long()] -= 1
    g *= torch.where(ok, s["dloss"].double(), 0.0)[:, None]
    size_of = (g.abs().T @ x.abs()).cpu()
    unit = seq_util.UNIT[dtype] if size == 2 else 0.0
    # logits within (K + 2) units of at most 2 |x| |w| <= 64, p within twice that
    bound = (unit + 2 * (K + 2) * 2.0 ** -24 * 64 + (M + 8) * 2.0 ** -24) * size_of
    ref.within(got["dw"], (g.T @ x).cpu(), bound, dtype)


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("M,K,V", [(1, 64, 9000), (7, 131, 12000), (16, 128, 8200), (17, 96, 8200)])
def test_few_rows_of_many_words(M, K, V, dtype):
    s = make(M, K, V, dtype, seed=M + K, mean=False)
    one = check(s)
    two = run(s)
    assert all(torch.equal(one[k], two[k]) for k in one)


# few logits from long rows, whose product is split along them
FEW = [(1, 2048, 300), (5, 4014, 728), (157, 1100, 19), (1044, 1918, 9), (64, 1536, 4096),
       (4000, 1030, 64), (65, 2100, 257), (3, 1024, 1)]


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("M,K,V", FEW)
def test_few_logits(M, K, V, dtype):
    s = make(M, K, V, dtype, seed=M + K + V, mean=False)
    one = check(s)
    two = run(s)
    assert all(torch.equal(one[k], two[k]) for k in one)


def test_few_logits_of_rows_that_take_no_part():
    s = make(200, 2070, 300, torch.bfloat16, ignored=0.3, mean=False)  # 33 steps, 20 tiles
    off = (s["labels"] < 0) | (s["labels"] >= 300)
    clean = run(s)
    s["x"][off] = float("nan")
    s["dloss"][off] = float("inf")
    got = run(s)
    assert bool((got["loss"][off] == 0).all()) and bool((got["dx"][off] == 0).all())
    assert torch.equal(got["dw"], clean["dw"]) and torch.equal(got["dx"], clean["dx"])
    assert torch.equal(got["loss"][~off], clean["loss"][~off])


@pytest.mark.parametrize("V", [3, 700])
def test_few_logits_that_are_infinite(V):
    """Rows of 1024: +inf, -inf alone, and -inf beside finite ones."""
    x, w = torch.zeros(3, 1024, device="cuda"), torch.zeros(V, 1024, device="cuda")
    w[:, 0] = 3e38
    x[0, 0], x[1, 0] = 3.0, -3.0
    w[0, 2], w[1:, 1] = -3e38, 2.0
    x[2, 2], x[2, 1] = 3.0, 1.0
    labels = torch.tensor([0, 0, 1], dtype=torch.int32, device="cuda")
    f = adst.linear_cross_entropy(x, w, labels)
    want = torch.tensor([float("inf"), float("-inf"),
                         2.0 + torch.log(torch.tensor(V - 1.0))], device="cuda")
    assert torch.equal(torch.isinf(f["lse"]), torch.isinf(want))
    assert bool((f["lse"][:2] == want[:2]).all()) and abs(float(f["lse"][2] - want[2])) < 1e-5
    assert abs(float(f["loss"][2]) - float(want[2] - 2)) < 1e-5


def test_rows_without_a_label_take_no_part_whatever_they_hold():
    s = make(200, 70, 300, torch.bfloat16, ignored=0.3, mean=False)
    off = (s["labels"] < 0) | (s["labels"] >= 300)
    zero = torch.zeros(200, dtype=torch.bool, device="cuda")
    zero[::7] = True
    s["dloss"][zero] = 0.0
    clean = run(s)
    s["x"][off | zero] = float("nan")
    s["dloss"][off] = float("inf")
    got = run(s)
    assert bool((got["loss"][off] == 0).all()) and bool((got["dx"][off | zero] == 0).all())
    assert torch.equal(got["dw"], clean["dw"]) and torch.equal(got["dx"], clean["dx"])
    keep = ~(off | zero)
    assert torch.equal(got["loss"][keep], clean["loss"][keep])


def test_all_rows_without_a_label():
    s = make(70, 40, 130, torch.float16)
    s["labels"].fill_(-1)
    got = run(s)
    assert all(bool((got[k] == 0).all()) for k in ("loss", "dx", "dw"))


@pytest.mark.parametrize("dtype", seq_util.TYPES)
def test_far_logits(dtype):
    """Logits of hundreds: nothing overflows, and a label far below the largest has a loss of
    that distance."""
    s = make(40, 64, 200, dtype, scale=60.0)
    got = check(s)
    assert float(got["loss"].max()) > 100


def test_infinite_logits():
    x = torch.tensor([[1.0, 0.0], [1.0, 0.0], [0.0, 1.0]], device="cuda")
    w = torch.tensor([[3.4e38, 1.0], [3.4e38, 2.0], [-3.4e38, 3.0]], device="cuda") * 1.0
    x[0] *= 10  # logits inf, inf, -inf
    x[1] *= -10
    labels = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    f = adst.linear_cross_entropy(x, w, labels)
    want = torch.logsumexp((x.double() @ w.double().T).float().double(), 1)
    assert torch.equal(torch.isinf(f["lse"]), torch.isinf(want))
    assert abs(float(f["lse"][2]) - float(want[2])) < 1e-5
    one = adst.linear_cross_entropy(x[:1], torch.full((70, 2), -3.4e38, device="cuda"),
                                    labels[:1])
    assert float(one["lse"]) == float("-inf")


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("how", ["rows apart", "offset", "repeated"])
def test_strides(how, dtype):
    s = make(150, 64, 200, dtype)
    if how == "rows apart":
        for k in ("x", "w"):
            wide = torch.full((s[k].shape[0], 64 + 3), float("nan"), dtype=dtype, device="cuda")
            wide[:, :64] = s[k]
            s[k] = wide[:, :64]
    elif how == "offset":
        for k in ("x", "w"):
            flat = torch.zeros(s[k].numel() + 1, dtype=dtype, device="cuda")
            flat[1:] = s[k].reshape(-1)
            s[k] = flat[1:].view(s[k].shape)
    else:
        s["x"] = s["x"][:1].expand(150, 64)
    check(s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [28, 27, 26])
def test_rows_gigabytes_apart(bits, dtype):
    """Offsets of neighbouring rows that pass 32 bits, within a wave's eight rows too; strides on
    both sides of 2^28 bytes."""
    s = make(9, 64, 11, dtype)
    for k, stride in (("x", 1 << bits), ("w", 1 << bits)) if bits > 27 else \
            (("x", (1 << bits) - 64), ("w", (1 << bits) - 128)):
        rows = s[k].shape[0]
        flat = torch.empty((rows - 1) * stride + 64, dtype=dtype, device="cuda")
        far = flat.as_strided((rows, 64), (stride, 1))
        far.copy_(s[k])
        s[k] = far
    check(s)


def test_each_gradient_alone_and_no_dloss():
    s = make(90, 40, 130, torch.float32)
    f = adst.linear_cross_entropy(s["x"], s["w"], s["labels"])
    args = (s["x"], s["w"], s["labels"], f["lse"])
    both = adst.linear_cross_entropy_vjp(*args)
    ones = adst.linear_cross_entropy_vjp(*args, torch.ones(90, device="cuda"))
    dx = adst.linear_cross_entropy_vjp(*args, want_dw=False)
    dw = adst.linear_cross_entropy_vjp(*args, want_dx=False)
    assert dx["dw"] is None and dw["dx"] is None
    for k in ("dx", "dw"):
        assert torch.equal(both[k], ones[k]) and torch.equal(both[k], {"dx": dx, "dw": dw}[k][k])


def test_no_rows():
    s = make(0, 8, 20, torch.bfloat16)
    got = run(s)
    assert got["loss"].shape == (0,) and got["dx"].shape == (0, 8)
    assert got["dw"].shape == (20, 8) and bool((got["dw"] == 0).all())


@pytest.mark.parametrize("dtype", seq_util.TYPES)
def test_the_same_bits_each_time(dtype):
    s = make(400, 96, 1500, dtype, mean=False)
    one = run(s)
    for _ in range(3):
        two = run(s)
        assert all(torch.equal(one[k], two[k]) for k in one)


def test_gradients_against_differences():
    """In float64 with step 1e-6: the truncation is of order 1e-12, the rounding of order
    1e-16 / 1e-6 of a loss of order 10."""
    s = make(6, 5, 9, torch.float64, mean=False)

    def loss():
        f = adst.linear_cross_entropy(s["x"], s["w"], s["labels"])
        return float((f["loss"] * s["dloss"]).sum())

    got = run(s)
    for name in ("x", "w"):
        flat = s[name].view(-1)
        for i in range(flat.numel()):
            keep, L = flat[i].item(), []
            for e in (1e-6, -1e-6):
                flat[i] = keep + e
                L.append(loss())
            flat[i] = keep
            assert abs((L[0] - L[1]) / 2e-6 - float(got["d" + name].view(-1)[i])) < 1e-7, (name, i)


@pytest.mark.parametrize("dtype", seq_util.TYPES)
@pytest.mark.parametrize("K", [1, 8, 255, 256, 512, 1535, 1536, 2048])
def test_no_rows_at_any_width(K, dtype):
    """Widths on both sides of where the logits' product is split, which without rows has no tiles."""
    got = run(make(0, K, 20, dtype))
    assert got["loss"].shape == got["lse"].shape == (0,) and got["dx"].shape == (0, K)
    assert got["dw"].shape == (20, K) and bool((got["dw"] == 0).all())


@pytest.mark.parametrize("dtype,least", [(torch.bfloat16, 2.0 ** -20), (torch.float16, 2.0 ** -20),
                                         (torch.float32, 2.0 ** -30)])
def test_rows_of_unequal_weights(dtype, least):
    """A row's dx is as exact as it would be alone, however much larger another row's weight is:
    g of 40000 equal probabilities is off by one rounding to the type, relative to each. Rows
    of zeros have equal logits, and so p = 1 / V to 4 roundings."""
    M, K, V = 40, 32, 40000
    g = torch.Generator().manual_seed(5)
    x = torch.zeros(M, K, dtype=dtype, device="cuda")
    w = (torch.rand(V, K, generator=g, dtype=torch.float64) + 0.5).to(dtype).cuda()
    labels = torch.randint(0, V, (M,), generator=g).to(torch.int32).cuda()
    dloss = torch.full((M,), least, device="cuda")
    dloss[7] = 1.0
    dloss *= 512.0
    got = adst.linear_cross_entropy_vjp(x, w, labels, adst.linear_cross_entropy(x, w, labels)["lse"],
                                        dloss)["dx"]
    wd = w.double()
    want = (wd.mean(0) - wd[labels.long()]) * dloss.double()[:, None]
    unit = seq_util.UNIT[dtype] if dtype != torch.float32 else 0.0
    size = wd.mean(0) + wd[labels.long()]  # sum of |g| w, for a weight of 1
    bound = (unit + (V + 32) * 2.0 ** -24) * size * dloss.double()[:, None]
    ref.within(got, want.cpu(), bound.cpu(), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_label_s_entry_is_exact_for_any_weight(dtype):
    """One word is so likely that the others' probabilities are below the type's roundings of
    them, and the label is another one: g is then (dloss, -dloss) times 1 to 4 roundings of 32
    bits, and dx the difference of two words times dloss, whatever the weights."""
    M, K, V = 30, 64, 70
    g = torch.Generator().manual_seed(6)
    w = torch.randn(V, K, generator=g).to(dtype).cuda()
    w[:, 0] = 0
    w[5, 0] = 40.0
    x = torch.zeros(M, K, dtype=dtype, device="cuda")
    x[:, 0] = 1.0
    labels = torch.randint(6, V, (M,), generator=g).to(torch.int32).cuda()
    dloss = (torch.rand(M, generator=g) + 0.1).cuda()
    lse = adst.linear_cross_entropy(x, w, labels)["lse"]
    got = adst.linear_cross_entropy_vjp(x, w, labels, lse, dloss, want_dw=False)["dx"]
    wd, d = w.double(), dloss.double()[:, None]
    want = (wd[5] - wd[labels.long()]) * d
    # the others: exp(-40) each; the exponential's argument of 40 is rounded twice
    bound = ((V + 100) * 2.0 ** -24 + V * 2.0 ** -57) * (wd.abs().max() * 2 * d).expand(M, K)
    ref.within(got, want.cpu(), bound.cpu(), dtype)
