"""The token operators together: the example's layer, its gradients against differences and its
one-token form; in captured graphs, on other streams, with offsets beyond 32 bits, and through both
ways from Python to the C calls."""
import os
import sys

import pytest
import torch

import paper_2509_02197_amd as adst
from tests import token_util as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
import token_layer as ex  # noqa: E402

pytestmark = pytest.mark.gpu
SILU = adst.ADST_ACT_SILU


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    adst.lib()


@pytest.mark.parametrize("ragged", [False, True])
def test_gradients_against_differences(ragged):
    """In float64, with step 1e-6: the truncation is of order 1e-12, the rounding of order
    1e-16 / 1e-6 of the loss."""
    tokens = ex.probe_tokens(2, 20, 2, 11)
    lens = torch.tensor([20, 7, 1, 0], dtype=torch.int32, device="cuda") if ragged else None
    layer = ex.TokenLayer(11, 24, states=5, dtype=torch.float64)
    loss, grads = layer.loss_and_gradients(tokens, lens)
    g = torch.Generator().manual_seed(2)
    for name, grad in grads.items():
        p = {**layer.matrices, **layer.channels}[name].view(-1)
        for i in torch.randint(0, p.numel(), (4,), generator=g).tolist():
            keep = p[i].item()
            L = []
            for e in (1e-6, -1e-6):
                p[i] = keep + e
                L.append(float(layer.loss_and_gradients(tokens, lens)[0]))
            p[i] = keep
            d = (L[0] - L[1]) / 2e-6
            assert abs(d - float(grad.reshape(-1)[i])) <= 1e-8 * (1 + float(loss)), (name, i)


def test_one_token_at_a_time_is_the_whole_row():
    """In float64: sums of at most a hundred terms, whose order differs, in values of order 1,
    through 40 steps whose states forget."""
    tokens = ex.probe_tokens(2, 40, 3, 17)
    layer = ex.TokenLayer(17, 40, dtype=torch.float64)
    whole = layer.forward(tokens[:, :-1])[0].view(6, 40, 40)
    off = (ex.serve(layer, tokens[:, :-1]) - whole).abs().max()
    assert float(off) < 1e-10 * float(whole.abs().max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [32, 8])
def test_the_example_runs(bits, dtype):
    losses, off = ex.train(boxes=2, steps=40, probes=4, words=32, width=64, updates=4, bits=bits,
                           dtype=dtype)
    assert all(v == v and v < 100 for v in losses) and off == off


# ------------------------------------------------------- graphs and streams
def inputs(seed=0, B=3, T=700, D=96, N=16, V=300, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, kind=dtype):
        return torch.randn(*shape, generator=g).to(kind).cuda()

    f = torch.float32
    lens = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32).cuda()
    labels = torch.randint(-1, V, (B * T,), generator=g, dtype=torch.int32).cuda()
    return {"x": normal(B, T, D), "w": normal(4, D, kind=f), "b": normal(D, kind=f),
            "x0": normal(B, 3, D), "delta": normal(B, T, D), "A": -normal(D, N, kind=f).exp(),
            "B": normal(B, T, 2, N), "C": normal(B, T, 2, N), "D": normal(D, kind=f),
            "z": normal(B, T, D), "bias": normal(D, kind=f), "h0": normal(B, D, N, kind=f),
            "dhT": normal(B, D, N, kind=f), "lens": lens, "vocab": normal(V, D), "labels": labels,
            "dloss": normal(B * T, kind=f), "window": normal(5, 3, D),
            "state": normal(5, D, N, kind=f),
            "slots": torch.randperm(5, generator=g)[:B].to(torch.int32).cuda()}


def run(s, **kw):
    """Every call once, the steps on clones of the pools."""
    window, state = s["window"].clone(), s["state"].clone()
    if "stream" in kw:
        kw["stream"].wait_stream(torch.cuda.current_stream())
    conv = dict(x0=s["x0"], lens=s["lens"], act=SILU, **kw)
    scan = dict(D=s["D"], z=s["z"], delta_bias=s["bias"], h0=s["h0"], lens=s["lens"],
                softplus=True, **kw)
    c = adst.causal_conv(s["x"], s["w"], s["b"], **conv)
    f = adst.selective_scan(c["y"], s["delta"], s["A"], s["B"], s["C"], want_ck=True, **scan)
    rows = f["y"].view(-1, f["y"].shape[2])
    e = adst.linear_cross_entropy(rows, s["vocab"], s["labels"], **kw)
    eb = adst.linear_cross_entropy_vjp(rows, s["vocab"], s["labels"], e["lse"], s["dloss"], **kw)
    fb = adst.selective_scan_vjp(c["y"], s["delta"], s["A"], s["B"], s["C"],
                                 eb["dx"].view(f["y"].shape), dhT=s["dhT"], ck=f["ck"], **scan)
    cb = adst.causal_conv_vjp(s["x"], fb["dx"], s["w"], s["b"], dxT=c["xT"], **conv)
    cy = adst.causal_conv_step(s["x"][:, 0], s["w"], window, s["b"], s["slots"], act=SILU, **kw)
    fy = adst.selective_scan_step(cy, s["delta"][:, 0], s["A"], s["B"][:, 0], s["C"][:, 0], state,
                                  D=s["D"], z=s["z"][:, 0], delta_bias=s["bias"],
                                  slots=s["slots"], softplus=True, **kw)
    out = {f"{i}.{k}": v for i, d in enumerate((c, f, e, eb, fb, cb)) for k, v in d.items()}
    return {**out, "window": window, "state": state, "cy": cy, "fy": fy}


def same(one, two):
    for k in one:
        # (checkpoints of chunks beyond a row's length are not written)
        assert k == "1.ck" or torch.equal(one[k], two[k]), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_a_graph(dtype):
    """Captured calls, replayed between eager ones, give the eager results each time; two graphs
    in turn too."""
    graphs = []
    for seed in (0, 7):
        s = inputs(seed, dtype=dtype)
        run(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run(s)
        graphs.append((s, graph, got))
    for seed in (1, 2, 3):
        new = inputs(seed, dtype=dtype)
        want = run(new)
        for s, graph, _ in graphs:
            for k, v in new.items():
                s[k].copy_(v)
            graph.replay()
        run(inputs(seed + 10, dtype=dtype))
        torch.cuda.synchronize()
        for _, _, got in graphs:
            same(want, got)


def test_on_other_streams():
    """Two streams at once, named and as torch's current one: the checked way from Python and
    the native one give the same bits."""
    s = inputs()
    one = run(s)
    torch.cuda.synchronize()
    named, current = torch.cuda.Stream(), torch.cuda.Stream()
    two = run(s, stream=named)
    with torch.cuda.stream(current):
        three = run(s)
    torch.cuda.synchronize()
    same(one, two)
    same(one, three)


def test_the_checked_way_gives_the_native_results():
    s = inputs()
    one = run(s)
    two = run(s, stream=torch.cuda.current_stream())
    same(one, two)


# ----------------------------------------------------- offsets past 32 bits
def test_long_sequences_offsets():
    """2^32 values and more: the last row is what it is alone."""
    B, T, D = 3, 1 << 20, 1400
    x = torch.empty(B, T, D, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(4, D, device="cuda")
    y = adst.causal_conv(x, w, act=SILU)["y"]
    assert torch.equal(y[2:], adst.causal_conv(x[2:], w, act=SILU)["y"])
    r = adst.causal_conv_vjp(x, y, w, act=SILU, want_dw=False, want_db=False)["dx"]
    assert torch.equal(r[2:], adst.causal_conv_vjp(x[2:], y[2:], w, act=SILU)["dx"])
    del r
    A = -torch.rand(D, 2, device="cuda")
    bc = torch.randn(B, T, 4, dtype=torch.bfloat16, device="cuda")
    args = dict(softplus=True, want_ck=True)
    f = adst.selective_scan(x, y, A, bc[..., :2], bc[..., 2:], **args)
    # row 2 three times: a batch of as many rows has as many segments
    x3, y3, bc3 = (torch.cat([t[2:]] * 3) for t in (x, y, bc))
    p = adst.selective_scan(x3, y3, A, bc3[..., :2], bc3[..., 2:], **args)
    assert torch.equal(f["y"][2], p["y"][0]) and torch.equal(f["hT"][2], p["hT"][2])
    g = adst.selective_scan_vjp(x, y, A, bc[..., :2], bc[..., 2:], f["y"], ck=f["ck"],
                                softplus=True)
    h = adst.selective_scan_vjp(x3, y3, A, bc3[..., :2], bc3[..., 2:], p["y"], ck=p["ck"],
                                softplus=True)
    for k in ("dx", "ddelta", "dB", "dC"):
        assert torch.equal(g[k][2], h[k][0]), k


def test_more_logits_than_32_bits_count():
    M, K, V = 70000, 24, 62000
    g = torch.Generator().manual_seed(0)
    x, w = (torch.randn(n, K, generator=g).to(torch.bfloat16).cuda() for n in (M, V))
    labels = torch.randint(0, V, (M,), generator=g, dtype=torch.int32).cuda()
    labels[:-100] = -1  # w's gradient comes from the last rows alone
    f = adst.linear_cross_entropy(x, w, labels)
    r = adst.linear_cross_entropy_vjp(x, w, labels, f["lse"])
    want = ref.xent(x[-100:], w, labels[-100:])
    ref.check({"loss": f["loss"][-100:], "lse": f["lse"][-100:], "dx": r["dx"][-100:],
               "dw": r["dw"]}, want, torch.bfloat16, ("dx", "dw"))
    assert bool((r["dx"][:-100] == 0).all())


# ------------------------------------------------------------------ refusals
def test_refusals():
    s = inputs(T=6, D=4, N=2, V=9)
    x, w, A, B, C = s["x"], s["w"], s["A"], s["B"], s["C"]
    lens64 = torch.zeros(3, dtype=torch.int64, device="cuda")
    odd = torch.zeros(3, 6, 8, dtype=x.dtype, device="cuda")[..., ::2]
    flat, vocab, labels = x.reshape(18, 4), s["vocab"], s["labels"]
    lse = torch.zeros(18, device="cuda")
    for call in (
            lambda: adst.causal_conv(x[0], w), lambda: adst.causal_conv(x, w[:, :3]),
            lambda: adst.causal_conv(x, w.double()), lambda: adst.causal_conv(odd, w),
            lambda: adst.causal_conv(x, w.cpu()), lambda: adst.causal_conv(x, w, lens=lens64),
            lambda: adst.causal_conv(x, w, x0=s["x0"][:, :2]),
            lambda: adst.causal_conv(x, torch.zeros(9, 4, device="cuda")),
            lambda: adst.causal_conv_vjp(x, None, w), lambda: adst.causal_conv_vjp(x, odd, w),
            lambda: adst.causal_conv_step(x[:, 0], w, s["window"][:, :2]),
            lambda: adst.causal_conv_step(x[:, 0], w, s["window"].float()),
            lambda: adst.selective_scan(x, s["delta"], A.double(), B, C),
            lambda: adst.selective_scan(x, s["delta"], A, B, C[..., :1]),
            lambda: adst.selective_scan(x, odd, A, B, C),
            lambda: adst.selective_scan(x, s["delta"], A, B[:, :, :1].repeat(1, 1, 3, 1), C),
            lambda: adst.selective_scan(x, s["delta"], A, B, C, h0=s["h0"].double()),
            lambda: adst.selective_scan_vjp(x, s["delta"], A, B, C, None),
            lambda: adst.selective_scan_vjp(x, s["delta"], A, B, C, x, ck=lse),
            lambda: adst.selective_scan_step(x, s["delta"], A, B, C, s["state"]),
            lambda: adst.selective_scan_step(x[:, 0], s["delta"][:, 0], A, B[:, 0], C[:, 0],
                                             s["state"].double()),
            lambda: adst.linear_cross_entropy(flat, vocab[:, :3], labels),
            lambda: adst.linear_cross_entropy(flat, vocab.float(), labels),
            lambda: adst.linear_cross_entropy(flat, vocab, labels.long()),
            lambda: adst.linear_cross_entropy(flat[::2], vocab, labels),
            lambda: adst.linear_cross_entropy_vjp(flat, vocab, labels, None),
            lambda: adst.linear_cross_entropy_vjp(flat, vocab, labels, lse.double()),
            lambda: adst.linear_cross_entropy_vjp(flat, vocab, labels, lse, lse[:5])):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(adst.AdstError):
        adst.causal_conv(x, w, act=7)
    with pytest.raises(adst.AdstError):
        adst.selective_scan(x, s["delta"], torch.zeros(4, 129, device="cuda"),
                            torch.zeros(3, 6, 129, dtype=x.dtype, device="cuda"),
                            torch.zeros(3, 6, 129, dtype=x.dtype, device="cuda"))


def test_a_batch_without_tokens():
    """Rows of no tokens alone: the mean over none is 0, and so are the gradients."""
    tokens = ex.probe_tokens(1, 12, 3, 11)
    layer = ex.TokenLayer(11, 24)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    loss, grads = layer.loss_and_gradients(tokens, none)
    assert float(loss) == 0
    assert all(bool((g == 0).all()) for g in grads.values())
