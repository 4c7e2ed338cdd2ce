"""What the token operators refuse, on a host without a GPU: every bad argument is an error before
anything is enqueued (the pointers are never dereferenced)."""
import ctypes

import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="host-only argument checks")
BAD, BIG, SMALL = adst.ADST_ERR_ARG, adst.ADST_ERR_UNSUPPORTED, adst.ADST_ERR_WORKSPACE
MUCH = 1 << 40


def at(i):
    return (i + 1) << 32


def flat(f):
    """Strides by their fields' names."""
    out = {}
    for k, v in f.items():
        out.update({k + "_batch": v[0], k + "_step": v[1]} if isinstance(v, tuple) else {k: v})
    return out


def fails(status, call, *args):
    with pytest.raises(adst.AdstError) as e:
        call(*args)
    assert e.value.status == status, str(e.value)
    assert adst.adst_last_error()


# ------------------------------------------------------------- convolution
def conv(**over):
    f = dict(dtype=adst.ADST_F32, weight_dtype=adst.ADST_F32, act=1, taps=4, batch=2, steps=100,
             channels=8, stride_x=(800, 8), stride_dy=(800, 8))
    f.update(over)
    return adst.adst_conv_problem(**flat(f))


def conv_fwd(prob=None, x=at(0), w=at(1), b=at(2), x0=at(3), lens=at(4), y=at(5), xT=at(6)):
    return prob or conv(), x, w, b, x0, lens, y, xT, 0


def conv_rev(prob=None, x=at(0), dy=at(1), w=at(2), b=at(3), x0=at(4), lens=at(5), dxT=at(6),
             dx=at(7), dw=at(8), db=at(9), dx0=at(10), ws=at(11), n=MUCH):
    return prob or conv(), x, dy, w, b, x0, lens, dxT, dx, dw, db, dx0, ws, n, 0


def conv_one(prob=None, x=at(0), w=at(1), b=at(2), slots=at(3), window=at(4), n=4, y=at(5)):
    return prob or conv(steps=1), x, w, b, slots, window, n, y, 0


@pytest.mark.parametrize("over,status", [
    (dict(dtype=4), BAD), (dict(dtype=-1), BAD), (dict(weight_dtype=adst.ADST_BF16), BAD),
    (dict(dtype=adst.ADST_BF16, weight_dtype=adst.ADST_F16), BAD),
    (dict(dtype=adst.ADST_F64), BAD), (dict(act=2), BAD), (dict(act=-1), BAD), (dict(taps=0), BAD),
    (dict(taps=9), BAD), (dict(batch=-1), BAD), (dict(steps=-1), BAD), (dict(channels=-1), BAD),
    (dict(stride_x=(800, -8)), BAD), (dict(stride_dy=(-1, 8)), BAD), (dict(steps=1 << 31), BIG),
    (dict(batch=1 << 31), BIG), (dict(channels=1 << 26), BIG),
    (dict(batch=1 << 30, channels=1 << 25), BIG)])
def test_conv_problems(over, status):
    p = conv(**over)
    fails(status, adst.adst_causal_conv_forward, *conv_fwd(p))
    fails(status, adst.adst_causal_conv_vjp, *conv_rev(p))
    assert adst.adst_causal_conv_workspace_bytes(p) == 0


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(w=None), dict(x=at(0) + 2), dict(w=at(1) + 1), dict(b=at(2) + 2),
    dict(x0=at(3) + 1), dict(lens=at(4) + 2), dict(y=at(5) + 2), dict(xT=at(6) + 2), dict(y=at(0)),
    dict(y=at(0) + 6396), dict(xT=at(5) + 6396), dict(xT=at(3) + 188), dict(y=at(1)),
    dict(lens=at(5) + 4), dict(xT=at(2))])
def test_conv_forward_arrays(kw):
    fails(BAD, adst.adst_causal_conv_forward, *conv_fwd(**kw))


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(dy=None), dict(w=None), dict(dy=at(1) + 2), dict(dx=at(7) + 1),
    dict(dw=at(8) + 2), dict(db=at(9) + 2), dict(dx0=at(10) + 2), dict(dxT=at(6) + 1),
    dict(dx=at(1)), dict(dx=at(0)), dict(dw=at(2)), dict(db=at(8) + 124), dict(dx0=at(6)),
    dict(ws=at(7)), dict(ws=at(0)), dict(ws=at(11) + 8), dict(lens=at(7))])
def test_conv_vjp_arrays(kw):
    fails(BAD, adst.adst_causal_conv_vjp, *conv_rev(**kw))


def test_conv_workspace():
    need = adst.adst_causal_conv_workspace_bytes(conv())
    assert need >= 5 * 8 * 4
    fails(SMALL, adst.adst_causal_conv_vjp, *conv_rev(n=need - 1))
    fails(SMALL, adst.adst_causal_conv_vjp, *conv_rev(ws=None))
    # a wider row's sums are no more than 1024 workgroups' of it
    wide = conv(batch=64, steps=100000, channels=5000, stride_x=(0, 5000), stride_dy=(0, 5000))
    assert adst.adst_causal_conv_workspace_bytes(wide) < 1024 * 5 * 5000 * 4


@pytest.mark.parametrize("kw,status", [
    (dict(prob=conv()), BAD), (dict(x=None), BAD), (dict(w=None), BAD), (dict(window=None), BAD),
    (dict(n=-1), BAD), (dict(slots=None, n=1), BAD), (dict(y=at(4)), BAD), (dict(window=at(0)), BAD),
    (dict(window=at(4) + 2), BAD), (dict(slots=at(3) + 1), BAD), (dict(slots=at(4) + 64), BAD),
    (dict(prob=conv(steps=1, batch=1 << 10, channels=1 << 21)), BIG)])
def test_conv_step_arguments(kw, status):
    fails(status, adst.adst_causal_conv_step, *conv_one(**kw))


# ---------------------------------------------------------- selective scan
def scan(**over):
    f = dict(dtype=adst.ADST_F32, softplus=1, batch=2, steps=100, channels=8, states=4, groups=2)
    f.update({"stride_" + k: (800, 8) for k in ("x", "delta", "b", "c", "z", "dy")})
    f.update(over)
    return adst.adst_scan_problem(**flat(f))


NAMES = ("x", "delta", "A", "B", "C", "D", "z", "delta_bias", "h0", "lens")
GRADS = ("dx", "ddelta", "dz", "dB", "dC", "dA", "dD", "ddelta_bias", "dh0")


def split(kw, names, first):
    held = {k: at(first + i) for i, k in enumerate(names)}
    held.update({k: kw.pop(k) for k in names if k in kw})
    return held


def scan_fwd(prob=None, y=at(20), hT=at(21), ck=at(22), ws=at(23), n=MUCH, **kw):
    return prob or scan(), adst.adst_scan_inputs(**split(kw, NAMES, 0)), y, hT, ck, ws, n, 0


def scan_rev(prob=None, ck=at(22), dy=at(24), dhT=at(25), ws=at(23), n=MUCH, **kw):
    return (prob or scan(), adst.adst_scan_inputs(**split(kw, NAMES, 0)), ck, dy, dhT,
            adst.adst_scan_gradients(**split(kw, GRADS, 10)), ws, n, 0)


def scan_one(prob=None, slots=at(20), state=at(21), n=4, y=at(22), **kw):
    kw = {"h0": None, "lens": None, **kw}
    return (prob or scan(steps=1), adst.adst_scan_inputs(**split(kw, NAMES, 0)), slots, state, n,
            y, 0)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=4), BAD), (dict(softplus=2), BAD), (dict(batch=-1), BAD), (dict(steps=-1), BAD),
    (dict(channels=-8), BAD), (dict(states=0), BAD), (dict(groups=0), BAD), (dict(groups=3), BAD),
    (dict(groups=16), BAD), (dict(states=129), BIG), (dict(dtype=adst.ADST_F64, states=65), BIG),
    (dict(steps=1 << 31), BIG), (dict(channels=1 << 26), BIG),
    (dict(batch=1 << 20, channels=1 << 20), BIG), (dict(batch=1 << 16, steps=1 << 16), BIG)] +
    [({"stride_" + k: (-1, 8)}, BAD) for k in ("x", "delta", "b", "c", "z", "dy")])
def test_scan_problems(over, status):
    p = scan(**over)
    fails(status, adst.adst_selective_scan_plan, p)
    fails(status, adst.adst_selective_scan_forward, *scan_fwd(p))
    fails(status, adst.adst_selective_scan_vjp, *scan_rev(p))


@pytest.mark.parametrize("dtype,states,span", [
    (adst.ADST_BF16, 1, 16), (adst.ADST_F32, 16, 16), (adst.ADST_F16, 17, 8),
    (adst.ADST_F32, 64, 4), (adst.ADST_BF16, 128, 2), (adst.ADST_F64, 16, 8),
    (adst.ADST_F64, 64, 4)])
def test_scan_plan(dtype, states, span):
    p = scan(dtype=dtype, states=states, steps=1001)
    i = adst.adst_selective_scan_plan(p)
    assert i.span == span
    assert i.ck_bytes == 2 * 8 * states * -(-1001 // span) * (8 if dtype == adst.ADST_F64 else 4)
    assert i.vjp_workspace_bytes > i.workspace_bytes > 0  # few rows: several segments
    many = scan(dtype=dtype, states=states, batch=1000, channels=64, groups=1)
    assert adst.adst_selective_scan_plan(many).workspace_bytes == 0
    assert adst.adst_selective_scan_plan(scan(dtype=dtype, states=states, steps=0)).ck_bytes == 0
    assert adst.lib().adst_selective_scan_plan(ctypes.byref(p), None) == BAD
    assert adst.lib().adst_selective_scan_plan(None, None) == BAD


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(delta=None), dict(A=None), dict(B=None), dict(C=None), dict(x=1 + at(0)),
    dict(A=at(2) + 2), dict(D=at(5) + 2), dict(h0=at(8) + 2), dict(lens=at(9) + 2),
    dict(y=at(20) + 2), dict(hT=at(21) + 2), dict(ck=at(22) + 2), dict(y=at(0)), dict(y=at(1) + 4),
    dict(y=at(3) + 6396), dict(hT=at(8)), dict(hT=at(20) + 6396), dict(ck=at(20)), dict(y=at(6)),
    dict(hT=at(9))])
def test_scan_forward_arrays(kw):
    fails(BAD, adst.adst_selective_scan_forward, *scan_fwd(**kw))
    if "y" in kw or "hT" in kw or "ck" in kw:
        return
    fails(BAD, adst.adst_selective_scan_vjp, *scan_rev(**kw))


@pytest.mark.parametrize("kw", [
    dict(dy=None), dict(dx=None), dict(ddelta=None), dict(dB=None), dict(dC=None), dict(dA=None),
    dict(dz=None), dict(z=None), dict(dy=at(24) + 2), dict(dhT=at(25) + 2), dict(dx=at(24)),
    dict(dB=at(14) + 4), dict(dA=at(2)), dict(dD=at(17)), dict(dh0=at(25)), dict(dx=at(22)),
    dict(ws=at(10)), dict(ws=at(23) + 4), dict(dA=at(15) + 2)])
def test_scan_vjp_arrays(kw):
    fails(BAD, adst.adst_selective_scan_vjp, *scan_rev(**kw))


def test_scan_workspaces():
    p = scan(steps=1000, stride_x=(8000, 8), stride_dy=(8000, 8))
    i = adst.adst_selective_scan_plan(p)
    fails(SMALL, adst.adst_selective_scan_forward, *scan_fwd(p, n=i.workspace_bytes - 1))
    fails(SMALL, adst.adst_selective_scan_forward, *scan_fwd(p, ws=None))
    fails(SMALL, adst.adst_selective_scan_vjp, *scan_rev(p, n=i.vjp_workspace_bytes - 1))
    fails(SMALL, adst.adst_selective_scan_vjp,
          *scan_rev(p, ck=None, n=i.vjp_workspace_bytes + i.ck_bytes - 1))


def test_scan_without_channels_needs_its_coefficients_gradients():
    p = scan(channels=0)
    fails(BAD, adst.adst_selective_scan_vjp, *scan_rev(p, dB=None))
    fails(BAD, adst.adst_selective_scan_vjp, *scan_rev(p, dC=None))


@pytest.mark.parametrize("kw,status", [
    (dict(prob=scan()), BAD), (dict(x=None), BAD), (dict(A=None), BAD), (dict(state=None), BAD),
    (dict(h0=at(8)), BAD), (dict(lens=at(9)), BAD), (dict(n=-1), BAD), (dict(slots=None, n=1), BAD),
    (dict(y=at(21)), BAD), (dict(state=at(0)), BAD), (dict(state=at(2)), BAD),
    (dict(state=at(21) + 2), BAD), (dict(slots=at(20) + 2), BAD),
    (dict(prob=scan(steps=1, batch=1 << 10, channels=1 << 16)), BIG)])
def test_scan_step_arguments(kw, status):
    fails(status, adst.adst_selective_scan_step, *scan_one(**kw))


# ----------------------------------------------------------- cross entropy
def xent(**over):
    f = dict(dtype=adst.ADST_F32, reserved=0, rows=10, width=16, vocab=50, stride_x=16, stride_w=16)
    f.update(over)
    return adst.adst_xent_problem(**f)


def xent_fwd(prob=None, x=at(0), w=at(1), labels=at(2), loss=at(3), lse=at(4), ws=at(5), n=MUCH):
    return prob or xent(), x, w, labels, loss, lse, ws, n, 0


def xent_rev(prob=None, x=at(0), w=at(1), labels=at(2), lse=at(3), dloss=at(4), dx=at(5),
             dw=at(6), ws=at(7), n=MUCH):
    return prob or xent(), x, w, labels, lse, dloss, dx, dw, ws, n, 0


@pytest.mark.parametrize("over,status", [
    (dict(dtype=4), BAD), (dict(dtype=-2), BAD), (dict(rows=-1), BAD), (dict(width=0), BAD),
    (dict(vocab=0), BAD), (dict(stride_x=-16), BAD), (dict(stride_w=-1), BAD),
    (dict(rows=1 << 31), BIG), (dict(width=1 << 31), BIG), (dict(vocab=1 << 31), BIG),
    (dict(vocab=1 << 25), BIG), (dict(rows=1 << 25), BIG), (dict(rows=1 << 18, vocab=1 << 17), BIG)])
def test_xent_problems(over, status):
    p = xent(**over)
    fails(status, adst.adst_linear_cross_entropy_plan, p)
    fails(status, adst.adst_linear_cross_entropy_forward, *xent_fwd(p))
    fails(status, adst.adst_linear_cross_entropy_vjp, *xent_rev(p))


def test_xent_plan():
    for dtype, size in ((adst.ADST_F64, 8), (adst.ADST_F32, 4), (adst.ADST_BF16, 2)):
        M, V = 8192, 100000
        i = adst.adst_linear_cross_entropy_plan(xent(dtype=dtype, rows=M, vocab=V, width=512))
        # a piece's g twice and sums, not the logits
        assert i.vjp_workspace_bytes < M * V * size / 2 and i.workspace_bytes < M * V * size / 10
    i = adst.adst_linear_cross_entropy_plan(xent(rows=0))
    assert i.workspace_bytes == i.vjp_workspace_bytes == 0
    assert adst.lib().adst_linear_cross_entropy_plan(ctypes.byref(xent()), None) == BAD
    assert adst.lib().adst_linear_cross_entropy_plan(None, None) == BAD


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(w=None), dict(labels=None), dict(x=at(0) + 2), dict(w=at(1) + 2),
    dict(labels=at(2) + 2)])
def test_xent_inputs(kw):
    fails(BAD, adst.adst_linear_cross_entropy_forward, *xent_fwd(**kw))
    fails(BAD, adst.adst_linear_cross_entropy_vjp, *xent_rev(**kw))


def test_xent_arrays():
    i = adst.adst_linear_cross_entropy_plan(xent())
    for kw in (dict(loss=at(4) + 36), dict(loss=at(0)), dict(lse=at(1) + 3196), dict(lse=at(2)),
               dict(loss=at(3) + 2), dict(ws=at(3)), dict(ws=at(5) + 8)):
        fails(BAD, adst.adst_linear_cross_entropy_forward, *xent_fwd(**kw))
    for kw in (dict(lse=None), dict(lse=at(3) + 2), dict(dloss=at(4) + 2), dict(dx=at(0)),
               dict(dw=at(1)), dict(dx=at(6) + 3196), dict(dw=at(2)), dict(dx=at(3)),
               dict(dw=at(4)), dict(ws=at(0)), dict(ws=at(6)), dict(dx=at(5) + 2)):
        fails(BAD, adst.adst_linear_cross_entropy_vjp, *xent_rev(**kw))
    fails(SMALL, adst.adst_linear_cross_entropy_forward, *xent_fwd(n=i.workspace_bytes - 1))
    fails(SMALL, adst.adst_linear_cross_entropy_vjp, *xent_rev(n=i.vjp_workspace_bytes - 1))
    fails(SMALL, adst.adst_linear_cross_entropy_vjp, *xent_rev(ws=None))


# ------------------------------------------- arrays that a call without steps reads
@pytest.mark.parametrize("over", [dict(steps=0), dict(batch=0), dict(steps=0, batch=0)])
@pytest.mark.parametrize("out", ["dx", "dw", "db", "dx0"])
def test_conv_vjp_needs_its_weights_without_steps_too(over, out):
    """The kernel that writes an output loads the taps first, whatever the extents."""
    none = {k: None for k in ("dx", "dw", "db", "dx0") if k != out}
    fails(BAD, adst.adst_causal_conv_vjp, *conv_rev(conv(**over), x=None, dy=None, w=None, **none))


@pytest.mark.parametrize("out", ["y", "hT", "ck"])
def test_scan_forward_needs_its_rates_without_steps_too(out):
    """The kernel that writes an output loads A first, whatever the steps."""
    none = {k: None for k in ("y", "hT", "ck") if k != out}
    kw = dict(x=None, delta=None, A=None, B=None, C=None, **none)
    fails(BAD, adst.adst_selective_scan_forward, *scan_fwd(scan(steps=0), **kw))


@pytest.mark.parametrize("over", [
    dict(groups=1 << 62), dict(groups=1 << 40, batch=1 << 20, steps=1 << 20),
    dict(groups=1, states=1, batch=1 << 30, steps=1 << 30),
    dict(groups=(1 << 63) - 1, states=128, batch=(1 << 31) - (1 << 17), steps=1 << 30)])
def test_scan_extents_without_channels(over):
    """Their products are refused, not wrapped: no number of channels bounds the groups then."""
    strides = {"stride_" + k: (0, 0) for k in ("x", "delta", "b", "c", "z", "dy")}
    p = scan(channels=0, **strides, **over)
    fails(BIG, adst.adst_selective_scan_plan, p)
    fails(BIG, adst.adst_selective_scan_vjp, *scan_rev(p))


@pytest.mark.parametrize("reserved", [1, -1, 1 << 30])
def test_xent_reserved_is_zero(reserved):
    p = xent(reserved=reserved)
    fails(BAD, adst.adst_linear_cross_entropy_plan, p)
    fails(BAD, adst.adst_linear_cross_entropy_forward, *xent_fwd(p))
    fails(BAD, adst.adst_linear_cross_entropy_vjp, *xent_rev(p))


@pytest.mark.parametrize("dtype,size", [(adst.ADST_F32, 4), (adst.ADST_BF16, 2), (adst.ADST_F16, 2)])
def test_xent_plan_of_several_pieces(dtype, size):
    """At the sizes of the GPU's test of several pieces: g of the whole vocabulary in two orders, or
    in one, would not fit the workspace."""
    M, K, V = (128 << 20) // size // 1024, 32, 2100
    i = adst.adst_linear_cross_entropy_plan(xent(dtype=dtype, rows=M, vocab=V, width=K, stride_x=K,
                                                 stride_w=K))
    assert i.vjp_workspace_bytes < M * V * size
