"""What the sequence operators refuse, on a host without a GPU: every bad
argument is an error before anything is enqueued (the pointers are never
dereferenced)."""
import ctypes

import pytest
import torch

import paper_2509_02197_amd as adst

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="host-only argument checks")
A, U, H, W = 0x100000000, 0x200000000, 0x300000000, 0x400000000
OUT1, OUT2, OUT3 = 0x500000000, 0x600000000, 0x700000000
WS = 0x800000000


def rec(**over):
    f = dict(dtype=adst.ADST_F32, gate=0, batch=2, steps=100, channels=8, stride_a_batch=800,
             stride_a_step=8, stride_u_batch=800, stride_u_step=8, stride_dh_batch=800,
             stride_dh_step=8)
    f.update(over)
    return adst.adst_recurrence_problem(**f)


def fails(status, call, *args, **kw):
    with pytest.raises(adst.AdstError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)
    assert adst.adst_last_error()


BAD_REC = [(dict(dtype=4), adst.ADST_ERR_ARG), (dict(dtype=-1), adst.ADST_ERR_ARG),
           (dict(gate=2), adst.ADST_ERR_ARG), (dict(batch=-1), adst.ADST_ERR_ARG),
           (dict(steps=-1), adst.ADST_ERR_ARG), (dict(channels=-3), adst.ADST_ERR_ARG),
           (dict(stride_a_step=-8), adst.ADST_ERR_ARG),
           (dict(stride_dh_batch=-1), adst.ADST_ERR_ARG),
           (dict(steps=1 << 31), adst.ADST_ERR_UNSUPPORTED),
           (dict(channels=1 << 40), adst.ADST_ERR_UNSUPPORTED),
           (dict(batch=1 << 30, channels=1 << 30), adst.ADST_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("over,status", BAD_REC)
def test_recurrence_problems(over, status):
    p = rec(**over)
    fails(status, adst.adst_recurrence_plan, p)
    fails(status, adst.adst_recurrence_forward, p, A, U, None, None, H, None, None, WS, 1 << 40, 0)
    fails(status, adst.adst_recurrence_vjp, p, A, U, None, None, None, H, None, OUT1, OUT2, None,
          WS, 1 << 40, 0)


def test_recurrence_plan():
    for dtype, size in ((adst.ADST_F64, 8), (adst.ADST_F32, 4), (adst.ADST_BF16, 4)):
        p = rec(dtype=dtype, steps=100000)
        i = adst.adst_recurrence_plan(p)
        spans = -(-100000 // i.span)
        assert i.ck_bytes == 2 * 8 * spans * size
        assert i.vjp_workspace_bytes >= i.workspace_bytes + i.ck_bytes
    assert adst.adst_recurrence_plan(rec(steps=0)).ck_bytes <= 2 * 8 * 8
    assert adst.lib().adst_recurrence_plan(ctypes.byref(rec()), None) == adst.ADST_ERR_ARG
    assert adst.lib().adst_recurrence_plan(None, None) == adst.ADST_ERR_ARG


def test_recurrence_arrays():
    p, bad = rec(), adst.ADST_ERR_ARG
    ck = adst.adst_recurrence_plan(p).ck_bytes
    big = 1 << 40

    def fwd(a=A, u=U, h0=None, lens=None, h=H, hT=OUT1, ck=None, ws=WS, n=big, prob=p):
        return prob, a, u, h0, lens, h, hT, ck, ws, n, 0

    for kw in (dict(a=None), dict(u=None), dict(a=A + 1), dict(h=H + 2), dict(hT=OUT1 + 1),
               dict(h=A), dict(h=U + 6396), dict(hT=H + 6396), dict(h0=OUT1 + 4),
               dict(ck=H), dict(lens=H), dict(lens=W + 2), dict(ck=OUT1 - ck + 4)):
        fails(bad, adst.adst_recurrence_forward, *fwd(**kw))

    def rev(a=A, u=U, h0=None, lens=None, ck=None, dh=H, dhT=None, da=OUT1, du=OUT2, dh0=OUT3,
            ws=WS, n=big):
        return p, a, u, h0, lens, ck, dh, dhT, da, du, dh0, ws, n, 0

    for kw in (dict(dh=None), dict(da=None), dict(du=None), dict(da=H), dict(du=OUT1 + 4),
               dict(dh0=A), dict(da=A), dict(dhT=OUT3), dict(ck=OUT2), dict(ws=OUT1), dict(ws=A)):
        fails(bad, adst.adst_recurrence_vjp, *rev(**kw))
    fails(adst.ADST_ERR_WORKSPACE, adst.adst_recurrence_vjp, *rev(n=ck - 1))
    fails(adst.ADST_ERR_WORKSPACE, adst.adst_recurrence_vjp, *rev(ws=None))


def test_recurrence_step_arguments():
    p = rec(steps=1)
    bad = adst.ADST_ERR_ARG

    def step(prob=p, a=A, u=U, slots=W, state=OUT1, n=4, h=H):
        return prob, a, u, slots, state, n, h, 0

    for kw in (dict(prob=rec(steps=2)), dict(a=None), dict(u=None), dict(state=None), dict(n=-1),
               dict(slots=None, n=1), dict(h=OUT1), dict(state=A), dict(state=OUT1 + 2),
               dict(slots=W + 1), dict(slots=OUT1 + 64)):
        fails(bad, adst.adst_recurrence_step, *step(**kw))


def norm(**over):
    f = dict(dtype=adst.ADST_F32, weight_dtype=adst.ADST_F32, rows=10, n=16, stride_x=16,
             stride_dy=16, eps=1e-5)
    f.update(over)
    return adst.adst_norm_problem(**f)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=9), adst.ADST_ERR_ARG), (dict(weight_dtype=adst.ADST_BF16), adst.ADST_ERR_ARG),
    (dict(dtype=adst.ADST_F64), adst.ADST_ERR_ARG),
    (dict(dtype=adst.ADST_BF16, weight_dtype=adst.ADST_F16), adst.ADST_ERR_ARG),
    (dict(rows=-1), adst.ADST_ERR_ARG), (dict(n=0), adst.ADST_ERR_ARG),
    (dict(stride_x=-1), adst.ADST_ERR_ARG), (dict(eps=-1.0), adst.ADST_ERR_ARG),
    (dict(eps=float("nan")), adst.ADST_ERR_ARG), (dict(eps=float("inf")), adst.ADST_ERR_ARG),
    (dict(n=1 << 31), adst.ADST_ERR_UNSUPPORTED), (dict(rows=1 << 33), adst.ADST_ERR_UNSUPPORTED)])
def test_norm_problems(over, status):
    p = norm(**over)
    fails(status, adst.adst_layer_norm_forward, p, A, None, None, H, None, None, 0)
    fails(status, adst.adst_layer_norm_vjp, p, A, U, None, W, W + 4096, H, OUT1, OUT2, WS, 1 << 40,
          0)


def test_norm_arrays():
    p, bad = norm(), adst.ADST_ERR_ARG
    need = adst.adst_layer_norm_workspace_bytes(p)
    assert need > 0

    def fwd(x=A, w=U, b=W, y=H, mean=OUT1, rstd=OUT2):
        return p, x, w, b, y, mean, rstd, 0

    for kw in (dict(x=None), dict(y=None), dict(x=A + 2), dict(w=U + 1), dict(y=A + 4),
               dict(y=U), dict(mean=OUT2), dict(rstd=H + 36), dict(mean=OUT1 + 2)):
        fails(bad, adst.adst_layer_norm_forward, *fwd(**kw))

    def rev(x=A, dy=U, w=None, mean=W, rstd=W + 4096, dx=H, dw=OUT1, db=OUT2, ws=WS, n=1 << 40):
        return p, x, dy, w, mean, rstd, dx, dw, db, ws, n, 0

    for kw in (dict(x=None), dict(dy=None), dict(mean=None), dict(rstd=None), dict(dx=A),
               dict(dx=U), dict(dw=OUT2), dict(db=H + 4), dict(dw=W), dict(ws=H), dict(ws=WS + 4)):
        fails(bad, adst.adst_layer_norm_vjp, *rev(**kw))
    fails(adst.ADST_ERR_WORKSPACE, adst.adst_layer_norm_vjp, *rev(n=need - 1))
    fails(adst.ADST_ERR_WORKSPACE, adst.adst_layer_norm_vjp, *rev(ws=None))


def adamw(tensor={}, **over):
    f = dict(dtype=adst.ADST_F32, grad_dtype=adst.ADST_BF16, copy_dtype=adst.ADST_BF16, bits=32,
             t=1, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=None)
    f.update(over)
    t = dict(p=A, grad=U, m=H, v=W, m_scale=OUT1, v_scale=OUT2, copy=None, n=1000, lr=1e-3,
             weight_decay=0.0)
    t.update(tensor)
    return adst.adst_adamw_problem(**f), (adst.adst_adamw_tensor * 1)(adst.adst_adamw_tensor(**t))


NAN = float("nan")


@pytest.mark.parametrize("args", [
    dict(dtype=adst.ADST_BF16), dict(dtype=adst.ADST_F64), dict(grad_dtype=adst.ADST_F64),
    dict(grad_dtype=7), dict(bits=16), dict(bits=8, dtype=adst.ADST_F64,
                                            grad_dtype=adst.ADST_F64),
    dict(copy_dtype=adst.ADST_F64), dict(t=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=NAN),
    dict(eps=-1e-8), dict(eps=NAN), dict(grad_scale=A + 400), dict(grad_scale=OUT3 + 2),
    dict(tensor=dict(p=None)), dict(tensor=dict(grad=None)), dict(tensor=dict(m=None)),
    dict(tensor=dict(v=None)), dict(tensor=dict(m_scale=None), bits=8),
    dict(tensor=dict(n=-1)), dict(tensor=dict(lr=NAN)), dict(tensor=dict(weight_decay=NAN)),
    dict(tensor=dict(p=A + 2)), dict(tensor=dict(grad=U + 1)), dict(tensor=dict(copy=OUT3 + 1)),
    dict(tensor=dict(m=A)), dict(tensor=dict(grad=W)), dict(tensor=dict(copy=H)),
    dict(tensor=dict(v_scale=OUT1 + 8), bits=8)])
def test_adamw_arguments(args):
    prob, rows = adamw(**args)
    fails(adst.ADST_ERR_ARG, adst.adst_adamw, prob, rows, 1, 0)


def test_adamw_sizes():
    prob, rows = adamw(tensor=dict(n=1 << 40, p=A))
    fails(adst.ADST_ERR_UNSUPPORTED, adst.adst_adamw, prob, rows, 1, 0)
    fails(adst.ADST_ERR_ARG, adst.adst_adamw, adamw()[0], None, 1, 0)
    fails(adst.ADST_ERR_ARG, adst.adst_adamw, adamw()[0], adamw()[1], -1, 0)
    adst.adst_adamw(adamw()[0], None, 0, 0)  # nothing to do
    prob, rows = adamw(tensor=dict(n=0, p=None, grad=None))
    prob.t = 5


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(adst.adst_recurrence_problem) == 80
    assert ctypes.sizeof(adst.adst_recurrence_info) == 32
    assert ctypes.sizeof(adst.adst_norm_problem) == 48
    assert ctypes.sizeof(adst.adst_adamw_tensor) == 80
    assert ctypes.sizeof(adst.adst_adamw_problem) == 56


@pytest.mark.parametrize("call", [
    lambda t: adst.recurrence(t(2, 3, 4), t(2, 3, 4)),
    lambda t: adst.recurrence_step(t(2, 4), t(2, 4), t(2, 4)),
    lambda t: adst.layer_norm(t(2, 3)), lambda t: adst.AdamW([t(3)])])
def test_tensors_on_the_host(call):
    with pytest.raises(ValueError, match="GPU"):
        call(torch.zeros)


def test_tensors_of_other_types():
    with pytest.raises(TypeError):
        adst.layer_norm(torch.zeros(3, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        adst.layer_norm([1.0, 2.0])
    with pytest.raises(ValueError):
        adst.AdamW([])


def test_the_native_calls_answer_none_to_anything_unusual():
    """sequence.py then handles it, or raises its error; no exception leaves the binding."""
    b = adst.sequence._binding()
    x, w = torch.zeros(4, 8), torch.zeros(8)
    h = torch.zeros(2, 3, 8)
    for call in (lambda: b.layer_norm(x, w, w, 1e-5), lambda: b.layer_norm(x, w, w, "eps"),
                 lambda: b.layer_norm(), lambda: b.layer_norm(1, 2, 3, 4),
                 lambda: b.layer_norm_vjp(x, x, None, None, None, 1, 1, 1),
                 lambda: b.recurrence(h, h, None, None, 0, True, True),
                 lambda: b.recurrence(h, h, None, None, 1.5, True, True),
                 lambda: b.recurrence_vjp(h, h, h, None, None, None, None, 0),
                 lambda: b.recurrence_step(x, x, x, None, 0),
                 lambda: b.adamw_step(0, 0, (), [], None, None, 1),
                 lambda: b.adamw_step(None, None, (x,), [x], None, None, 1)):
        assert call() is None
