"""The token operators of adst.h from Python: the causal convolution and the
selective scan with their VJPs and one-step forms, and the softmax cross
entropy of a vocabulary with its gradient.

The ``adst_*`` functions keep the C names and only marshal arguments. The
others take torch tensors, check them, allocate outputs and workspaces with
torch and make the call, as in ``sequence.py``: errors in the arguments are
ValueError or TypeError before anything is launched, and a call runs on torch's
current stream, or on `stream`.
"""
import ctypes

from . import (ADST_ACT_NONE, ADST_BF16, ADST_CONV_MAX_TAPS, ADST_F16, ADST_F32,
               _check, _ptr, _stream, adst_conv_problem, adst_scan_gradients, adst_scan_info,
               adst_scan_inputs, adst_scan_problem, adst_xent_info, adst_xent_problem, lib)
from .sequence import (_acc, _at, _binding, _bytes, _call, _channels_contiguous, _check_in_place,
                       _code, _codes, _expect, _require)


# ------------------------------------------------------------ the C calls
def adst_causal_conv_forward(prob, x, w, bias, x0, lens, y, xT, stream=None):
    _check(lib().adst_causal_conv_forward(ctypes.byref(prob), _ptr(x), _ptr(w), _ptr(bias),
                                          _ptr(x0), _ptr(lens), _ptr(y), _ptr(xT),
                                          _stream(stream)))


def adst_causal_conv_workspace_bytes(prob):
    return int(lib().adst_causal_conv_workspace_bytes(ctypes.byref(prob)))


def adst_causal_conv_vjp(prob, x, dy, w, bias, x0, lens, dxT, dx, dw, dbias, dx0, ws, ws_bytes,
                         stream=None):
    _check(lib().adst_causal_conv_vjp(ctypes.byref(prob), _ptr(x), _ptr(dy), _ptr(w), _ptr(bias),
                                      _ptr(x0), _ptr(lens), _ptr(dxT), _ptr(dx), _ptr(dw),
                                      _ptr(dbias), _ptr(dx0), _ptr(ws), ws_bytes,
                                      _stream(stream)))


def adst_causal_conv_step(prob, x, w, bias, slots, window, nstates, y, stream=None):
    _check(lib().adst_causal_conv_step(ctypes.byref(prob), _ptr(x), _ptr(w), _ptr(bias),
                                       _ptr(slots), _ptr(window), nstates, _ptr(y),
                                       _stream(stream)))


def adst_selective_scan_plan(prob):
    info = adst_scan_info()
    _check(lib().adst_selective_scan_plan(ctypes.byref(prob), ctypes.byref(info)))
    return info


def adst_selective_scan_forward(prob, inputs, y, hT, ck, ws, ws_bytes, stream=None):
    """inputs: an adst_scan_inputs of device addresses."""
    _check(lib().adst_selective_scan_forward(ctypes.byref(prob), ctypes.byref(inputs), _ptr(y),
                                             _ptr(hT), _ptr(ck), _ptr(ws), ws_bytes,
                                             _stream(stream)))


def adst_selective_scan_vjp(prob, inputs, ck, dy, dhT, gradients, ws, ws_bytes, stream=None):
    """inputs, gradients: an adst_scan_inputs and an adst_scan_gradients of device addresses."""
    _check(lib().adst_selective_scan_vjp(ctypes.byref(prob), ctypes.byref(inputs), _ptr(ck),
                                         _ptr(dy), _ptr(dhT), ctypes.byref(gradients), _ptr(ws),
                                         ws_bytes, _stream(stream)))


def adst_selective_scan_step(prob, inputs, slots, state, nstates, y, stream=None):
    _check(lib().adst_selective_scan_step(ctypes.byref(prob), ctypes.byref(inputs), _ptr(slots),
                                          _ptr(state), nstates, _ptr(y), _stream(stream)))


def adst_linear_cross_entropy_plan(prob):
    info = adst_xent_info()
    _check(lib().adst_linear_cross_entropy_plan(ctypes.byref(prob), ctypes.byref(info)))
    return info


def adst_linear_cross_entropy_forward(prob, x, w, labels, loss, lse, ws, ws_bytes, stream=None):
    _check(lib().adst_linear_cross_entropy_forward(ctypes.byref(prob), _ptr(x), _ptr(w),
                                                   _ptr(labels), _ptr(loss), _ptr(lse), _ptr(ws),
                                                   ws_bytes, _stream(stream)))


def adst_linear_cross_entropy_vjp(prob, x, w, labels, lse, dloss, dx, dw, ws, ws_bytes,
                                  stream=None):
    _check(lib().adst_linear_cross_entropy_vjp(ctypes.byref(prob), _ptr(x), _ptr(w), _ptr(labels),
                                               _ptr(lse), _ptr(dloss), _ptr(dx), _ptr(dw),
                                               _ptr(ws), ws_bytes, _stream(stream)))


# ------------------------------------------------------------------ checks
def _sequence(name, t, like=None):
    """Strides of t [batch, steps, channels] with contiguous channels, of like's shape, type and
    device."""
    if like is not None:
        _require(name, t)
        _expect(name, t, like.shape, like.dtype, like.device, contiguous=False)
    elif t.dim() != 3:
        raise ValueError(f"{name} must be [batch, steps, channels], not {tuple(t.shape)}")
    _channels_contiguous(name, t)
    return t.stride(0), t.stride(1)


def _weights(code, x, w, b, shape):
    """The code of the weights' type."""
    import torch
    wcode = _codes().get(w.dtype, -1)
    if wcode != code and not (code in (ADST_BF16, ADST_F16) and wcode == ADST_F32):
        raise ValueError(f"weights must be {x.dtype} (or float32 beside 16-bit types), "
                         f"not {w.dtype}")
    _expect("w", w, torch.Size(shape), w.dtype, x.device)
    _expect("b", b, torch.Size(shape[1:]), w.dtype, x.device)
    return wcode


def _lens(lens, x):
    import torch
    _expect("lens", lens, (x.shape[0],), torch.int32, x.device)


# ------------------------------------------------------------- convolution
def _taps(w, D):
    _require("w", w)
    if w.dim() != 2 or w.shape[1] != D or not 1 <= w.shape[0] <= ADST_CONV_MAX_TAPS:
        raise ValueError(f"w must be [taps, {D}] with 1 to {ADST_CONV_MAX_TAPS} taps, "
                         f"not {tuple(w.shape)}")
    return w.shape[0]


def _act(act):
    if not -1 << 31 <= act < 1 << 31:  # ctypes would cut it
        raise ValueError(f"unknown act {act}")
    return act


def _conv_problem(x, w, b, x0, lens, act, dy=None, dxT=None):
    code = _code("x", x)
    sx = _sequence("x", x)
    sd = (0, 0) if dy is None else _sequence("dy", dy, x)
    B, T, D = x.shape
    K = _taps(w, D)
    wcode = _weights(code, x, w, b, (K, D))
    for name, t in (("x0", x0), ("dxT", dxT)):
        _expect(name, t, (B, K - 1, D), x.dtype, x.device)
    _lens(lens, x)
    return adst_conv_problem(code, wcode, _act(act), K, B, T, D, *sx, *sd)


def causal_conv(x, w, b=None, x0=None, lens=None, act=ADST_ACT_NONE, want_y=True, stream=None):
    """y_t = act(b + sum over k of w[k] * x_{t - (taps - 1) + k}) over axis 1 of x
    [batch, steps, channels], for each channel; w [taps, channels] with 1 to 8 taps and b
    [channels], of x's dtype, or float32 beside 16-bit types; act ADST_ACT_NONE or
    ADST_ACT_SILU.

    x0 [batch, taps - 1, channels]: the inputs before the first, oldest first (zeros if None);
    lens [batch] int32: the steps of each row. x may have any strides with contiguous channels.
    Returns a dict: y (None unless want_y; 0 beyond lens) and xT, the window that follows each
    row: x0 of the next piece of it, or its state for causal_conv_step."""
    if stream is None:
        done = _binding().causal_conv(x, w, b, x0, lens, act, want_y)
        if done is not None:
            return done
    import torch
    prob = _conv_problem(x, w, b, x0, lens, act)
    B, T, D = x.shape

    def body(handle):
        y = torch.empty_like(x, memory_format=torch.contiguous_format) if want_y else None
        xT = torch.empty((B, prob.taps - 1, D), dtype=x.dtype, device=x.device)
        _check(lib().adst_causal_conv_forward(prob, x.data_ptr(), w.data_ptr(), _at(b), _at(x0),
                                              _at(lens), _at(y), xT.data_ptr(), handle))
        return {"y": y, "xT": xT}

    return _call(x.device, stream, (x, w, b, x0, lens), body)


def causal_conv_vjp(x, dy, w, b=None, x0=None, lens=None, dxT=None, act=ADST_ACT_NONE,
                    want_dx=True, want_dw=True, want_db=True, stream=None):
    """The VJP of causal_conv: dy = dL/dy, dxT = dL/dxT (optional). Returns a dict: dx, dw and db
    (in w's dtype), each None unless wanted, and dx0."""
    if stream is None:
        done = _binding().causal_conv_vjp(x, dy, w, b, x0, lens, dxT, act, want_dx, want_dw,
                                          want_db)
        if done is not None:
            return done
    import torch
    prob = _conv_problem(x, w, b, x0, lens, act, _given("dy", dy), dxT)
    B, T, D = x.shape

    def body(handle):
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want_dx else None
        dw = torch.empty_like(w) if want_dw else None
        db = torch.empty(D, dtype=w.dtype, device=x.device) if want_db else None
        dx0 = torch.empty((B, prob.taps - 1, D), dtype=x.dtype, device=x.device)
        need = adst_causal_conv_workspace_bytes(prob) if want_dw or want_db else 0
        ws = _bytes(need, x.device)
        _check(lib().adst_causal_conv_vjp(prob, x.data_ptr(), dy.data_ptr(), w.data_ptr(), _at(b),
                                          _at(x0), _at(lens), _at(dxT), _at(dx), _at(dw), _at(db),
                                          dx0.data_ptr(), _at(ws), need, handle))
        return {"dx": dx, "dw": dw, "db": db, "dx0": dx0}

    return _call(x.device, stream, (x, dy, w, b, x0, lens, dxT), body)


def _given(name, t):
    _require(name, t)
    return t


def causal_conv_step(x, w, window, b=None, slots=None, act=ADST_ACT_NONE, stream=None):
    """One step of every row of x [batch, channels] on the pool of windows
    [nstates, taps - 1, channels] of x's dtype, updated in place. slots [batch] int32: each row's
    window, no two the same; None: row b's is window[b]. Rows whose slot is outside the pool are
    idle: their y is 0. Returns y [batch, channels]."""
    if stream is None:
        y = _binding().causal_conv_step(x, w, window, b, slots, act)
        if y is not None:
            return y
    import torch
    code = _code("x", x)
    if x.dim() != 2:
        raise ValueError(f"x must be [batch, channels], not {tuple(x.shape)}")
    B, D = x.shape
    _channels_contiguous("x", x)
    K = _taps(w, D)
    wcode = _weights(code, x, w, b, (K, D))
    _require("window", window)
    if window.dim() != 3 or window.shape[1:] != (K - 1, D):
        raise ValueError(f"window must be [nstates, {K - 1}, {D}], not {tuple(window.shape)}")
    _expect("window", window, window.shape, x.dtype, x.device)
    _expect("slots", slots, (B,), torch.int32, x.device)
    prob = adst_conv_problem(code, wcode, _act(act), K, B, 1, D, x.stride(0), 0, 0, 0)

    def body(handle):
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        _check_in_place(lib().adst_causal_conv_step(prob, x.data_ptr(), w.data_ptr(), _at(b),
                                                    _at(slots), window.data_ptr(),
                                                    window.shape[0], y.data_ptr(), handle),
                        (window,))
        return y

    return _call(x.device, stream, (x, w, b, window, slots), body)


# ---------------------------------------------------------- selective scan
def _scan_problem(x, delta, A, B, C, D, z, delta_bias, softplus, dy=None):
    """The problem and its inputs' addresses, for x [batch, steps, channels]."""
    code = _code("x", x)
    acc = _acc(code)
    strides = [_sequence("x", x), _sequence("delta", delta, x)]
    Bt, T, Dn = x.shape
    _require("A", A)
    if A.dim() != 2 or A.shape[0] != Dn or A.shape[1] < 1:
        raise ValueError(f"A must be [{Dn}, states], not {tuple(A.shape)}")
    _expect("A", A, A.shape, acc, x.device)
    N = A.shape[1]
    groups = None
    for name, t in (("B", B), ("C", C)):
        _require(name, t)
        if t.dim() not in (3, 4):
            raise ValueError(f"{name} must be [batch, steps, groups, {N}] or [batch, steps, {N}]")
        if groups is None:
            groups = t.shape[2] if t.dim() == 4 else 1
            if groups < 1 or Dn % groups:
                raise ValueError(f"{groups} groups do not divide {Dn} channels")
        shape = (Bt, T, groups, N) if t.dim() == 4 else (Bt, T, N)
        _expect(name, t, shape, x.dtype, x.device, contiguous=False)
        _channels_contiguous(name, t)
        if t.dim() == 4 and groups > 1 and t.stride(2) != N:
            raise ValueError(f"{name}'s groups must be contiguous (stride {N}, not {t.stride(2)})")
        if t.dim() == 3 and groups != 1:
            raise ValueError(f"{name} must be [batch, steps, {groups}, {N}]")
        strides.append((t.stride(0), t.stride(1)))
    strides.append((0, 0) if z is None else _sequence("z", z, x))
    strides.append((0, 0) if dy is None else _sequence("dy", dy, x))
    for name, t in (("D", D), ("delta_bias", delta_bias)):
        _expect(name, t, (Dn,), acc, x.device)
    prob = adst_scan_problem(code, 1 if softplus else 0, Bt, T, Dn, N, groups,
                             *(s for pair in strides for s in pair))
    return prob, adst_scan_inputs(x.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(),
                                  C.data_ptr(), _at(D), _at(z), _at(delta_bias))


def _scan_rows(prob, inputs, x, h0, lens, dhT=None):
    states = (prob.batch, prob.channels, prob.states)
    for name, t in (("h0", h0), ("dhT", dhT)):
        _expect(name, t, states, _acc(prob.dtype), x.device)
    _lens(lens, x)
    inputs.h0, inputs.lens = _at(h0), _at(lens)


def selective_scan(x, delta, A, B, C, D=None, z=None, delta_bias=None, h0=None, lens=None,
                   softplus=False, want_y=True, want_ck=False, stream=None):
    """h_t[n] = exp(s_t A[n]) h_{t-1}[n] + s_t x_t B_t[n] and
    y_t = (sum over n of C_t[n] h_t[n] + D x_t) z_t sigmoid(z_t) over axis 1 of x, delta and z
    [batch, steps, channels], with s = delta + delta_bias, or softplus of that. A
    [channels, states] with 1 to 128 states (64 in float64), D and delta_bias [channels], in
    float32 (float64 for float64 inputs); B and C [batch, steps, groups, states], or without the
    groups' axis for one, of x's dtype: channel d reads group d // (channels // groups). The
    products of consecutive exp(s A) have to stay in range, which s A <= 0 ensures.

    h0 [batch, channels, states] (zeros if None), like A's type; lens [batch] int32: the steps of
    each row. x, delta, z, B and C may have any strides with contiguous channels (groups and
    states). Returns a dict: y (None unless want_y; 0 beyond lens), hT the last states, and ck
    (None unless want_ck) the checkpoints with which selective_scan_vjp recomputes the states."""
    if stream is None:
        done = _binding().selective_scan(x, delta, A, B, C, D, z, delta_bias, h0, lens, softplus,
                                         want_y, want_ck)
        if done is not None:
            return done
    import torch
    prob, inputs = _scan_problem(x, delta, A, B, C, D, z, delta_bias, softplus)
    _scan_rows(prob, inputs, x, h0, lens)
    info = adst_selective_scan_plan(prob)

    def body(handle):
        y = torch.empty_like(x, memory_format=torch.contiguous_format) if want_y else None
        hT = torch.empty((prob.batch, prob.channels, prob.states), dtype=A.dtype, device=x.device)
        ck = _bytes(info.ck_bytes, x.device) if want_ck else None
        ws = _bytes(info.workspace_bytes, x.device)
        _check(lib().adst_selective_scan_forward(prob, inputs, _at(y), hT.data_ptr(), _at(ck),
                                                 _at(ws), info.workspace_bytes, handle))
        return {"y": y, "hT": hT, "ck": ck}

    return _call(x.device, stream, (x, delta, A, B, C, D, z, delta_bias, h0, lens), body)


def selective_scan_vjp(x, delta, A, B, C, dy, D=None, z=None, delta_bias=None, h0=None, lens=None,
                       dhT=None, ck=None, softplus=False, stream=None):
    """The VJP of selective_scan: dy = dL/dy, dhT = dL/dhT (optional). ck: the checkpoints that
    selective_scan gave for the same inputs; None recomputes them. Returns a dict: dx, ddelta, dz,
    dB, dC, dA, dD, ddelta_bias (each like its input, None without it) and dh0."""
    if stream is None:
        done = _binding().selective_scan_vjp(x, delta, A, B, C, dy, D, z, delta_bias, h0, lens, dhT,
                                             ck, softplus)
        if done is not None:
            return done
    import torch
    prob, inputs = _scan_problem(x, delta, A, B, C, D, z, delta_bias, softplus, _given("dy", dy))
    _scan_rows(prob, inputs, x, h0, lens, dhT)
    info = adst_selective_scan_plan(prob)
    _expect("ck", ck, (info.ck_bytes,), torch.uint8, x.device)
    need = info.vjp_workspace_bytes + (0 if ck is not None else info.ck_bytes)

    def body(handle):
        def like(t):
            return None if t is None else torch.empty_like(t,
                                                           memory_format=torch.contiguous_format)

        out = {"dx": like(x), "ddelta": like(x), "dz": like(z), "dB": like(B), "dC": like(C),
               "dA": like(A), "dD": like(D), "ddelta_bias": like(delta_bias),
               "dh0": torch.empty((prob.batch, prob.channels, prob.states), dtype=A.dtype,
                                  device=x.device)}
        ws = _bytes(need, x.device)
        gradients = adst_scan_gradients(**{k: _at(t) for k, t in out.items()})
        _check(lib().adst_selective_scan_vjp(prob, inputs, _at(ck), dy.data_ptr(), _at(dhT),
                                             gradients, _at(ws), need, handle))
        return out

    return _call(x.device, stream, (x, delta, A, B, C, dy, D, z, delta_bias, h0, lens, dhT, ck),
                 body)


def selective_scan_step(x, delta, A, B, C, state, D=None, z=None, delta_bias=None, slots=None,
                        softplus=False, stream=None):
    """One step of every row of x, delta, z [batch, channels] and B, C [batch, groups, states]
    (or [batch, states]) on the pool of states [nstates, channels, states] (float32, float64 for
    float64 inputs), updated in place. slots [batch] int32: each row's state, no two the same;
    None: row b's is state[b]. Rows whose slot is outside the pool are idle: their y is 0. Returns
    y [batch, channels]."""
    if stream is None:
        y = _binding().selective_scan_step(x, delta, A, B, C, state, D, z, delta_bias, slots,
                                           softplus)
        if y is not None:
            return y
    import torch
    _code("x", x)
    if x.dim() != 2:
        raise ValueError(f"x must be [batch, channels], not {tuple(x.shape)}")

    def step(name, t, dims):
        if t is None:
            return None
        _require(name, t)
        if t.dim() not in dims:
            raise ValueError(f"{name} has shape {tuple(t.shape)}")
        return t.unsqueeze(1)

    prob, inputs = _scan_problem(x.unsqueeze(1), step("delta", delta, (2,)), A,
                                 step("B", B, (2, 3)), step("C", C, (2, 3)), D,
                                 step("z", z, (2,)), delta_bias, softplus)
    _require("state", state)
    if state.dim() != 3 or state.shape[1:] != A.shape:
        raise ValueError(f"state must be [nstates, {A.shape[0]}, {A.shape[1]}], "
                         f"not {tuple(state.shape)}")
    _expect("state", state, state.shape, A.dtype, x.device)
    _expect("slots", slots, (x.shape[0],), torch.int32, x.device)

    def body(handle):
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        _check_in_place(lib().adst_selective_scan_step(prob, inputs, _at(slots), state.data_ptr(),
                                                       state.shape[0], y.data_ptr(), handle),
                        (state,))
        return y

    return _call(x.device, stream, (x, delta, A, B, C, D, z, delta_bias, state, slots), body)


# ------------------------------------------------------------ cross entropy
def _xent_problem(x, w, labels):
    import torch
    code = _code("x", x)
    if x.dim() != 2 or x.shape[1] < 1:
        raise ValueError(f"x must be [rows, width], not {tuple(x.shape)}")
    _require("w", w)
    if w.dim() != 2 or w.shape[0] < 1 or w.shape[1] != x.shape[1]:
        raise ValueError(f"w must be [vocab, {x.shape[1]}], not {tuple(w.shape)}")
    _expect("w", w, w.shape, x.dtype, x.device, contiguous=False)
    _channels_contiguous("x", x)
    _channels_contiguous("w", w)
    _require("labels", labels)
    _expect("labels", labels, (x.shape[0],), torch.int32, x.device)
    return adst_xent_problem(code, 0, x.shape[0], x.shape[1], w.shape[0], x.stride(0), w.stride(0))


def linear_cross_entropy(x, w, labels, stream=None):
    """The softmax cross entropy of each row of x [rows, width] over the vocabulary w
    [vocab, width] of x's dtype: with logits x @ w.T, lse = log(sum(exp(logits))) and
    loss = lse - logits[label]. labels [rows] int32; a row whose label is outside [0, vocab) (as
    -1 is) has loss 0. The logits are not held. x and w may have any strides between rows. Returns
    a dict: loss and lse [rows], in float32 (float64 for float64 inputs)."""
    if stream is None:
        done = _binding().linear_cross_entropy(x, w, labels)
        if done is not None:
            return done
    import torch
    prob = _xent_problem(x, w, labels)
    info = adst_linear_cross_entropy_plan(prob)

    def body(handle):
        loss = torch.empty(prob.rows, dtype=_acc(prob.dtype), device=x.device)
        lse = torch.empty_like(loss)
        ws = _bytes(info.workspace_bytes, x.device)
        _check(lib().adst_linear_cross_entropy_forward(prob, x.data_ptr(), w.data_ptr(),
                                                       labels.data_ptr(), loss.data_ptr(),
                                                       lse.data_ptr(), _at(ws),
                                                       info.workspace_bytes, handle))
        return {"loss": loss, "lse": lse}

    return _call(x.device, stream, (x, w, labels), body)


def linear_cross_entropy_vjp(x, w, labels, lse, dloss=None, want_dx=True, want_dw=True,
                             stream=None):
    """The VJP of linear_cross_entropy: lse as it gave it, dloss = dL/dloss [rows] like lse (ones
    if None). Returns a dict: dx and dw like x and w (contiguous), each None unless wanted. A row
    without a label, or whose dloss is 0, adds nothing to dw, whatever it holds. The logits are
    computed again, for a piece of the vocabulary at a time; beside 16-bit types their gradients
    are rounded to the type (give x and w in float32 for 32 bits of them)."""
    if stream is None:
        done = _binding().linear_cross_entropy_vjp(x, w, labels, lse, dloss, want_dx, want_dw)
        if done is not None:
            return done
    import torch
    prob = _xent_problem(x, w, labels)
    acc = _acc(prob.dtype)
    _require("lse", lse)
    _expect("lse", lse, (prob.rows,), acc, x.device)
    _expect("dloss", dloss, (prob.rows,), acc, x.device)
    info = adst_linear_cross_entropy_plan(prob)

    def body(handle):
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want_dx else None
        dw = torch.empty_like(w, memory_format=torch.contiguous_format) if want_dw else None
        ws = _bytes(info.vjp_workspace_bytes, x.device)
        _check(lib().adst_linear_cross_entropy_vjp(prob, x.data_ptr(), w.data_ptr(),
                                                   labels.data_ptr(), lse.data_ptr(), _at(dloss),
                                                   _at(dx), _at(dw), _at(ws),
                                                   info.vjp_workspace_bytes, handle))
        return {"dx": dx, "dw": dw}

    return _call(x.device, stream, (x, w, labels, lse, dloss), body)
