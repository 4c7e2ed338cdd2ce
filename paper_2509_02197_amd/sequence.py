"""The sequence operators of adst.h from Python: the gated linear recurrence
with its VJP and its one-step form, layer norm with its VJP, and AdamW over
many tensors.

The ``adst_*`` functions keep the C names and only marshal arguments. The
others take torch tensors, check them, allocate outputs and workspaces with
torch and make the call. Errors in the arguments are ValueError or TypeError
before anything is launched. A call runs on torch's current stream, or on
`stream`; then its outputs and workspaces belong to that stream, and its
inputs are recorded as used there.
"""
import ctypes
import os
from operator import attrgetter

import numpy as np

from . import build as _build
from . import (ADST_BF16, ADST_ERR_HIP, ADST_F16, ADST_F32, ADST_F64, ADST_GATE_COEFF,
               ADST_GATE_SIGMOID, ADST_OK, ADST_STATE_BLOCK, AdstError, _check, _ptr, _stream, adst_adamw_problem,
               adst_adamw_tensor, adst_norm_problem, adst_recurrence_info,
               adst_recurrence_problem, lib)


# ------------------------------------------------------------ the C calls
def adst_recurrence_plan(prob):
    info = adst_recurrence_info()
    _check(lib().adst_recurrence_plan(ctypes.byref(prob), ctypes.byref(info)))
    return info


def adst_recurrence_forward(prob, a, u, h0, lens, h, hT, ck, ws, ws_bytes, stream=None):
    _check(lib().adst_recurrence_forward(ctypes.byref(prob), _ptr(a), _ptr(u), _ptr(h0),
                                         _ptr(lens), _ptr(h), _ptr(hT), _ptr(ck), _ptr(ws),
                                         ws_bytes, _stream(stream)))


def adst_recurrence_vjp(prob, a, u, h0, lens, ck, dh, dhT, da, du, dh0, ws, ws_bytes,
                        stream=None):
    _check(lib().adst_recurrence_vjp(ctypes.byref(prob), _ptr(a), _ptr(u), _ptr(h0), _ptr(lens),
                                     _ptr(ck), _ptr(dh), _ptr(dhT), _ptr(da), _ptr(du),
                                     _ptr(dh0), _ptr(ws), ws_bytes, _stream(stream)))


def adst_recurrence_step(prob, a, u, slots, state, nstates, h, stream=None):
    _check(lib().adst_recurrence_step(ctypes.byref(prob), _ptr(a), _ptr(u), _ptr(slots),
                                      _ptr(state), nstates, _ptr(h), _stream(stream)))


def adst_layer_norm_forward(prob, x, w, b, y, mean, rstd, stream=None):
    _check(lib().adst_layer_norm_forward(ctypes.byref(prob), _ptr(x), _ptr(w), _ptr(b), _ptr(y),
                                         _ptr(mean), _ptr(rstd), _stream(stream)))


def adst_layer_norm_workspace_bytes(prob):
    return int(lib().adst_layer_norm_workspace_bytes(ctypes.byref(prob)))


def adst_layer_norm_vjp(prob, x, dy, w, mean, rstd, dx, dw, db, ws, ws_bytes, stream=None):
    _check(lib().adst_layer_norm_vjp(ctypes.byref(prob), _ptr(x), _ptr(dy), _ptr(w), _ptr(mean),
                                     _ptr(rstd), _ptr(dx), _ptr(dw), _ptr(db), _ptr(ws),
                                     ws_bytes, _stream(stream)))


def adst_adamw(prob, tensors, n, stream=None):
    """tensors: a ctypes array of adst_adamw_tensor."""
    _check(lib().adst_adamw(ctypes.byref(prob), tensors, n, _stream(stream)))


# ------------------------------------------------------------------ checks
_BINDING = None


def _binding():
    """The native form of this file's ordinary calls (csrc/binding.cpp): it answers None to
    anything else, which the code here then handles, and raises what HIP fails."""
    global _BINDING
    if _BINDING is None:
        import torch  # noqa: F401  (whose libraries the binding is linked with)
        lib()
        if not os.path.exists(_build.BINDING):
            _build.build()
        from . import _binding as module
        module.error = AdstError
        _BINDING = module
    return _BINDING


_CODES = None


def _codes():
    global _CODES
    if _CODES is None:
        import torch
        _CODES = {torch.float64: ADST_F64, torch.float32: ADST_F32, torch.bfloat16: ADST_BF16,
                  torch.float16: ADST_F16}
    return _CODES


def _code(name, t):
    if not hasattr(t, "data_ptr"):
        raise ValueError(f"{name} must be a torch tensor")
    code = (_CODES or _codes()).get(t.dtype)
    if code is None:
        raise TypeError(f"{name} has unsupported dtype {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU, not {t.device}")
    return code


def _acc(code):
    """The accumulation type: that of states, statistics and their gradients."""
    import torch
    return torch.float64 if code == ADST_F64 else torch.float32


def _expect(name, t, shape, dtype, device, contiguous=True):
    if t is None:
        return
    try:  # what a right tensor passes at once
        if t.dtype is dtype and t.shape == shape and t.device == device and \
                (not contiguous or t.is_contiguous()):
            return
    except AttributeError:
        pass
    if isinstance(name, tuple):
        name = "{}[{}]".format(*name)
    if not hasattr(t, "data_ptr"):
        raise ValueError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, not {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _require(name, t):
    if not hasattr(t, "data_ptr"):
        raise ValueError(f"{name} is required" if t is None else f"{name} must be a torch tensor")


def _expect_all(name, tensors, shapes, dtype, device):
    """_expect for a list: what a right list passes at once, then one by one for the message."""
    import torch
    kind = torch.Tensor
    try:
        if list(map(_shape_of, tensors)) == shapes and set(map(_dtype_of, tensors)) == {dtype} and \
                set(map(kind.get_device, tensors)) == {device.index} and \
                all(map(kind.is_contiguous, tensors)):
            return
    except (AttributeError, TypeError):
        pass
    for i, (t, shape) in enumerate(zip(tensors, shapes)):
        _require(f"{name}[{i}]", t)
        _expect((name, i), t, shape, dtype, device)


def _channels_contiguous(name, t):
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}'s last axis must be contiguous (stride 1, not {t.stride(-1)})")


def _call(device, stream, inputs, body):
    """body(stream handle) on the tensors' device, allocations of body included."""
    import torch
    if stream is None and torch._C._cuda_getDevice() == device.index:
        return body(torch._C._cuda_getCurrentRawStream(device.index))
    with torch.cuda.device(device):
        if stream is None:
            return body(torch.cuda.current_stream(device).cuda_stream)
        handle = _stream(stream)
        on = (torch.cuda.ExternalStream(handle, device=device) if handle
              else torch.cuda.default_stream(device))
        with torch.cuda.stream(on):
            for t in inputs:
                if t is not None:
                    t.record_stream(on)
            return body(handle)


def _bytes(n, device):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _check_in_place(status, tensors):
    """_check of a call that writes the tensors in place: autograd's checks of saved tensors are
    to see the change."""
    import torch
    if status in (ADST_OK, ADST_ERR_HIP):
        torch.autograd.graph.increment_version(tensors)
    _check(status)


def _at(t):
    return None if t is None else t.data_ptr()


# -------------------------------------------------------------- recurrence
def _recurrence_problem(a, u, gate, dh=None):
    code = _code("a", a)
    if a.dim() != 3:
        raise ValueError(f"a must be [batch, steps, channels], not {tuple(a.shape)}")
    _require("u", u)
    _expect("u", u, a.shape, a.dtype, a.device, contiguous=False)
    _channels_contiguous("a", a)
    _channels_contiguous("u", u)
    B, T, D = a.shape
    sd = (0, 0)
    if dh is not None:
        _expect("dh", dh, a.shape, a.dtype, a.device, contiguous=False)
        _channels_contiguous("dh", dh)
        sd = (dh.stride(0), dh.stride(1))
    return adst_recurrence_problem(code, gate, B, T, D, a.stride(0), a.stride(1), u.stride(0),
                                   u.stride(1), *sd)


def _check_lens(lens, a):
    import torch
    _expect("lens", lens, (a.shape[0],), torch.int32, a.device)


def recurrence(a, u, h0=None, lens=None, gate=ADST_GATE_COEFF, want_h=True, want_ck=False,
               stream=None):
    """h_t = c_t * h_{t-1} + d_t over axis 1 of a, u [batch, steps, channels], with
    (c, d) = (a, u), or (s, (1 - s) * u), s = sigmoid(a), for ADST_GATE_SIGMOID. The products of
    consecutive coefficients have to stay in range, which abs(a) <= 1 ensures.

    h0 [batch, channels] (zeros if None), in float32 (float64 for float64 inputs); lens
    [batch] int32: the steps of each row. a and u may have any strides with contiguous
    channels. Returns a dict: h (None unless want_h), hT the last states, and ck (None unless
    want_ck) the checkpoints with which recurrence_vjp recomputes the states."""
    if stream is None:
        done = _binding().recurrence(a, u, h0, lens, gate, want_h, want_ck)
        if done is not None:
            return done
    import torch
    prob = _recurrence_problem(a, u, gate)
    B, T, D = a.shape
    acc = _acc(prob.dtype)
    _expect("h0", h0, (B, D), acc, a.device)
    _check_lens(lens, a)
    info = adst_recurrence_plan(prob)

    def body(handle):
        h = torch.empty_like(a, memory_format=torch.contiguous_format) if want_h else None
        hT = torch.empty((B, D), dtype=acc, device=a.device)
        ck = _bytes(info.ck_bytes, a.device) if want_ck else None
        ws = _bytes(info.workspace_bytes, a.device)
        _check(lib().adst_recurrence_forward(prob, a.data_ptr(), u.data_ptr(), _at(h0), _at(lens),
                                             _at(h), hT.data_ptr(), _at(ck), _at(ws),
                                             info.workspace_bytes, handle))
        return {"h": h, "hT": hT, "ck": ck}

    return _call(a.device, stream, (a, u, h0, lens), body)


def recurrence_vjp(a, u, dh, h0=None, lens=None, dhT=None, ck=None, gate=ADST_GATE_COEFF,
                   stream=None):
    """The VJP of recurrence: dh = dL/dh, dhT = dL/dhT (optional). ck: the checkpoints that
    recurrence gave for the same a, u, h0, lens and gate; None recomputes them, at the price of
    one more pass over a and u. Returns a dict: da, du [batch, steps, channels] and dh0."""
    if stream is None:
        done = _binding().recurrence_vjp(a, u, dh, h0, lens, dhT, ck, gate)
        if done is not None:
            return done
    import torch
    _require("dh", dh)
    prob = _recurrence_problem(a, u, gate, dh)
    B, T, D = a.shape
    acc = _acc(prob.dtype)
    _expect("h0", h0, (B, D), acc, a.device)
    _expect("dhT", dhT, (B, D), acc, a.device)
    _check_lens(lens, a)
    info = adst_recurrence_plan(prob)
    _expect("ck", ck, (info.ck_bytes,), torch.uint8, a.device)
    need = info.workspace_bytes if ck is not None else info.vjp_workspace_bytes

    def body(handle):
        da = torch.empty_like(a, memory_format=torch.contiguous_format)
        du = torch.empty_like(da)
        dh0 = torch.empty((B, D), dtype=acc, device=a.device)
        ws = _bytes(need, a.device)
        _check(lib().adst_recurrence_vjp(prob, a.data_ptr(), u.data_ptr(), _at(h0), _at(lens),
                                         _at(ck), dh.data_ptr(), _at(dhT), da.data_ptr(),
                                         du.data_ptr(), dh0.data_ptr(), _at(ws), need, handle))
        return {"da": da, "du": du, "dh0": dh0}

    return _call(a.device, stream, (a, u, dh, h0, lens, dhT, ck), body)


def recurrence_step(a, u, state, slots=None, gate=ADST_GATE_COEFF, stream=None):
    """One step of every row of a, u [batch, channels] on the pool of states
    [nstates, channels] (float32, float64 for float64 inputs), updated in place. slots [batch]
    int32: each row's state, no two the same; None: row b's is state[b]. Rows whose slot is
    outside the pool are idle: their h is 0. Returns h [batch, channels]."""
    if stream is None:
        h = _binding().recurrence_step(a, u, state, slots, gate)
        if h is not None:
            return h
    import torch
    code = _code("a", a)
    if a.dim() != 2:
        raise ValueError(f"a must be [batch, channels], not {tuple(a.shape)}")
    B, D = a.shape
    _require("u", u)
    _expect("u", u, (B, D), a.dtype, a.device, contiguous=False)
    _channels_contiguous("a", a)
    _channels_contiguous("u", u)
    _require("state", state)
    if state.dim() != 2 or state.shape[1] != D:
        raise ValueError(f"state must be [nstates, {D}]")
    _expect("state", state, state.shape, _acc(code), a.device)
    _expect("slots", slots, (B,), torch.int32, a.device)
    prob = adst_recurrence_problem(code, gate, B, 1, D, a.stride(0), 0, u.stride(0), 0, 0, 0)

    def body(handle):
        h = torch.empty_like(a, memory_format=torch.contiguous_format)
        _check_in_place(lib().adst_recurrence_step(prob, a.data_ptr(), u.data_ptr(), _at(slots),
                                                   state.data_ptr(), state.shape[0],
                                                   h.data_ptr(), handle), (state,))
        return h

    return _call(a.device, stream, (a, u, state, slots), body)


# -------------------------------------------------------------- layer norm
def _rows(name, t, n):
    """Rows and row stride of t [..., n], whose leading axes have to merge into one."""
    if t.dim() < 1 or t.shape[-1] != n:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not [..., {n}]")
    _channels_contiguous(name, t)
    if t.dim() == 1:
        return 1, n
    if t.dim() == 2 or t.is_contiguous():
        return t.numel() // n, t.stride(0) if t.dim() == 2 else n
    rows, stride = 1, None
    for size, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride = s
        elif s != stride * rows:
            raise ValueError(f"{name}'s leading axes must be one axis of equally spaced rows")
        rows *= size
    return rows, n if stride is None else stride


def _norm_problem(x, w, b, eps, dy=None):
    code = _code("x", x)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"x must be [..., n] with n >= 1, not {tuple(x.shape)}")
    n = x.shape[-1]
    if x.is_contiguous():
        rows, sx = x.numel() // n, n
    else:
        rows, sx = _rows("x", x, n)
    sdy = n
    if dy is not None:
        _expect("dy", dy, x.shape, x.dtype, x.device, contiguous=False)
        _, sdy = _rows("dy", dy, n)
    wcode = code
    given = w if w is not None else b
    if given is not None:
        wcode = (_CODES or _codes()).get(getattr(given, "dtype", None), -1)
        if wcode != code and not (code in (ADST_BF16, ADST_F16) and wcode == ADST_F32):
            raise ValueError(f"weights must be {x.dtype} (or float32 beside 16-bit types), "
                             f"not {getattr(given, 'dtype', type(given))}")
        _expect("w", w, (n,), given.dtype, x.device)
        _expect("b", b, (n,), given.dtype, x.device)
    return adst_norm_problem(code, wcode, rows, n, sx, sdy, eps)


def layer_norm(x, w=None, b=None, eps=1e-5, stream=None):
    """Layer norm over the last axis of x [..., n]; w and b [n] of x's dtype, or float32 beside
    16-bit types. Returns a dict: y (contiguous), and mean and rstd of each row (float32, or
    float64 for float64) for layer_norm_vjp."""
    if stream is None:
        done = _binding().layer_norm(x, w, b, eps)
        if done is not None:
            return done
    import torch
    prob = _norm_problem(x, w, b, eps)
    acc = _acc(prob.dtype)

    def body(handle):
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        mean = torch.empty(x.shape[:-1], dtype=acc, device=x.device)
        rstd = torch.empty_like(mean)
        _check(lib().adst_layer_norm_forward(prob, x.data_ptr(), _at(w), _at(b), y.data_ptr(),
                                             mean.data_ptr(), rstd.data_ptr(), handle))
        return {"y": y, "mean": mean, "rstd": rstd}

    return _call(x.device, stream, (x, w, b), body)


def layer_norm_vjp(x, dy, mean, rstd, w=None, want_dx=True, want_dw=True, want_db=True,
                   stream=None):
    """The VJP of layer_norm: mean and rstd as it gave them. Returns a dict: dx [..., n]
    (contiguous), dw and db [n] in w's dtype (x's without w), each None unless wanted."""
    if stream is None:
        done = _binding().layer_norm_vjp(x, dy, mean, rstd, w, want_dx, want_dw, want_db)
        if done is not None:
            return done
    import torch
    _require("dy", dy)
    prob = _norm_problem(x, w, None, 0.0, dy)
    acc = _acc(prob.dtype)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _require(name, t)
        _expect(name, t, x.shape[:-1], acc, x.device)
    wt = w.dtype if w is not None else x.dtype

    def body(handle):
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want_dx else None
        dw = torch.empty(prob.n, dtype=wt, device=x.device) if want_dw else None
        db = torch.empty(prob.n, dtype=wt, device=x.device) if want_db else None
        need = adst_layer_norm_workspace_bytes(prob) if want_dw or want_db else 0
        ws = _bytes(need, x.device)
        _check(lib().adst_layer_norm_vjp(prob, x.data_ptr(), dy.data_ptr(), _at(w),
                                         mean.data_ptr(), rstd.data_ptr(), _at(dx), _at(dw),
                                         _at(db), _at(ws), need, handle))
        return {"dx": dx, "dw": dw, "db": db}

    return _call(x.device, stream, (x, dy, mean, rstd, w), body)


# ------------------------------------------------------------------- AdamW
_dtype_of, _shape_of = attrgetter("dtype"), attrgetter("shape")


class AdamW:
    """AdamW over a list of tensors, one call a step, updated in place.

    params: contiguous float32 (or float64) tensors on one GPU, none of which shares memory with
    another (a tied weight is listed once). bits: 32 for states in the
    parameters' type, 8 for blocks of 256 e4m3 codes with a scale each (float32 parameters).
    state: {"m", "v"} (and "m_scale", "v_scale" with 8 bits), lists of tensors like those this
    object holds under these names, to go on from; zeros if None. copies: contiguous tensors
    shaped like params, one dtype of float32, bfloat16 and float16, that receive the new
    parameters in it. lr and weight_decay: a number, or one for each tensor. The lists params,
    m, v, m_scale, v_scale and copies may be replaced by others like them; each step looks up
    and checks what they hold. lr, weight_decay, betas and eps may be assigned between steps."""

    def __init__(self, params, bits=32, state=None, copies=None, lr=1e-3, betas=(0.9, 0.999),
                 eps=1e-8, weight_decay=0.01):
        import torch
        self.params = tuple(params)
        n = len(self.params)
        if n == 0:
            raise ValueError("params is empty")
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        first = self.params[0]
        code = _code("params[0]", first)
        if code not in (ADST_F32, ADST_F64) or (bits == 8 and code == ADST_F64):
            raise TypeError(f"parameters must be float32, or float64 with 32-bit states, "
                            f"not {first.dtype}")
        self.device = first.device
        for i, p in enumerate(self.params):
            _require(f"params[{i}]", p)
        shapes = list(map(_shape_of, self.params))
        _expect_all("params", self.params, shapes, first.dtype, self.device)
        self.copies = None if copies is None else tuple(copies)
        copy_code = ADST_BF16
        if self.copies is not None:
            if len(self.copies) != n:
                raise ValueError(f"{len(self.copies)} copies of {n} parameters")
            copy_code = _code("copies[0]", self.copies[0])
            if copy_code == ADST_F64:
                raise TypeError("copies must be float32, bfloat16 or float16")
            _expect_all("copies", self.copies, shapes, self.copies[0].dtype, self.device)
        self._bits = bits
        self.t = 0
        self._numel = [p.numel() for p in self.params]
        blocks = [(-(-k // ADST_STATE_BLOCK),) for k in self._numel]
        self._states = ("m", "v", "m_scale", "v_scale") if bits == 8 else ("m", "v")
        # what each list holds: the tensors' shapes and type
        self._held = {"params": (shapes, first.dtype)}
        if self.copies is not None:
            self._held["copies"] = shapes, self.copies[0].dtype
        for name in self._states:
            self._held[name] = (
                (blocks, torch.float32) if name.endswith("scale") else
                (shapes, torch.float8_e4m3fn if bits == 8 else first.dtype))
            needed, dtype = self._held[name]
            if state is None:
                held = tuple(torch.zeros(s, dtype=dtype, device=self.device) for s in needed)
            else:
                if name not in state:
                    raise ValueError(f"state has no {name}")
                held = tuple(state[name])
                if len(held) != n:
                    raise ValueError(f"{len(held)} tensors of state {name} for {n} parameters")
                _expect_all(name, held, needed, dtype, self.device)
            setattr(self, name, held)
        for name in self._held:
            at = [x for x in map(torch.Tensor.data_ptr, getattr(self, name)) if x]
            if len(set(at)) < len(at):  # two workgroups would update the same values
                raise ValueError(f"{name} has the same tensor twice")
        self._n = n
        self._rows = (adst_adamw_tensor * n)()
        # the same memory as 8-byte words: p, grad, m, v, m_scale, v_scale, copy, n, lr, decay
        self._words = np.frombuffer(self._rows, dtype=np.uint64).reshape(n, -1)
        self._words[:, 7] = self._numel
        self._prob = adst_adamw_problem(code, ADST_F32, copy_code, bits)
        self.lr, self.weight_decay, self.betas, self.eps = lr, weight_decay, betas, eps
        self._descriptors = ctypes.addressof(self._prob), ctypes.addressof(self._rows), n

    def _expect_held(self):
        """The lists hold what they did when this object was made: another list, or other memory
        (which a module gives its parameters when it is moved), is taken where it is alike."""
        if self.copies is not None and "copies" not in self._held:
            raise ValueError("copies were not there when the object was made")
        for name, (shapes, dtype) in self._held.items():
            tensors = getattr(self, name)
            if name == "copies" and tensors is None:
                continue
            if len(tensors) != self._n:
                raise ValueError(f"{len(tensors)} {name} for {self._n} parameters")
            _expect_all(name, tensors, shapes, dtype, self.device)

    def _rates(self, name, value, word):
        """value, one number or one for each tensor, into the descriptors."""
        values = [value] * self._n if isinstance(value, (int, float)) else list(value)
        if len(values) != self._n:
            raise ValueError(f"{len(values)} values of {name} for {self._n} parameters")
        self._words.view(np.float64)[:, word] = values
        return value

    # What the descriptors hold is changed with the attribute.
    @property
    def lr(self):
        return self._lr

    @lr.setter
    def lr(self, value):
        self._lr = self._rates("lr", value, 8)

    @property
    def weight_decay(self):
        return self._weight_decay

    @weight_decay.setter
    def weight_decay(self, value):
        self._weight_decay = self._rates("weight_decay", value, 9)

    @property
    def betas(self):
        return self._prob.beta1, self._prob.beta2

    @betas.setter
    def betas(self, value):
        self._prob.beta1, self._prob.beta2 = map(float, value)

    @property
    def eps(self):
        return self._prob.eps

    @eps.setter
    def eps(self, value):
        self._prob.eps = float(value)

    @property
    def bits(self):  # of the states that this object was made with
        return self._bits

    def step(self, grads, lr=None, weight_decay=None, t=None, grad_scale=None, stream=None):
        """One step with contiguous gradients like params (float32, bfloat16 or float16, one
        dtype; float64 for float64). lr, weight_decay: from now on. t: the step's number, one more
        than the last one's if None. grad_scale: a float32 tensor of one value that multiplies the
        gradients; where it is not finite nothing is updated (the step's number counts on)."""
        if lr is not None:
            self.lr = lr
        if weight_decay is not None:
            self.weight_decay = weight_decay
        if t is None:
            t = self.t + 1
        states = ((self.m, self.v, self.m_scale, self.v_scale) if self.bits == 8 else
                  (self.m, self.v))
        if stream is None and _binding().adamw_step(*self._descriptors, self.params, states,
                                                    grads, self.copies, grad_scale, t):
            self.t = t
            return
        import torch
        self._expect_held()
        if len(grads) != self._n:
            raise ValueError(f"{len(grads)} gradients for {self._n} parameters")
        code = _code("grads[0]", grads[0])
        if (code == ADST_F64) != (self._prob.dtype == ADST_F64):
            raise TypeError(f"gradients of {self.params[0].dtype} parameters in {grads[0].dtype}")
        device, kind = self.device, torch.Tensor
        try:  # what a right list passes at once
            right = set(map(_dtype_of, grads)) == {grads[0].dtype} and \
                set(map(kind.get_device, grads)) == {device.index} and \
                list(map(kind.numel, grads)) == self._numel and \
                all(map(kind.is_contiguous, grads))
        except (AttributeError, TypeError):
            right = False
        for i, (g, n) in enumerate(() if right else zip(grads, self._numel)):
            _require(f"grads[{i}]", g)
            if g.dtype != grads[0].dtype or g.device != device or g.numel() != n or \
                    not g.is_contiguous():
                raise ValueError(f"grads[{i}] must be contiguous, of {n} values in "
                                 f"{grads[0].dtype} on {device}")
        rows = self._rows
        self._words[:, 0] = list(map(kind.data_ptr, self.params))
        self._words[:, 1] = list(map(kind.data_ptr, grads))
        for word, tensors in enumerate(states, 2):
            self._words[:, word] = list(map(kind.data_ptr, tensors))
        self._words[:, 6] = 0 if self.copies is None else list(map(kind.data_ptr, self.copies))
        if grad_scale is not None:
            _require("grad_scale", grad_scale)
            _expect("grad_scale", grad_scale, grad_scale.shape, torch.float32, device)
            if grad_scale.numel() != 1:
                raise ValueError("grad_scale must have one value")
        prob = self._prob
        prob.grad_dtype = code
        prob.t = t
        prob.grad_scale = None if grad_scale is None else grad_scale.data_ptr()
        written = (*self.params, *(self.copies or ()), *(t for held in states for t in held))
        used = () if stream is None else (*written, *grads, grad_scale)
        _call(device, stream, used, lambda handle: _check_in_place(
            lib().adst_adamw(prob, rows, self._n, handle), written))
        self.t = prob.t
