// The ordinary calls of sequence.py, from tensors to the C call without Python
// in between: a small call's time is the host's, and each attribute that
// Python looks up is a good part of it (layer norm of 32 rows: 10.1 us through
// Python, 6.7 from here, of which 3 are the launch; one step of AdamW over 121
// tensors: 37 and 14). Each function returns None for anything that is not
// ordinary (a wrong or unusual argument, tensors on another device than the
// current one), before anything is launched; sequence.py then goes its own
// way, which handles the unusual and raises the errors. A call that HIP fails
// may have launched some of its work: it is never made again but raises
// sequence.py's AdstError. Nothing else here throws into Python.

#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "adst.h"

namespace {

typedef PyObject* const* Args;

struct Odd {};  // not an ordinary call
struct Failed {  // a call that HIP failed
  adst_status status;
};

void need(bool ok) {
  if (!ok) throw Odd();
}

at::Tensor tensor(PyObject* o) {
  need(THPVariable_Check(o));
  return THPVariable_Unpack(o);
}
at::Tensor maybe(PyObject* o) { return o == Py_None ? at::Tensor() : tensor(o); }
void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

int code_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kDouble: return ADST_F64;
    case at::kFloat: return ADST_F32;
    case at::kBFloat16: return ADST_BF16;
    case at::kHalf: return ADST_F16;
    default: throw Odd();
  }
}
at::ScalarType acc_of(int code) { return code == ADST_F64 ? at::kDouble : at::kFloat; }

// The current device, if the tensor is there, and its current stream.
struct Here {
  c10::Device device;
  hipStream_t stream;
};
Here here(const at::Tensor& t) {
  need(t.is_cuda());
  const c10::DeviceIndex current = c10::hip::current_device();
  need(t.get_device() == current);
  return {t.device(), c10::hip::getCurrentHIPStream(current).stream()};
}

void same(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, const Here& h,
          bool contiguous) {
  if (!t.defined()) return;
  need(t.scalar_type() == type && t.sizes() == shape && t.device() == h.device &&
       (contiguous ? t.is_contiguous() : t.size(-1) < 2 || t.stride(-1) == 1));
}

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, const Here& h) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(h.device));
}
at::Tensor bytes(uint64_t n, const Here& h) {
  return n ? make({(int64_t)n}, at::kByte, h) : at::Tensor();
}

void run(adst_status s) {
  if (s == ADST_ERR_HIP) throw Failed{s};
  need(s == ADST_OK);
}

// A tensor that a call writes in place: autograd's checks of saved tensors are
// to see the change.
void changed(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// {name: tensor or None}
class Dict {
 public:
  Dict() : d_(PyDict_New()) { need(d_); }
  ~Dict() { Py_XDECREF(d_); }
  void put(const char* name, const at::Tensor& t) {
    PyObject* v = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    need(v);
    const int r = PyDict_SetItemString(d_, name, v);
    Py_DECREF(v);
    need(r == 0);
  }
  PyObject* take() {
    PyObject* d = d_;
    d_ = nullptr;
    return d;
  }

 private:
  PyObject* d_;
  Dict(const Dict&) = delete;
};

int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  need(!(v == -1 && PyErr_Occurred()));
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  need(!(v == -1.0 && PyErr_Occurred()));
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  need(v >= 0);
  return v != 0;
}

// Sets the module's error, AdstError(status, text), or what keeps it from that.
PyObject* raise(PyObject* module, adst_status status) {
  PyObject* const error = PyObject_GetAttrString(module, "error");
  if (!error) return nullptr;
  PyObject* const text =
      PyUnicode_FromFormat("%s: %s", adst_status_str(status), adst_last_error());
  PyObject* const args = text ? Py_BuildValue("(iN)", (int)status, text) : nullptr;
  if (args) PyErr_SetObject(error, args);
  Py_XDECREF(args);
  Py_DECREF(error);
  return nullptr;
}

template <class F>
PyObject* ordinary(PyObject* module, F f) {
  try {
    return f();
  } catch (const Failed& failed) {
    return raise(module, failed.status);
  } catch (...) {
    PyErr_Clear();
    return Py_NewRef(Py_None);
  }
}

// ---------------------------------------------------------------- layer norm
// The problem for x [..., n] contiguous (dy too), w and b [n] or undefined.
adst_norm_problem norm_problem(const at::Tensor& x, const at::Tensor& dy, const at::Tensor& w,
                               const at::Tensor& b, double eps, const Here& h) {
  need(x.dim() >= 1 && x.size(-1) >= 1 && x.is_contiguous());
  const int64_t n = x.size(-1);
  const int code = code_of(x);
  same(dy, x.sizes(), x.scalar_type(), h, true);
  int wcode = code;
  const at::Tensor& given = w.defined() ? w : b;
  if (given.defined()) {
    wcode = code_of(given);
    need(wcode == code || (wcode == ADST_F32 && (code == ADST_BF16 || code == ADST_F16)));
    same(w, {n}, given.scalar_type(), h, true);
    same(b, {n}, given.scalar_type(), h, true);
  }
  return {code, wcode, x.numel() / n, n, n, n, eps};
}

// (x, w, b, eps)
PyObject* layer_norm(PyObject* module, Args a, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 4);
    const at::Tensor x = tensor(a[0]), w = maybe(a[1]), b = maybe(a[2]);
    const Here h = here(x);
    const adst_norm_problem p = norm_problem(x, {}, w, b, number(a[3]), h);
    const at::ScalarType acc = acc_of(p.dtype);
    const at::IntArrayRef rows = x.sizes().slice(0, x.dim() - 1);
    const at::Tensor y = at::empty_like(x), mean = make(rows, acc, h), rstd = make(rows, acc, h);
    Dict d;
    d.put("y", y);
    d.put("mean", mean);
    d.put("rstd", rstd);
    run(adst_layer_norm_forward(&p, x.data_ptr(), at_of(w), at_of(b), y.data_ptr(),
                                mean.data_ptr(), rstd.data_ptr(), h.stream));
    return d.take();
  });
}

// (x, dy, mean, rstd, w, want_dx, want_dw, want_db)
PyObject* layer_norm_vjp(PyObject* module, Args a, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 8);
    const at::Tensor x = tensor(a[0]), dy = tensor(a[1]), mean = tensor(a[2]), rstd = tensor(a[3]),
                     w = maybe(a[4]);
    const Here h = here(x);
    const adst_norm_problem p = norm_problem(x, dy, w, {}, 0.0, h);
    const at::IntArrayRef rows = x.sizes().slice(0, x.dim() - 1);
    same(mean, rows, acc_of(p.dtype), h, true);
    same(rstd, rows, acc_of(p.dtype), h, true);
    const bool dx_ = truth(a[5]), dw_ = truth(a[6]), db_ = truth(a[7]);
    const at::ScalarType wt = w.defined() ? w.scalar_type() : x.scalar_type();
    const at::Tensor none, dx = dx_ ? at::empty_like(x) : none,
                     dw = dw_ ? make({p.n}, wt, h) : none, db = db_ ? make({p.n}, wt, h) : none;
    const uint64_t need_bytes = dw_ || db_ ? adst_layer_norm_workspace_bytes(&p) : 0;
    const at::Tensor ws = bytes(need_bytes, h);
    Dict d;
    d.put("dx", dx);
    d.put("dw", dw);
    d.put("db", db);
    run(adst_layer_norm_vjp(&p, x.data_ptr(), dy.data_ptr(), at_of(w), mean.data_ptr(),
                            rstd.data_ptr(), at_of(dx), at_of(dw), at_of(db), at_of(ws),
                            need_bytes, h.stream));
    return d.take();
  });
}

// ---------------------------------------------------------------- recurrence
adst_recurrence_problem recurrence_problem(const at::Tensor& a, const at::Tensor& u,
                                           const at::Tensor& dh, int64_t gate, const Here& h) {
  need(a.dim() == 3);
  same(a, a.sizes(), a.scalar_type(), h, false);
  same(u, a.sizes(), a.scalar_type(), h, false);
  same(dh, a.sizes(), a.scalar_type(), h, false);
  adst_recurrence_problem p{};
  p.dtype = code_of(a);
  p.gate = (int32_t)gate;
  p.batch = a.size(0);
  p.steps = a.size(1);
  p.channels = a.size(2);
  for (int i = 0; i < 2; ++i) {
    p.stride_a[i] = a.stride(i);
    p.stride_u[i] = u.stride(i);
    p.stride_dh[i] = dh.defined() ? dh.stride(i) : 0;
  }
  return p;
}
void states(const adst_recurrence_problem& p, const at::Tensor& t, const Here& h) {
  same(t, {p.batch, p.channels}, acc_of(p.dtype), h, true);
}
at::Tensor like(const at::Tensor& a) { return at::empty_like(a, at::MemoryFormat::Contiguous); }

// (a, u, h0, lens, gate, want_h, want_ck)
PyObject* recurrence(PyObject* module, Args x, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 7);
    const at::Tensor a = tensor(x[0]), u = tensor(x[1]), h0 = maybe(x[2]), lens = maybe(x[3]);
    const Here h = here(a);
    const adst_recurrence_problem p = recurrence_problem(a, u, {}, whole(x[4]), h);
    states(p, h0, h);
    same(lens, {p.batch}, at::kInt, h, true);
    adst_recurrence_info info;
    run(adst_recurrence_plan(&p, &info));
    const at::Tensor none, out = truth(x[5]) ? like(a) : none,
                     hT = make({p.batch, p.channels}, acc_of(p.dtype), h),
                     ck = truth(x[6]) ? bytes(info.ck_bytes, h) : none,
                     ws = bytes(info.workspace_bytes, h);
    Dict d;
    d.put("h", out);
    d.put("hT", hT);
    d.put("ck", ck);
    run(adst_recurrence_forward(&p, a.data_ptr(), u.data_ptr(), at_of(h0),
                                static_cast<const int32_t*>(at_of(lens)), at_of(out),
                                hT.data_ptr(), at_of(ck), at_of(ws), info.workspace_bytes,
                                h.stream));
    return d.take();
  });
}

// (a, u, dh, h0, lens, dhT, ck, gate)
PyObject* recurrence_vjp(PyObject* module, Args x, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 8);
    const at::Tensor a = tensor(x[0]), u = tensor(x[1]), dh = tensor(x[2]), h0 = maybe(x[3]),
                     lens = maybe(x[4]), dhT = maybe(x[5]), ck = maybe(x[6]);
    const Here h = here(a);
    const adst_recurrence_problem p = recurrence_problem(a, u, dh, whole(x[7]), h);
    states(p, h0, h);
    states(p, dhT, h);
    same(lens, {p.batch}, at::kInt, h, true);
    adst_recurrence_info info;
    run(adst_recurrence_plan(&p, &info));
    same(ck, {(int64_t)info.ck_bytes}, at::kByte, h, true);
    const uint64_t size = ck.defined() ? info.workspace_bytes : info.vjp_workspace_bytes;
    const at::Tensor da = like(a), du = like(a),
                     dh0 = make({p.batch, p.channels}, acc_of(p.dtype), h), ws = bytes(size, h);
    Dict d;
    d.put("da", da);
    d.put("du", du);
    d.put("dh0", dh0);
    run(adst_recurrence_vjp(&p, a.data_ptr(), u.data_ptr(), at_of(h0),
                            static_cast<const int32_t*>(at_of(lens)), at_of(ck), dh.data_ptr(),
                            at_of(dhT), da.data_ptr(), du.data_ptr(), dh0.data_ptr(), at_of(ws),
                            size, h.stream));
    return d.take();
  });
}

// (a, u, state, slots, gate)
PyObject* recurrence_step(PyObject* module, Args x, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 5);
    const at::Tensor a = tensor(x[0]), u = tensor(x[1]), state = tensor(x[2]), slots = maybe(x[3]);
    const Here h = here(a);
    need(a.dim() == 2 && state.dim() == 2 && state.size(1) == a.size(1));
    same(a, a.sizes(), a.scalar_type(), h, false);
    same(u, a.sizes(), a.scalar_type(), h, false);
    adst_recurrence_problem p{};
    p.dtype = code_of(a);
    p.gate = (int32_t)whole(x[4]);
    p.batch = a.size(0);
    p.steps = 1;
    p.channels = a.size(1);
    p.stride_a[0] = a.stride(0);
    p.stride_u[0] = u.stride(0);
    same(state, state.sizes(), acc_of(p.dtype), h, true);
    same(slots, {p.batch}, at::kInt, h, true);
    const at::Tensor out = like(a);
    PyObject* const r = THPVariable_Wrap(out);
    need(r);
    const adst_status status =
        adst_recurrence_step(&p, a.data_ptr(), u.data_ptr(),
                             static_cast<const int32_t*>(at_of(slots)), state.data_ptr(),
                             state.size(0), out.data_ptr(), h.stream);
    if (status != ADST_OK) Py_DECREF(r);
    if (status == ADST_OK || status == ADST_ERR_HIP) changed(state);
    run(status);
    return r;
  });
}

// --------------------------------------------------------------------- AdamW
// (problem's address, descriptors' address, their number, params, states,
// grads, copies or None, grad_scale or None, t), states the tuple of m and v,
// with 8 bits also of their scales: True where the step was made. The problem
// and the descriptors are the caller's; the addresses, the gradients' type, the
// scale and t are filled in here. What a tensor was when the object was made,
// it has to be at each step.
PyObject* adamw_step(PyObject* module, Args a, Py_ssize_t n) {
  return ordinary(module, [&] {
    need(n == 9 && (PyList_Check(a[5]) || PyTuple_Check(a[5])));
    auto* const prob = static_cast<adst_adamw_problem*>(PyLong_AsVoidPtr(a[0]));
    auto* const rows = static_cast<adst_adamw_tensor*>(PyLong_AsVoidPtr(a[1]));
    need(prob && rows);
    const Py_ssize_t count = (Py_ssize_t)whole(a[2]);
    need(count > 0 && PySequence_Fast_GET_SIZE(a[5]) == count);
    const auto tuple = [count](PyObject* o) {
      need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == count);
      return PySequence_Fast_ITEMS(o);
    };
    const auto held = [](PyObject* o) -> const at::Tensor& {
      need(THPVariable_Check(o));
      return THPVariable_Unpack(o);
    };
    const bool coded = prob->bits == 8;
    need(PyTuple_Check(a[4]) && PyTuple_GET_SIZE(a[4]) == (coded ? 4 : 2));
    PyObject** const params = tuple(a[3]);
    PyObject** const ms = tuple(PyTuple_GET_ITEM(a[4], 0));
    PyObject** const vs = tuple(PyTuple_GET_ITEM(a[4], 1));
    PyObject** const m_scales = coded ? tuple(PyTuple_GET_ITEM(a[4], 2)) : nullptr;
    PyObject** const v_scales = coded ? tuple(PyTuple_GET_ITEM(a[4], 3)) : nullptr;
    PyObject** const copies = a[6] == Py_None ? nullptr : tuple(a[6]);
    PyObject** const grads = PySequence_Fast_ITEMS(a[5]);
    const Here h = here(held(params[0]));
    const at::ScalarType type = held(grads[0]).scalar_type();
    const int code = code_of(held(grads[0]));
    need((code == ADST_F64) == (prob->dtype == ADST_F64));
    const at::ScalarType kind = prob->dtype == ADST_F64 ? at::kDouble : at::kFloat;
    const at::ScalarType state = coded ? at::kFloat8_e4m3fn : kind;
    // the tensor's address, where it is one of `numel` values in order
    const auto at = [&](PyObject* o, at::ScalarType type, int64_t numel) {
      const at::Tensor& t = held(o);
      need(t.scalar_type() == type && t.device() == h.device && t.numel() == numel &&
           t.is_contiguous());
      return t.data_ptr();
    };
    for (Py_ssize_t i = 0; i < count; ++i) {
      adst_adamw_tensor& r = rows[i];
      r.grad = at(grads[i], type, r.n);
      r.p = at(params[i], kind, r.n);
      r.m = at(ms[i], state, r.n);
      r.v = at(vs[i], state, r.n);
      const at::IntArrayRef shape = held(params[i]).sizes();
      need(held(ms[i]).sizes() == shape && held(vs[i]).sizes() == shape);
      if (coded) {
        const int64_t blocks = (r.n + ADST_STATE_BLOCK - 1) / ADST_STATE_BLOCK;
        r.m_scale = static_cast<float*>(at(m_scales[i], at::kFloat, blocks));
        r.v_scale = static_cast<float*>(at(v_scales[i], at::kFloat, blocks));
      }
      r.copy = nullptr;
      if (copies) {
        const at::Tensor& c = held(copies[i]);
        need(code_of(c) == prob->copy_dtype && c.sizes() == shape);
        r.copy = at(copies[i], c.scalar_type(), r.n);
      }
    }
    const at::Tensor scale = maybe(a[7]);
    if (scale.defined())
      need(scale.scalar_type() == at::kFloat && scale.numel() == 1 && scale.device() == h.device);
    prob->grad_dtype = code;
    prob->grad_scale = static_cast<const float*>(at_of(scale));
    prob->t = whole(a[8]);
    const adst_status status = adst_adamw(prob, rows, (int32_t)count, h.stream);
    if (status == ADST_OK || status == ADST_ERR_HIP)
      for (PyObject** list : {params, ms, vs, m_scales, v_scales, copies})
        for (Py_ssize_t i = 0; list && i < count; ++i) changed(held(list[i]));
    run(status);
    return Py_NewRef(Py_True);
  });
}

#define CALL(name) \
  { #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr }
PyMethodDef kMethods[] = {CALL(layer_norm),     CALL(layer_norm_vjp),  CALL(recurrence),
                          CALL(recurrence_vjp), CALL(recurrence_step), CALL(adamw_step),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&kModule); }
