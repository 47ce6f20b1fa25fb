// The binding's marshalling in native code: torch tensors and parameter objects in, one C ABI call
// (include/hago.h) out.  What bounds a small operator is the host: the same work done with ctypes took
// 7 - 8 us of Python per call beside the 2.3 us of the kernel launch itself.
//
// Every function takes the arguments of the binding's function of the same name, positionally, and either
// issues the call on the current stream or (prepare) returns a Prepared object that re-issues it.  The
// library's addresses come from the binding, which loads it: this module links to torch only.
#include <Python.h>

#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <functional>
#include <vector>

#include "../../include/hago.h"

namespace {

// ---- the library's entry points, filled in by bind()
#define HAGO_ENTRIES(X)                                                                                            \
  X(hago_simquant) X(hago_simquant_wrap) X(hago_simquant_batched) X(hago_quantize) X(hago_dequantize)              \
  X(hago_simquant_codes) X(hago_absmax) X(hago_requantize) X(hago_qdense) X(hago_qconv2d) X(hago_qconv2d_ws)       \
  X(hago_qconv2d_static) X(hago_bit_range) X(hago_mx_quantize) X(hago_mx_rmsnorm) X(hago_mx_silu_mul)                 \
  X(hago_mx_dense) X(hago_mx_dense_grouped) X(hago_rope) X(hago_mx_cache_write) X(hago_mx_cache_read)                 \
  X(hago_mx_attention) X(hago_mx_attention_workspace_bytes)
struct Library {
#define X(name) decltype(&::name) name;
  HAGO_ENTRIES(X)
#undef X
} L;
PyObject* g_check = nullptr;  // raises the binding's error for a status

struct Raised {};  // a Python error is set

PyObject* intern(const char* s) { return PyUnicode_InternFromString(s); }

int64_t as_int(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
// int(o): floats, numpy scalars and one-element tensors too
int64_t as_converted_int(PyObject* o) {
  PyObject* k = PyNumber_Long(o);
  if (!k) throw Raised{};
  const long long v = PyLong_AsLongLong(k);
  Py_DECREF(k);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
bool as_bool(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}
int64_t attr_int(PyObject* o, PyObject* name) {
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) throw Raised{};
  const long long r = PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (r == -1 && PyErr_Occurred()) throw Raised{};
  return r;
}
int64_t attr_converted_int(PyObject* o, PyObject* name) {
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) throw Raised{};
  try {
    const int64_t r = as_converted_int(v);
    Py_DECREF(v);
    return r;
  } catch (...) {
    Py_DECREF(v);
    throw;
  }
}
void require(bool ok) {
  if (!ok) {
    PyErr_SetNone(PyExc_AssertionError);
    throw Raised{};
  }
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a torch tensor is needed");
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}
void* pointer(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

void check(hago_status s) {
  if (s == HAGO_OK) return;
  PyObject* r = PyObject_CallFunction(g_check, "i", (int)s);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "libhago call failed");
  throw Raised{};
}

at::ScalarType scalar_type(int64_t code) {
  switch (code) {
    case HAGO_U8: return at::kByte;
    case HAGO_I8: return at::kChar;
    case HAGO_I16: return at::kShort;
    case HAGO_I32: case HAGO_I24: return at::kInt;
    case HAGO_F32: return at::kFloat;
  }
  PyErr_SetObject(PyExc_KeyError, PyLong_FromLongLong(code));
  throw Raised{};
}
// of the microscaled products' results
at::ScalarType product_type(int64_t code) { return code == HAGO_BF16 ? at::kBFloat16 : code == HAGO_F16 ? at::kHalf : scalar_type(code); }

// `given`, or a new tensor of the shape and type on `like`'s device (a new reference either way).
PyObject* output(PyObject* given, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  if (given != Py_None) {
    tensor(given);
    Py_INCREF(given);
    return given;
  }
  PyObject* r = THPVariable_Wrap(at::Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt)));
  if (!r) throw Raised{};
  return r;
}

hago_qtype qtype(PyObject* q) {
  static PyObject *dtype = intern("dtype"), *bits = intern("bits"), *sgn = intern("is_signed"), *zp = intern("zero_point");
  return hago_qtype{(hago_dtype)attr_int(q, dtype), (int32_t)attr_int(q, bits), (int32_t)attr_converted_int(q, sgn), (int32_t)attr_int(q, zp)};
}

struct Ref {  // a reference of our own
  PyObject* o = nullptr;
  Ref() = default;
  Ref(const Ref&) = delete;
  ~Ref() { Py_XDECREF(o); }
};
struct RequantTensors {  // kept by the Prepared object: the attributes they come from may be set to others
  Ref mult, shift;
};

struct MaybeRequant {  // a copy of the caller's parameters
  bool present = false;
  hago_requant rq{};
  const hago_requant* ptr() const { return present ? &rq : nullptr; }
};

MaybeRequant requant(PyObject* o, RequantTensors& tensors) {
  MaybeRequant r;
  if (o == Py_None) return r;
  static PyObject *mult = intern("multiplier"), *shift = intern("shift"), *pc = intern("per_channel"), *out = intern("out"),
                  *lo = intern("clip_lo"), *hi = intern("clip_hi"), *rounding = intern("rounding");
  auto ptr_of = [&](PyObject* name, Ref& t) {
    t.o = PyObject_GetAttr(o, name);
    if (!t.o) throw Raised{};
    return static_cast<const int32_t*>(pointer(t.o));  // (only None is NULL, the shift-only form)
  };
  r.present = true;
  r.rq.multiplier = ptr_of(mult, tensors.mult);
  r.rq.shift = ptr_of(shift, tensors.shift);
  r.rq.per_channel = (int32_t)attr_int(o, pc);
  PyObject* q = PyObject_GetAttr(o, out);
  if (!q) throw Raised{};
  try {
    r.rq.out = qtype(q);
  } catch (...) {
    Py_DECREF(q);
    throw;
  }
  Py_DECREF(q);
  r.rq.clip_lo = (int32_t)attr_int(o, lo);
  r.rq.clip_hi = (int32_t)attr_int(o, hi);
  r.rq.rounding = (int32_t)attr_int(o, rounding);
  return r;
}

// ---- a call with its arguments already marshalled
struct Prepared {
  PyObject_HEAD
  vectorcallfunc vectorcall;
  std::function<hago_status()>* fn;
  PyObject* keep;  // everything the call's pointers belong to
  PyObject* out;
};

PyObject* prepared_call(PyObject* self, PyObject* const*, size_t nargs, PyObject* names) {
  Prepared* p = reinterpret_cast<Prepared*>(self);
  if (PyVectorcall_NARGS(nargs) != 0 || (names && PyTuple_GET_SIZE(names) != 0)) {
    PyErr_SetString(PyExc_TypeError, "a prepared call takes no arguments");
    return nullptr;
  }
  hago_status s;
  Py_BEGIN_ALLOW_THREADS
  s = (*p->fn)();
  Py_END_ALLOW_THREADS
  if (s != HAGO_OK) {
    try {
      check(s);
    } catch (Raised&) {
    }
    return nullptr;
  }
  Py_INCREF(p->out);
  return p->out;
}

int prepared_traverse(PyObject* self, visitproc visit, void* arg) {
  Prepared* p = reinterpret_cast<Prepared*>(self);
  Py_VISIT(p->keep);
  Py_VISIT(p->out);
  return 0;
}
int prepared_clear(PyObject* self) {
  Prepared* p = reinterpret_cast<Prepared*>(self);
  Py_CLEAR(p->keep);
  Py_CLEAR(p->out);
  return 0;
}
void prepared_dealloc(PyObject* self) {
  PyObject_GC_UnTrack(self);
  delete reinterpret_cast<Prepared*>(self)->fn;
  prepared_clear(self);
  Py_TYPE(self)->tp_free(self);
}
PyObject* prepared_out(PyObject* self, void*) {
  PyObject* o = reinterpret_cast<Prepared*>(self)->out;
  Py_INCREF(o);
  return o;
}
int set_prepared_out(PyObject* self, PyObject* value, void*) {
  if (!value) {
    PyErr_SetString(PyExc_AttributeError, "out");
    return -1;
  }
  Py_INCREF(value);
  Py_XSETREF(reinterpret_cast<Prepared*>(self)->out, value);
  return 0;
}
PyGetSetDef prepared_getset[] = {
    {"out", prepared_out, set_prepared_out, "what a call returns: the output tensor(s) (another value does not change where the launch writes)", nullptr}, {}};

PyTypeObject PreparedType = [] {
  PyTypeObject t = {PyVarObject_HEAD_INIT(nullptr, 0)};
  t.tp_name = "paper_2103_14949_amd._native.Prepared";
  t.tp_doc = "A library call with its arguments already marshalled; calling it re-issues the same launch\n"
             "(same buffers, same stream) and returns the output.";
  t.tp_basicsize = sizeof(Prepared);
  t.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_GC | Py_TPFLAGS_HAVE_VECTORCALL;
  t.tp_vectorcall_offset = offsetof(Prepared, vectorcall);
  t.tp_call = PyVectorcall_Call;
  t.tp_dealloc = prepared_dealloc;
  t.tp_traverse = prepared_traverse;
  t.tp_clear = prepared_clear;
  t.tp_getset = prepared_getset;
  return t;
}();

// Issues f now, or wraps it.  Takes over the reference to `out`; `keep`: the other arguments, borrowed (or NULL).
template <class F>
PyObject* issue(const F& f, PyObject* out, bool prepare, std::initializer_list<PyObject*> keep) {
  if (!prepare) {
    hago_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f();
    Py_END_ALLOW_THREADS
    if (s != HAGO_OK) {
      Py_DECREF(out);
      check(s);
    }
    return out;
  }
  PyObject* k = PyTuple_New((Py_ssize_t)keep.size() + 1);
  Prepared* p = k ? PyObject_GC_New(Prepared, &PreparedType) : nullptr;
  if (!p) {
    Py_XDECREF(k);
    Py_DECREF(out);
    throw Raised{};
  }
  Py_ssize_t i = 0;
  auto hold = [&](PyObject* o) {
    Py_INCREF(o);
    PyTuple_SET_ITEM(k, i++, o);
  };
  for (PyObject* o : keep) hold(o ? o : Py_None);
  hold(out);  // (p->out may be set to something else)
  p->vectorcall = prepared_call;
  p->fn = new std::function<hago_status()>(f);
  p->keep = k;
  p->out = out;
  PyObject_GC_Track(p);
  return reinterpret_cast<PyObject*>(p);
}

// ---- the functions
void need_args(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return;
  PyErr_Format(PyExc_TypeError, "%zd arguments wanted, got %zd", want, n);
  throw Raised{};
}

struct Tensor3 {  // x[outer, channels, inner]
  const at::Tensor& t;
  int64_t outer, channels, inner;
};
Tensor3 tensor3(PyObject* o) {
  const at::Tensor& t = tensor(o);
  require(t.dim() == 3 && t.is_contiguous());
  return Tensor3{t, t.size(0), t.size(1), t.size(2)};
}

int32_t per_channel_of(PyObject* o, PyObject* scale) {
  return o == Py_None ? (tensor(scale).numel() > 1 ? 1 : 0) : (int32_t)as_converted_int(o);
}

struct Clip {
  int32_t lo, hi;
};
Clip clip_of(PyObject* lo, PyObject* hi, const hago_qtype& q, int32_t most_bits) {
  Clip c;
  check(L.hago_bit_range(q.bits < most_bits ? q.bits : most_bits, q.is_signed ? 1 : 0, &c.lo, &c.hi));
  if (lo != Py_None) c.lo = (int32_t)as_converted_int(lo);
  if (hi != Py_None) c.hi = (int32_t)as_converted_int(hi);
  return c;
}

// simquant, simquant_wrap: (x, scale, zero_point, q, clip_lo, clip_hi, per_channel, out, prepare)
template <class Fn>
PyObject* simquant_with(Fn fn, int32_t most_bits, PyObject* const* a, Py_ssize_t n) {
  need_args(n, 9);
  const Tensor3 x = tensor3(a[0]);
  const hago_qtype q = qtype(a[3]);
  const Clip c = clip_of(a[4], a[5], q, most_bits);
  const int32_t pc = per_channel_of(a[6], a[1]);
  const float* scale = static_cast<const float*>(pointer(a[1]));
  const int32_t* zp = static_cast<const int32_t*>(pointer(a[2]));
  PyObject* out = output(a[7], x.t.sizes(), x.t.scalar_type(), x.t);
  const float* src = static_cast<const float*>(x.t.data_ptr());
  float* dst = static_cast<float*>(pointer(out));
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return fn(src, dst, o, ch, in, scale, zp, pc, q, c.lo, c.hi, st); }, out, as_bool(a[8]), {a[0], a[1], a[2]});
}

PyObject* f_simquant(PyObject* const* a, Py_ssize_t n) { return simquant_with(L.hago_simquant, 64, a, n); }
PyObject* f_simquant_wrap(PyObject* const* a, Py_ssize_t n) { return simquant_with(L.hago_simquant_wrap, 25, a, n); }

// (x, scales, zero_points, q, clip_lo, clip_hi, per_channel, out, prepare)
PyObject* f_simquant_batched(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 9);
  const Tensor3 x = tensor3(a[0]);
  const at::Tensor &scales = tensor(a[1]), &zps = tensor(a[2]);
  require(scales.is_contiguous() && zps.is_contiguous());
  auto ints = [](PyObject* seq) {
    std::vector<int32_t> v;
    PyObject* f = PySequence_Fast(seq, "clip limits are sequences");
    if (!f) throw Raised{};
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(f); ++i) {
      try {
        v.push_back((int32_t)as_converted_int(PySequence_Fast_GET_ITEM(f, i)));
      } catch (...) {
        Py_DECREF(f);
        throw;
      }
    }
    Py_DECREF(f);
    return v;
  };
  const std::vector<int32_t> lo = ints(a[4]), hi = ints(a[5]);
  const int64_t nb = (int64_t)lo.size();
  require((int64_t)hi.size() == nb && scales.size(0) == nb && zps.size(0) == nb);
  const hago_qtype q = qtype(a[3]);
  const int32_t pc = as_bool(a[6]) ? 1 : 0;
  const int64_t shape[4] = {nb, x.outer, x.channels, x.inner};
  PyObject* out = output(a[7], at::IntArrayRef(shape, 4), at::kFloat, x.t);
  const float* src = static_cast<const float*>(x.t.data_ptr());
  float* dst = static_cast<float*>(pointer(out));
  const float* sp = static_cast<const float*>(scales.data_ptr());
  const int32_t* zp = static_cast<const int32_t*>(zps.data_ptr());
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  auto call = [=](const int32_t* l, const int32_t* h) {
    // (an empty list has no address of its own, and the library wants one only for nb > 0)
    return L.hago_simquant_batched(src, dst, o, ch, in, (int32_t)nb, sp, zp, pc, q, l, h, st);
  };
  if (as_bool(a[8])) return issue([call, lo, hi] { return call(lo.data(), hi.data()); }, out, true, {a[0], a[1], a[2]});
  return issue([&] { return call(lo.data(), hi.data()); }, out, false, {});
}

// (x, scale, zero_point, q, clip_lo, clip_hi, per_channel, out, prepare)
PyObject* f_quantize(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 9);
  const Tensor3 x = tensor3(a[0]);
  const hago_qtype q = qtype(a[3]);
  const Clip c = clip_of(a[4], a[5], q, 64);
  const int32_t pc = per_channel_of(a[6], a[1]);
  const float* scale = static_cast<const float*>(pointer(a[1]));
  const int32_t* zp = static_cast<const int32_t*>(pointer(a[2]));
  PyObject* out = output(a[7], x.t.sizes(), scalar_type(q.dtype), x.t);
  const float* src = static_cast<const float*>(x.t.data_ptr());
  void* dst = pointer(out);
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return L.hago_quantize(src, dst, o, ch, in, scale, zp, pc, q, c.lo, c.hi, st); }, out, as_bool(a[8]),
               {a[0], a[1], a[2]});
}

// (x, scale, zero_point, q, clip_lo, clip_hi, per_channel, out, out_codes, prepare)
PyObject* f_simquant_codes(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 10);
  const Tensor3 x = tensor3(a[0]);
  const hago_qtype q = qtype(a[3]);
  const Clip c = clip_of(a[4], a[5], q, 64);
  const int32_t pc = per_channel_of(a[6], a[1]);
  const float* scale = static_cast<const float*>(pointer(a[1]));
  const int32_t* zp = static_cast<const int32_t*>(pointer(a[2]));
  PyObject* y = output(a[7], x.t.sizes(), x.t.scalar_type(), x.t);
  PyObject* codes;
  try {
    codes = output(a[8], x.t.sizes(), scalar_type(q.dtype), x.t);
  } catch (...) {
    Py_DECREF(y);
    throw;
  }
  const float* src = static_cast<const float*>(x.t.data_ptr());
  float* dst = static_cast<float*>(pointer(y));
  void* dq = pointer(codes);
  PyObject* both = PyTuple_New(2);
  if (!both) throw Raised{};
  PyTuple_SET_ITEM(both, 0, y);
  PyTuple_SET_ITEM(both, 1, codes);
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return L.hago_simquant_codes(src, dst, dq, o, ch, in, scale, zp, pc, q, c.lo, c.hi, st); }, both,
               as_bool(a[9]), {a[0], a[1], a[2]});
}

// (codes, q, scale, zero_point, per_channel, out, prepare)
PyObject* f_dequantize(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 7);
  const Tensor3 x = tensor3(a[0]);
  const hago_qtype q = qtype(a[1]);
  const int32_t pc = per_channel_of(a[4], a[2]);
  const float* scale = static_cast<const float*>(pointer(a[2]));
  const int32_t* zp = static_cast<const int32_t*>(pointer(a[3]));
  PyObject* out = output(a[5], x.t.sizes(), at::kFloat, x.t);
  const void* src = x.t.data_ptr();
  float* dst = static_cast<float*>(pointer(out));
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return L.hago_dequantize(src, q, dst, o, ch, in, scale, zp, pc, st); }, out, as_bool(a[6]),
               {a[0], a[2], a[3]});
}

// (x, per_channel, out, prepare)
PyObject* f_absmax(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 4);
  const Tensor3 x = tensor3(a[0]);
  const int32_t pc = as_bool(a[1]) ? 1 : 0;
  const int64_t nthr = pc ? x.channels : 1;
  PyObject* out = output(a[2], at::IntArrayRef(&nthr, 1), at::kFloat, x.t);
  const float* src = static_cast<const float*>(x.t.data_ptr());
  float* dst = static_cast<float*>(pointer(out));
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return L.hago_absmax(src, o, ch, in, pc, dst, st); }, out, as_bool(a[3]), {a[0]});
}

// (acc, rq, out, prepare)
PyObject* f_requantize(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 4);
  const Tensor3 x = tensor3(a[0]);
  RequantTensors tensors;
  const MaybeRequant rq = requant(a[1], tensors);
  int code;
  switch (x.t.scalar_type()) {
    case at::kByte: code = HAGO_U8; break;
    case at::kChar: code = HAGO_I8; break;
    case at::kShort: code = HAGO_I16; break;
    case at::kInt: code = HAGO_I32; break;
    default: code = HAGO_F32;
  }
  PyObject* out = output(a[2], x.t.sizes(), scalar_type(rq.rq.out.dtype), x.t);
  const void* src = x.t.data_ptr();
  void* dst = pointer(out);
  const int64_t o = x.outer, ch = x.channels, in = x.inner;
  void* st = stream();
  return issue([=] { return L.hago_requantize(src, (hago_dtype)code, o, ch, in, rq.ptr(), dst, st); }, out, as_bool(a[3]),
               {a[0], tensors.mult.o, tensors.shift.o});
}

// (a, a_t, w, w_t, bias, acc_dtype, rq, flags, out, prepare)
PyObject* f_qdense(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 10);
  const at::Tensor &act = tensor(a[0]), &w = tensor(a[2]);
  require(act.dim() == 2 && w.dim() == 2 && act.is_contiguous() && w.is_contiguous());
  const int64_t M = act.size(0), K = act.size(1), N = w.size(0);
  require(w.size(1) == K);
  const hago_qtype at_ = qtype(a[1]), wt = qtype(a[3]);
  const int32_t* bias = static_cast<const int32_t*>(pointer(a[4]));
  const int64_t acc = as_int(a[5]);
  RequantTensors tensors;
  const MaybeRequant rq = requant(a[6], tensors);
  const uint32_t flags = (uint32_t)as_int(a[7]);
  const int64_t shape[2] = {M, N};
  PyObject* out = output(a[8], at::IntArrayRef(shape, 2), scalar_type(rq.present ? rq.rq.out.dtype : acc), act);
  const void *ap = act.data_ptr(), *wp = w.data_ptr();
  void* dst = pointer(out);
  void* st = stream();
  return issue([=] { return L.hago_qdense(ap, at_, wp, wt, bias, M, N, K, (hago_dtype)acc, rq.ptr(), dst, flags, st); }, out,
               as_bool(a[9]), {a[0], a[2], a[4], tensors.mult.o, tensors.shift.o});
}

void pair(PyObject* o, int32_t (&v)[2]) {
  for (Py_ssize_t i = 0; i < 2; ++i) {
    PyObject* e = PySequence_GetItem(o, i);
    if (!e) throw Raised{};
    const long long r = PyLong_AsLongLong(e);
    Py_DECREF(e);
    if (r == -1 && PyErr_Occurred()) throw Raised{};
    v[i] = (int32_t)r;
  }
}

// (a, a_t, w, w_t, bias, layout, stride, pad, groups, acc_dtype, rq, flags, out, prepare, workspace, static_scratch)
PyObject* f_qconv2d(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 16);
  const at::Tensor &act = tensor(a[0]), &w = tensor(a[2]);
  require(act.dim() == 4 && w.dim() == 4 && act.is_contiguous() && w.is_contiguous());
  const hago_qtype at_ = qtype(a[1]), wt = qtype(a[3]);
  const int32_t* bias = static_cast<const int32_t*>(pointer(a[4]));
  const int64_t layout = as_int(a[5]);
  const bool nchw = layout == HAGO_NCHW;
  const int64_t B = act.size(0), C = act.size(nchw ? 1 : 3), H = act.size(nchw ? 2 : 1), W = act.size(nchw ? 3 : 2);
  const int64_t O = w.size(0), KH = w.size(nchw ? 2 : 1), KW = w.size(nchw ? 3 : 2);
  int32_t stride[2], pad[2];
  pair(a[6], stride);
  pair(a[7], pad);
  const int32_t groups = (int32_t)as_int(a[8]);
  const int64_t acc = as_int(a[9]);
  RequantTensors tensors;
  const MaybeRequant rq = requant(a[10], tensors);
  const uint32_t flags = (uint32_t)as_int(a[11]);
  auto extent = [&](int64_t size, int64_t k, int i) -> int64_t {
    if (stride[i] == 0) {
      PyErr_SetString(PyExc_ZeroDivisionError, "stride 0");
      throw Raised{};
    }
    const int64_t num = size + 2 * (int64_t)pad[i] - k, s = stride[i];
    int64_t q = num / s;
    if (num % s != 0 && (num < 0) != (s < 0)) --q;  // floor
    return q + 1 > 0 ? q + 1 : 0;
  };
  const int64_t OH = extent(H, KH, 0), OW = extent(W, KW, 1);
  const int64_t cf[4] = {B, O, OH, OW}, cl[4] = {B, OH, OW, O};
  PyObject* out = output(a[12], at::IntArrayRef(nchw ? cf : cl, 4), scalar_type(rq.present ? rq.rq.out.dtype : acc), act);
  const void *ap = act.data_ptr(), *wp = w.data_ptr();
  void* dst = pointer(out);
  const bool prepare = as_bool(a[13]);
  void* st = stream();
  const int32_t kh = (int32_t)KH, kw = (int32_t)KW, sh = stride[0], sw = stride[1], ph = pad[0], pw = pad[1];
  if (a[14] != Py_None) {
    const at::Tensor& wst = tensor(a[14]);
    const int64_t bytes = wst.numel() * (int64_t)wst.element_size();
    void* ws = wst.numel() ? wst.data_ptr() : nullptr;
    return issue([=] { return L.hago_qconv2d_ws(ap, at_, wp, wt, bias, (hago_layout)layout, B, C, H, W, O, kh, kw, sh, sw, ph, pw,
                                                groups, (hago_dtype)acc, rq.ptr(), dst, ws, bytes, flags, st); },
                 out, prepare, {a[0], a[2], a[4], tensors.mult.o, tensors.shift.o, a[14]});
  }
  auto fn = as_bool(a[15]) ? L.hago_qconv2d_static : L.hago_qconv2d;
  return issue([=] { return fn(ap, at_, wp, wt, bias, (hago_layout)layout, B, C, H, W, O, kh, kw, sh, sw, ph, pw, groups,
                               (hago_dtype)acc, rq.ptr(), dst, flags, st); },
               out, prepare, {a[0], a[2], a[4], tensors.mult.o, tensors.shift.o});
}

// ---- microscaled operators
// The tensors of a call lie on the device that it is issued on (the library takes addresses of that one only).
void on_current_device(std::initializer_list<PyObject*> tensors) {
  for (PyObject* o : tensors)
    if (o && o != Py_None) require(tensor(o).is_cuda() && tensor(o).get_device() == c10::hip::current_device());
}
hago_dtype real_type(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return HAGO_F32;
    case at::kBFloat16: return HAGO_BF16;
    case at::kHalf: return HAGO_F16;
    default: PyErr_SetString(PyExc_TypeError, "a float32, bfloat16 or float16 tensor is needed"); throw Raised{};
  }
}
// A tensor that the caller gave, of this shape and type; None is left alone.
void given(PyObject* o, at::IntArrayRef shape, at::ScalarType type) {
  if (o == Py_None) return;
  const at::Tensor& t = tensor(o);
  require(t.sizes() == shape && t.scalar_type() == type && t.is_contiguous());
}
int64_t mx_padded(int64_t cols) { return (cols + 127) / 128 * 128; }
int64_t mx_code_bytes(int64_t cols, int64_t format) { return format == HAGO_MX_FP4 ? mx_padded(cols) / 2 : mx_padded(cols); }
void require_format(int64_t f) { require(f == HAGO_MX_FP4 || f == HAGO_MX_FP8); }

struct MxRows {  // x[rows, columns], rows at any distance
  hago_dtype type;
  at::ScalarType scalar;
  int64_t rows, columns, stride;
  const void* src;
};
MxRows mx_rows(PyObject* o) {
  const at::Tensor& t = tensor(o);
  require(t.dim() == 2);
  const int64_t rows = t.size(0), columns = t.size(1);
  require(t.numel() == 0 || ((columns <= 1 || t.stride(1) == 1) && (rows <= 1 || t.stride(0) >= columns)));
  return {real_type(t), t.scalar_type(), rows, columns, rows > 1 && columns ? t.stride(0) : columns, t.data_ptr()};
}

PyObject* g_mx = nullptr;  // the binding's class MX(codes, scales, fmt, cols)

// What such an operator returns: an MX, and behind it the residual and the values where they are asked for (a tuple then).
// `out` is None or an MX whose tensors are taken; residual and values are True, a tensor, or False (values: or None).
struct MxResults {
  PyObject* all = nullptr;
  Ref code_tensor, scale_tensor;  // (the MX can be given others while a call is under way or prepared)
  void *codes = nullptr, *scales = nullptr, *residual = nullptr, *values = nullptr;
  MxResults(const at::Tensor& like, const MxRows& x, int64_t cols, PyObject* format, PyObject* out, PyObject* residual, PyObject* values);
};
MxResults::MxResults(const at::Tensor& like, const MxRows& x, int64_t cols, PyObject* format, PyObject* out, PyObject* keep_residual, PyObject* keep_values) {
  static PyObject *n_codes = intern("codes"), *n_scales = intern("scales"), *n_fmt = intern("fmt"), *n_cols = intern("cols");
  const int64_t f = as_int(format);
  require_format(f);
  const int64_t code_shape[2] = {x.rows, mx_code_bytes(cols, f)}, scale_shape[2] = {x.rows, mx_padded(cols) / 32}, shape[2] = {x.rows, cols};
  const bool has_residual = keep_residual != Py_False, has_values = keep_values != Py_None && keep_values != Py_False;
  Ref mx, res, val, &c = code_tensor, &s = scale_tensor;
  if (out != Py_None) {
    require(attr_int(out, n_fmt) == f && attr_int(out, n_cols) == cols);
    c.o = PyObject_GetAttr(out, n_codes);
    s.o = c.o ? PyObject_GetAttr(out, n_scales) : nullptr;
    if (!s.o) throw Raised{};
    tensor(c.o), tensor(s.o);
    given(c.o, at::IntArrayRef(code_shape, 2), at::kByte);
    given(s.o, at::IntArrayRef(scale_shape, 2), at::kByte);
    on_current_device({c.o, s.o});
    Py_INCREF(out);
    mx.o = out;
  }
  auto optional = [&](PyObject* o, bool has, Ref& r) {
    if (!has) return;
    if (o != Py_True) given(o, at::IntArrayRef(shape, 2), x.scalar), on_current_device({o});
    r.o = output(o == Py_True ? Py_None : o, at::IntArrayRef(shape, 2), x.scalar, like);
  };
  optional(keep_residual, has_residual, res);
  optional(keep_values, has_values, val);
  if (!mx.o) {
    c.o = output(Py_None, at::IntArrayRef(code_shape, 2), at::kByte, like);
    s.o = output(Py_None, at::IntArrayRef(scale_shape, 2), at::kByte, like);
    Ref n;
    n.o = PyLong_FromLongLong(cols);
    PyObject* args[4] = {c.o, s.o, format, n.o};
    mx.o = n.o ? PyObject_Vectorcall(g_mx, args, 4, nullptr) : nullptr;
    if (!mx.o) throw Raised{};
  }
  codes = tensor(c.o).data_ptr(), scales = tensor(s.o).data_ptr();
  if (has_residual) residual = tensor(res.o).data_ptr();
  if (has_values) values = tensor(val.o).data_ptr();
  auto take = [](Ref& v) {
    PyObject* o = v.o;
    v.o = nullptr;
    return o;
  };
  if (!has_residual && !has_values) {
    all = take(mx);
    return;
  }
  all = PyTuple_New(1 + has_residual + has_values);
  if (!all) throw Raised{};
  Py_ssize_t i = 0;
  PyTuple_SET_ITEM(all, i++, take(mx));
  if (has_residual) PyTuple_SET_ITEM(all, i++, take(res));
  if (has_values) PyTuple_SET_ITEM(all, i++, take(val));
}

// mx_quantize, mx_silu_mul: (x, format, values, out, prepare)
template <class Fn>
PyObject* mx_quantize_with(Fn fn, bool gated, PyObject* const* a, Py_ssize_t n) {
  need_args(n, 5);
  const MxRows x = mx_rows(a[0]);
  require(!gated || x.columns % 2 == 0);
  const int64_t cols = gated ? x.columns / 2 : x.columns, format = as_int(a[1]);
  on_current_device({a[0]});
  const bool prepare = as_bool(a[4]);
  void* st = stream();
  const MxResults r(tensor(a[0]), x, cols, a[1], a[3], Py_False, a[2]);
  return issue([=, codes = r.codes, scales = r.scales, values = r.values] {
                 return fn(x.src, x.type, x.rows, cols, x.stride, (hago_mx_format)format, codes, scales, values, st);
               },
               r.all, prepare, {a[0], r.code_tensor.o, r.scale_tensor.o});
}
PyObject* f_mx_quantize(PyObject* const* a, Py_ssize_t n) { return mx_quantize_with(L.hago_mx_quantize, false, a, n); }
PyObject* f_mx_silu_mul(PyObject* const* a, Py_ssize_t n) { return mx_quantize_with(L.hago_mx_silu_mul, true, a, n); }

// (x, gamma, residual, eps, format, values, out, out_residual, prepare); out_residual None: a new tensor where there is a residual
PyObject* f_mx_rmsnorm(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 9);
  const MxRows x = mx_rows(a[0]);
  const int64_t shape[2] = {x.rows, x.columns};
  given(a[1], at::IntArrayRef(&x.columns, 1), x.scalar);
  given(a[2], at::IntArrayRef(shape, 2), x.scalar);
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw Raised{};
  const int64_t format = as_int(a[4]);
  on_current_device({a[0], a[1], a[2]});
  const void *gamma = pointer(a[1]), *res = pointer(a[2]);
  const bool prepare = as_bool(a[8]);
  PyObject* keep = a[7] != Py_None ? a[7] : a[2] != Py_None ? Py_True : Py_False;
  void* st = stream();
  const MxResults r(tensor(a[0]), x, x.columns, a[4], a[6], keep, a[5]);
  return issue([=, residual = r.residual, codes = r.codes, scales = r.scales, values = r.values] {
                 return L.hago_mx_rmsnorm(x.src, res, gamma, x.type, x.rows, x.columns, x.stride, (float)eps, (hago_mx_format)format, residual, codes, scales,
                                          values, st);
               },
               r.all, prepare, {a[0], a[1], a[2], r.code_tensor.o, r.scale_tensor.o});
}

// An MX: its tensors (references of its own) and what they say.
struct MxOperand {
  Ref codes, scales;
  int64_t format, cols, rows, groups;
  const void* code_ptr() const { return tensor(codes.o).data_ptr(); }
  const void* scale_ptr() const { return tensor(scales.o).data_ptr(); }
  // [rows, cols], or with dims == 3 [groups, rows, cols]
  MxOperand(PyObject* mx, int64_t dims) {
    static PyObject *n_codes = intern("codes"), *n_scales = intern("scales"), *n_fmt = intern("fmt"), *n_cols = intern("cols");
    format = attr_int(mx, n_fmt), cols = attr_int(mx, n_cols);
    codes.o = PyObject_GetAttr(mx, n_codes);
    scales.o = codes.o ? PyObject_GetAttr(mx, n_scales) : nullptr;
    if (!scales.o) throw Raised{};
    require_format(format);
    require(cols >= 0);
    const at::Tensor &c = tensor(codes.o), &s = tensor(scales.o);
    require(c.dim() == dims && s.dim() == dims && c.scalar_type() == at::kByte && s.scalar_type() == at::kByte && c.is_contiguous() && s.is_contiguous());
    require(c.size(dims - 1) == mx_code_bytes(cols, format) && s.size(dims - 1) == mx_padded(cols) / 32 && c.size(dims - 2) == s.size(dims - 2));
    require(dims == 2 || c.size(0) == s.size(0));
    rows = c.size(dims - 2), groups = dims == 3 ? c.size(0) : 1;
  }
};

// (a, w, bias, out_dtype, out, prepare)
PyObject* f_mx_dense(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 6);
  const MxOperand act(a[0], 2), w(a[1], 2);
  require(w.format == HAGO_MX_FP4 && w.cols == act.cols);
  const int64_t M = act.rows, N = w.rows, K = act.cols, shape[2] = {M, N}, format = act.format, type = as_int(a[3]);
  given(a[2], at::IntArrayRef(&N, 1), at::kFloat);
  given(a[4], at::IntArrayRef(shape, 2), product_type(type));
  on_current_device({act.codes.o, act.scales.o, w.codes.o, w.scales.o, a[2], a[4]});
  const float* bias = static_cast<const float*>(pointer(a[2]));
  const bool prepare = as_bool(a[5]);
  const void *ac = act.code_ptr(), *as = act.scale_ptr(), *wc = w.code_ptr(), *ws = w.scale_ptr();
  void* st = stream();
  PyObject* out = output(a[4], at::IntArrayRef(shape, 2), product_type(type), tensor(act.codes.o));
  void* dst = pointer(out);
  return issue([=] { return L.hago_mx_dense(ac, as, (hago_mx_format)format, wc, ws, bias, M, N, K, (hago_dtype)type, dst, st); }, out, prepare,
               {act.codes.o, act.scales.o, w.codes.o, w.scales.o, a[2]});
}

// (a, w, offsets, rows, bias, out_dtype, out, prepare)
PyObject* f_mx_dense_grouped(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 8);
  const MxOperand act(a[0], 2), w(a[1], 3);
  require(w.format == HAGO_MX_FP4 && w.cols == act.cols);
  const int64_t E = w.groups, N = w.rows, K = act.cols, entries = E + 1, bias_shape[2] = {E, N}, format = act.format, type = as_int(a[5]);
  tensor(a[2]);
  given(a[2], at::IntArrayRef(&entries, 1), at::kInt);
  int64_t T = act.rows;
  if (a[3] != Py_None) {
    require(tensor(a[3]).dim() == 1);
    T = tensor(a[3]).size(0);
    given(a[3], at::IntArrayRef(&T, 1), at::kInt);
  }
  const int64_t shape[2] = {T, N};
  given(a[4], at::IntArrayRef(bias_shape, 2), at::kFloat);
  given(a[6], at::IntArrayRef(shape, 2), product_type(type));
  on_current_device({act.codes.o, act.scales.o, w.codes.o, w.scales.o, a[2], a[3], a[4], a[6]});
  const int32_t *offsets = static_cast<const int32_t*>(pointer(a[2])), *index = static_cast<const int32_t*>(pointer(a[3]));
  const float* bias = static_cast<const float*>(pointer(a[4]));
  const bool prepare = as_bool(a[7]);
  const void *ac = act.code_ptr(), *as = act.scale_ptr(), *wc = w.code_ptr(), *ws = w.scale_ptr();
  const int64_t a_rows = act.rows;
  void* st = stream();
  PyObject* out = output(a[6], at::IntArrayRef(shape, 2), product_type(type), tensor(act.codes.o));
  void* dst = pointer(out);
  return issue([=] { return L.hago_mx_dense_grouped(ac, as, (hago_mx_format)format, a_rows, index, wc, ws, bias, offsets, T, E, N, K, (hago_dtype)type, dst, st); },
               out, prepare, {act.codes.o, act.scales.o, w.codes.o, w.scales.o, a[2], a[3], a[4]});
}

// ---- rotary positions, and the operators around a paged cache
struct Heads {  // x[T, heads, dim], rows and heads at any distance
  hago_dtype type;
  at::ScalarType scalar;
  int64_t T, heads, dim, row, head;
  const void* src;
};
Heads heads_of(PyObject* o) {
  const at::Tensor& t = tensor(o);
  require(t.dim() == 3);
  const int64_t T = t.size(0), heads = t.size(1), dim = t.size(2);
  const bool any = t.numel() != 0;
  require(!any || dim <= 1 || t.stride(2) == 1);
  return {real_type(t), t.scalar_type(), T, heads, dim, any && T > 1 ? t.stride(0) : heads * dim, any && heads > 1 ? t.stride(1) : dim, t.data_ptr()};
}

// (x, positions, frequencies, axes, interleaved, out, prepare)
PyObject* f_rope(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 7);
  const Heads x = heads_of(a[0]);
  const at::Tensor &positions = tensor(a[1]), &frequencies = tensor(a[2]);
  const int64_t pairs = frequencies.numel(), axes = positions.dim() == 2 ? positions.size(0) : 1;
  require(positions.scalar_type() == at::kInt && positions.is_contiguous() && (positions.dim() == 1 || positions.dim() == 2) &&
          positions.size(positions.dim() - 1) == x.T && axes >= 1);
  given(a[2], at::IntArrayRef(&pairs, 1), at::kFloat);
  given(a[3], at::IntArrayRef(&pairs, 1), at::kInt);
  require(2 * pairs <= x.dim);
  const bool neighbours = as_bool(a[4]), prepare = as_bool(a[6]);
  on_current_device({a[0], a[1], a[2], a[3], a[5]});
  if (a[5] != Py_None) {
    const Heads o = heads_of(a[5]);
    require(o.scalar == x.scalar && o.T == x.T && o.heads == x.heads && o.dim == x.dim);
  }
  const int32_t *pos = positions.data_ptr<int32_t>(), *axis = static_cast<const int32_t*>(pointer(a[3]));
  const float* freq = frequencies.data_ptr<float>();
  void* st = stream();
  const int64_t shape[3] = {x.T, x.heads, x.dim};
  PyObject* out = output(a[5], at::IntArrayRef(shape, 3), x.scalar, tensor(a[0]));
  const Heads y = heads_of(out);
  void* dst = const_cast<void*>(y.src);
  return issue([=] {
                 return L.hago_rope(x.src, x.type, x.T, x.heads, x.dim, x.row, x.head, pos, axes, freq, axis, pairs, neighbours ? HAGO_ROPE_NEIGHBOURS : HAGO_ROPE_HALVES,
                                    dst, y.row, y.head, st);
               },
               out, prepare, {a[0], a[1], a[2], a[3]});
}

// An MXCache and the sequences of a call.
struct MxCacheOperand {
  Ref t[4];  // codes and scales of keys, of values
  hago_mx_cache cache;
  hago_mx_sequences sequences;
  PyObject *table, *lengths, *offsets;
  MxCacheOperand(PyObject* o, PyObject* table, PyObject* lengths, PyObject* offsets) : table(table), lengths(lengths), offsets(offsets) {
    static PyObject* const names[4] = {intern("k_codes"), intern("k_scales"), intern("v_codes"), intern("v_scales")};
    static PyObject *k_fmt = intern("k_fmt"), *v_fmt = intern("v_fmt"), *n_dim = intern("dim");
    const int64_t formats[2] = {attr_int(o, k_fmt), attr_int(o, v_fmt)}, dim = attr_int(o, n_dim), blocks = (dim + 31) / 32;
    require_format(formats[0]), require_format(formats[1]);
    require(dim >= 0);
    for (int i = 0; i < 4; ++i) {
      t[i].o = PyObject_GetAttr(o, names[i]);
      if (!t[i].o) throw Raised{};
      const at::Tensor& x = tensor(t[i].o);
      require(x.dim() == 4 && x.scalar_type() == at::kByte && x.is_contiguous());
      require(x.sizes().slice(0, 3) == tensor(t[0].o).sizes().slice(0, 3));
      require(x.size(3) == (i % 2 ? blocks : blocks * (formats[i / 2] == HAGO_MX_FP4 ? 16 : 32)));
    }
    const at::Tensor &x = tensor(t[0].o), &b = tensor(table);
    cache = {x.data_ptr(), tensor(t[1].o).data_ptr(), tensor(t[2].o).data_ptr(), tensor(t[3].o).data_ptr(), (hago_mx_format)formats[0], (hago_mx_format)formats[1],
             x.size(0), x.size(1), x.size(2), dim};
    require(b.dim() == 2 && b.scalar_type() == at::kInt);
    const int64_t seqs = b.size(0), cols = b.size(1), ends = seqs + 1;
    require(b.numel() == 0 || ((cols <= 1 || b.stride(1) == 1) && (seqs <= 1 || b.stride(0) >= cols)));
    tensor(lengths), tensor(offsets);
    given(lengths, at::IntArrayRef(&seqs, 1), at::kInt);
    given(offsets, at::IntArrayRef(&ends, 1), at::kInt);
    sequences = {static_cast<const int32_t*>(b.data_ptr()), tensor(lengths).data_ptr<int32_t>(), tensor(offsets).data_ptr<int32_t>(), seqs, cols,
                 seqs > 1 && cols ? b.stride(0) : cols};
  }
  void on_device(std::initializer_list<PyObject*> others) const {
    on_current_device({t[0].o, t[1].o, t[2].o, t[3].o, table, lengths, offsets});
    on_current_device(others);
  }
};
// A new reference to (a, b), whose references it takes over.
PyObject* pair_of(Ref& a, Ref& b) {
  PyObject* both = PyTuple_New(2);
  if (!both) throw Raised{};
  PyTuple_SET_ITEM(both, 0, a.o);
  PyTuple_SET_ITEM(both, 1, b.o);
  a.o = b.o = nullptr;
  return both;
}

// (cache, k, v, table, lengths, offsets, values, prepare)
PyObject* f_mx_cache_write(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 8);
  const MxCacheOperand m(a[0], a[3], a[4], a[5]);
  const Heads k = heads_of(a[1]), v = heads_of(a[2]);
  require(k.scalar == v.scalar && k.T == v.T && k.heads == m.cache.kv_heads && v.heads == k.heads && k.dim == m.cache.dim && v.dim == k.dim);
  m.on_device({a[1], a[2]});
  const bool values = as_bool(a[6]), prepare = as_bool(a[7]);
  void *st = stream(), *k_values = nullptr, *v_values = nullptr;
  PyObject* out = a[0];
  if (values) {
    const int64_t shape[3] = {k.T, k.heads, k.dim};
    Ref kv, vv;
    kv.o = output(Py_None, at::IntArrayRef(shape, 3), k.scalar, tensor(a[1]));
    vv.o = output(Py_None, at::IntArrayRef(shape, 3), k.scalar, tensor(a[1]));
    k_values = pointer(kv.o), v_values = pointer(vv.o);
    out = pair_of(kv, vv);
  } else {
    Py_INCREF(out);
  }
  return issue([=, cache = m.cache, sequences = m.sequences] {
                 return L.hago_mx_cache_write(&cache, &sequences, k.src, k.row, k.head, v.src, v.row, v.head, k.type, k.T, k_values, v_values, st);
               },
               out, prepare, {m.t[0].o, m.t[1].o, m.t[2].o, m.t[3].o, a[1], a[2], a[3], a[4], a[5]});
}

// (cache, table, lengths, offsets, rows, out_dtype, out, prepare)
PyObject* f_mx_cache_read(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 8);
  const MxCacheOperand m(a[0], a[1], a[2], a[3]);
  const int64_t T = as_int(a[4]), type = as_int(a[5]), shape[3] = {T, m.cache.kv_heads, m.cache.dim};
  const at::ScalarType scalar = product_type(type);
  require(T >= 0);
  const bool prepare = as_bool(a[7]);
  PyObject *kg = Py_None, *vg = Py_None;
  if (a[6] != Py_None) {
    require(PyTuple_Check(a[6]) && PyTuple_GET_SIZE(a[6]) == 2);
    kg = PyTuple_GET_ITEM(a[6], 0), vg = PyTuple_GET_ITEM(a[6], 1);
    tensor(kg), tensor(vg);
    given(kg, at::IntArrayRef(shape, 3), scalar);
    given(vg, at::IntArrayRef(shape, 3), scalar);
  }
  m.on_device({kg, vg});
  void* st = stream();
  Ref k, v;
  k.o = output(kg, at::IntArrayRef(shape, 3), scalar, tensor(m.t[0].o));
  v.o = output(vg, at::IntArrayRef(shape, 3), scalar, tensor(m.t[0].o));
  void *kp = pointer(k.o), *vp = pointer(v.o);
  return issue([=, cache = m.cache, sequences = m.sequences] { return L.hago_mx_cache_read(&cache, &sequences, (hago_dtype)type, T, kp, vp, st); }, pair_of(k, v),
               prepare, {m.t[0].o, m.t[1].o, m.t[2].o, m.t[3].o, a[1], a[2], a[3]});
}

// (q, cache, table, lengths, offsets, scale, causal, window, lse, out, workspace, prepare)
PyObject* f_mx_attention(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 12);
  const MxCacheOperand m(a[1], a[2], a[3], a[4]);
  const Heads q = heads_of(a[0]);
  require(q.dim == m.cache.dim && (m.cache.kv_heads ? q.heads % m.cache.kv_heads == 0 : q.heads == 0));
  double scale = q.dim ? 1.0 / std::sqrt((double)q.dim) : 1.0;
  if (a[5] != Py_None) {
    scale = PyFloat_AsDouble(a[5]);
    if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
  }
  const bool causal = as_bool(a[6]), prepare = as_bool(a[11]);
  const int64_t window = as_int(a[7]), shape[3] = {q.T, q.heads, q.dim};
  const bool has_lse = a[8] != Py_None && a[8] != Py_False;
  if (has_lse && a[8] != Py_True) tensor(a[8]), given(a[8], at::IntArrayRef(shape, 2), at::kFloat), on_current_device({a[8]});
  given(a[9], at::IntArrayRef(shape, 3), q.scalar);
  m.on_device({a[0], a[9], a[10]});
  int64_t bytes = L.hago_mx_attention_workspace_bytes(q.T, m.sequences.seqs, q.heads, m.cache.kv_heads, q.dim);
  if (a[10] != Py_None) {
    const at::Tensor& w = tensor(a[10]);
    require(w.scalar_type() == at::kByte && w.is_contiguous() && w.numel() >= bytes);
  }
  void* st = stream();
  Ref out, lse, workspace;
  out.o = output(a[9], at::IntArrayRef(shape, 3), q.scalar, tensor(a[0]));
  if (has_lse) lse.o = output(a[8] == Py_True ? Py_None : a[8], at::IntArrayRef(shape, 2), at::kFloat, tensor(a[0]));
  const int64_t room = bytes < 0 ? 0 : bytes;  // (the call says what is wrong)
  workspace.o = output(a[10], at::IntArrayRef(&room, 1), at::kByte, tensor(a[0]));
  void *dst = pointer(out.o), *w = pointer(workspace.o);
  float* sums = has_lse ? static_cast<float*>(pointer(lse.o)) : nullptr;
  bytes = tensor(workspace.o).numel();
  PyObject* all;
  if (has_lse) {
    all = pair_of(out, lse);
  } else {
    all = out.o;
    out.o = nullptr;
  }
  return issue([=, cache = m.cache, sequences = m.sequences] {
                 return L.hago_mx_attention(&cache, &sequences, q.src, q.type, q.T, q.heads, q.row, q.head, (float)scale, causal, window, dst, sums, w, bytes, st);
               },
               all, prepare, {m.t[0].o, m.t[1].o, m.t[2].o, m.t[3].o, a[0], a[2], a[3], a[4], workspace.o});
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    return F(args, n);
  } catch (Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// bind({name: address}, check, MX)
PyObject* f_bind(PyObject* const* a, Py_ssize_t n) {
  need_args(n, 3);
  Library lib;
#define X(name)                                                        \
  {                                                                    \
    PyObject* v = PyMapping_GetItemString(a[0], #name);                \
    if (!v) throw Raised{};                                            \
    void* p = PyLong_AsVoidPtr(v);                                     \
    Py_DECREF(v);                                                      \
    if (!p && PyErr_Occurred()) throw Raised{};                        \
    lib.name = reinterpret_cast<decltype(&::name)>(p);                 \
  }
  HAGO_ENTRIES(X)
#undef X
  L = lib;
  Py_INCREF(a[1]);
  Py_XSETREF(g_check, a[1]);
  Py_INCREF(a[2]);
  Py_XSETREF(g_mx, a[2]);
  Py_RETURN_NONE;
}

// entries(): the names bind() wants
PyObject* f_entries(PyObject* const*, Py_ssize_t n) {
  need_args(n, 0);
  static const char* const names[] = {
#define X(name) #name,
      HAGO_ENTRIES(X)
#undef X
  };
  const Py_ssize_t count = (Py_ssize_t)(sizeof(names) / sizeof(names[0]));
  PyObject* t = PyTuple_New(count);
  if (!t) throw Raised{};
  for (Py_ssize_t i = 0; i < count; ++i) PyTuple_SET_ITEM(t, i, PyUnicode_FromString(names[i]));
  return t;
}

#define HAGO_METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<f_##name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HAGO_METHOD(bind), HAGO_METHOD(entries), HAGO_METHOD(simquant), HAGO_METHOD(simquant_wrap),
                         HAGO_METHOD(simquant_batched), HAGO_METHOD(quantize), HAGO_METHOD(simquant_codes),
                         HAGO_METHOD(dequantize), HAGO_METHOD(absmax), HAGO_METHOD(requantize), HAGO_METHOD(qdense),
                         HAGO_METHOD(qconv2d), HAGO_METHOD(mx_quantize), HAGO_METHOD(mx_silu_mul), HAGO_METHOD(mx_rmsnorm),
                         HAGO_METHOD(mx_dense), HAGO_METHOD(mx_dense_grouped), HAGO_METHOD(rope),
                         HAGO_METHOD(mx_cache_write), HAGO_METHOD(mx_cache_read), HAGO_METHOD(mx_attention), {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Native marshalling of the libhago binding.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  if (PyType_Ready(&PreparedType) < 0) return nullptr;
  PyObject* m = PyModule_Create(&module);
  if (!m) return nullptr;
  Py_INCREF(&PreparedType);
  if (PyModule_AddObject(m, "Prepared", reinterpret_cast<PyObject*>(&PreparedType)) < 0) return nullptr;
  return m;
}
