// The two calls a serving program makes per layer and generated token, decode attention and the decode step, from Python
// without ctypes: arguments are read from the tensors and the cache object, outputs allocated, the C ABI called.  Nothing
// is kept from one call for the next.  Through ctypes a step over a short context took longer on the host than on the GPU
// (a descriptor of 14 fields, two allocations at 1.4 us, 18 converted arguments); one sequence of 640 tokens, 32 heads:
// 11.1 -> 6.8 us a step, which is its time on the GPU.
//   The calls for chunks likewise (below), with their checks of types, shapes and devices.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <cstring>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/akvq.h"

namespace {

constexpr int64_t kHeadDim = 128;

// Attribute names of the cache object, made once.
struct Names {
  PyObject *B, *Hkv, *G, *T_cap, *S_cap, *T_len, *k_codes, *v_codes, *k_meta, *v_meta, *k_sal, *v_sal, *sal_idx, *sal_cnt,
      *fine_mask, *W, *k_win, *v_win, *workspace, *decode, *struct_, *window_struct,
      *page_rows, *n_pages, *max_pages, *max_len, *table, *seq_len, *paged_struct, *bits;
} names;
// What the package's own cache class describes itself with, and the types of the descriptions (plain_cache).
struct Plain {
  PyObject *struct_ = nullptr, *window_struct = nullptr, *cache_type = nullptr, *window_type = nullptr;
} plain;

struct Held {  // an owned reference
  PyObject *p = nullptr;
  Held() = default;
  explicit Held(PyObject *q) : p(q) {}
  Held(const Held &) = delete;
  Held &operator=(const Held &) = delete;
  ~Held() { Py_XDECREF(p); }
};
struct Failed {};  // a Python error is set

[[noreturn]] void refuse(const char *why) {
  PyErr_SetString(PyExc_AssertionError, why);
  throw Failed();
}
#define REQUIRE(cond) do { if (!(cond)) refuse(#cond); } while (0)

int64_t int_attr(PyObject *o, PyObject *name) {
  Held v(PyObject_GetAttr(o, name));
  if (!v.p) throw Failed();
  const long long x = PyLong_AsLongLong(v.p);
  if (x == -1 && PyErr_Occurred()) throw Failed();
  return x;
}
const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor is expected");
    throw Failed();
  }
  return THPVariable_Unpack(o);
}
// device pointer of a tensor attribute (null for None where that is allowed); the object keeps the tensor
void *ptr_attr(PyObject *o, PyObject *name, bool optional = false) {
  Held v(PyObject_GetAttr(o, name));
  if (!v.p) throw Failed();
  if (optional && v.p == Py_None) return nullptr;
  return tensor(v.p).data_ptr();
}
// A cache whose method `name` is not the package's own (a derived class, a method put on the object) is asked by that method;
// true: its description is in `out`, which `held` keeps, or it has none.  Otherwise the attributes are read, which say what the
// own method would say without making the description in Python (3 us).
template <typename T>
bool described(PyObject *cache, PyObject *name, PyObject *own, PyObject *type, Held &held, T &out) {
  Held method(PyObject_GetAttr(cache, name));
  if (!method.p) {  // nothing to ask
    if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw Failed();
    PyErr_Clear();
    return false;
  }
  if (PyMethod_Check(method.p) && PyMethod_GET_FUNCTION(method.p) == own) return false;
  held.p = PyObject_CallNoArgs(method.p);
  if (!held.p) throw Failed();
  if (held.p == Py_None) return true;
  const int is = type ? PyObject_IsInstance(held.p, type) : 0;
  if (is < 0) throw Failed();
  Py_buffer view;
  if (is == 0 || PyObject_GetBuffer(held.p, &view, PyBUF_SIMPLE) != 0) {
    PyErr_Format(PyExc_TypeError, "%U() of the cache did not return a descriptor", name);
    throw Failed();
  }
  const bool fits = view.len == (Py_ssize_t)sizeof(T);
  if (fits) std::memcpy(&out, view.buf, sizeof(T));
  PyBuffer_Release(&view);
  if (!fits) {
    PyErr_Format(PyExc_TypeError, "%U() of the cache returned a descriptor of another size", name);
    throw Failed();
  }
  return true;
}
double number(PyObject *o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Failed();
  return x;
}
long integer(PyObject *o) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) throw Failed();
  return x;
}

struct Call {
  akvq_cache cache;
  akvq_window win;
  akvq_rope rope;
  const akvq_window *win_p = nullptr;
  const akvq_rope *rope_p = nullptr;
  Held rope_pair, cache_held, win_held;  // keep what the pointers come from
  uint32_t *fine_mask = nullptr;
  int Hq = 0, n_split = 0;
  uint32_t flags = 0;
  float sm_scale = 0.0f;
  const void *q = nullptr;
  at::Tensor out, lse, ws_tensor;
  void *ws = nullptr;
  size_t ws_bytes = 0;
  void *stream = nullptr;
};

// What both calls share.  more_rows: rows the call itself adds to the cache; check_out: out is looked at.
void gather(Call &c, PyObject *cache, PyObject *q_obj, PyObject *scale, PyObject *n_split, PyObject *flags, PyObject *out,
            PyObject *lse, PyObject *rope, int64_t more_rows, bool check_out) {
  akvq_cache &k = c.cache;
  const int32_t cache_B = (int32_t)int_attr(cache, names.B), Hkv = (int32_t)int_attr(cache, names.Hkv);
  const int32_t T_len = (int32_t)int_attr(cache, names.T_len);
  if (!described(cache, names.struct_, plain.struct_, plain.cache_type, c.cache_held, k)) {
    k.B = cache_B;
    k.Hkv = Hkv;
    k.G = (int32_t)int_attr(cache, names.G);
    k.T_cap = (int32_t)int_attr(cache, names.T_cap);
    k.S_cap = (int32_t)int_attr(cache, names.S_cap);
    k.T_len = T_len;
    k.k_codes = static_cast<uint32_t *>(ptr_attr(cache, names.k_codes));
    k.v_codes = static_cast<uint32_t *>(ptr_attr(cache, names.v_codes));
    k.k_meta = static_cast<uint32_t *>(ptr_attr(cache, names.k_meta));
    k.v_meta = static_cast<uint32_t *>(ptr_attr(cache, names.v_meta));
    k.k_sal = static_cast<uint16_t *>(ptr_attr(cache, names.k_sal));
    k.v_sal = static_cast<uint16_t *>(ptr_attr(cache, names.v_sal));
    k.sal_idx = static_cast<int32_t *>(ptr_attr(cache, names.sal_idx));
    k.sal_cnt = static_cast<int32_t *>(ptr_attr(cache, names.sal_cnt));
  } else if (c.cache_held.p == Py_None) {
    PyErr_SetString(PyExc_TypeError, "struct() of the cache returned None");
    throw Failed();
  }
  c.fine_mask = static_cast<uint32_t *>(ptr_attr(cache, names.fine_mask, true));
  const int64_t W = int_attr(cache, names.W);
  if (more_rows != 0 || W != 0 || c.fine_mask != nullptr || rope != Py_None) {
    if (described(cache, names.window_struct, plain.window_struct, plain.window_type, c.win_held, c.win)) {
      if (c.win_held.p != Py_None) c.win_p = &c.win;
    } else if (W != 0) {
      c.win = akvq_window{static_cast<uint16_t *>(ptr_attr(cache, names.k_win)),
                          static_cast<uint16_t *>(ptr_attr(cache, names.v_win)), (int32_t)W};
      c.win_p = &c.win;
    }
  }
  const at::Tensor &q = tensor(q_obj);
  REQUIRE(q.scalar_type() == at::kHalf && q.is_contiguous());
  if (q.dim() != 3) {
    PyErr_SetString(PyExc_ValueError, "q has to be [B, Hq, 128]");
    throw Failed();
  }
  const int64_t B = q.size(0);
  c.Hq = (int)q.size(1);
  c.q = q.data_ptr();
  c.sm_scale = (float)number(scale);
  c.flags = (uint32_t)integer(flags);
  const long n = integer(n_split);
  c.n_split = n > 0 ? (int)n : 0;
  const int most = n > 0 ? (int)n : akvq_decode_default_splits(cache_B, Hkv, (int)(T_len + more_rows));
  Held bytes(PyLong_FromSize_t(akvq_decode_workspace_bytes((int)B, c.Hq, most)));
  PyObject *args[3] = {cache, names.decode, bytes.p};
  Held ws(PyObject_VectorcallMethod(names.workspace, args, 3 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr));
  if (!ws.p) throw Failed();
  c.ws_tensor = tensor(ws.p);
  c.ws = c.ws_tensor.data_ptr();
  c.ws_bytes = (size_t)c.ws_tensor.numel();
  const at::ScalarType dtype = (c.flags & AKVQ_OUT_FP16) ? at::kHalf : at::kFloat;
  if (out == Py_None) c.out = at::empty({B, c.Hq, kHeadDim}, q.options().dtype(check_out ? dtype : at::kFloat).requires_grad(false));
  else c.out = tensor(out);
  if (check_out) REQUIRE(c.out.scalar_type() == dtype && c.out.is_contiguous());
  if (lse == Py_None) c.lse = at::empty({B, c.Hq}, q.options().dtype(at::kFloat).requires_grad(false));
  else c.lse = tensor(lse);
  if (rope != Py_None) {  // (a pair of two tensors: None inside it is an error)
    c.rope_pair.p = PySequence_Tuple(rope);
    if (!c.rope_pair.p) throw Failed();
    if (PyTuple_GET_SIZE(c.rope_pair.p) != 2) {
      PyErr_SetString(PyExc_ValueError, "rope has to be a pair (cos, sin)");
      throw Failed();
    }
    const at::Tensor &cos = tensor(PyTuple_GET_ITEM(c.rope_pair.p, 0)), &sin = tensor(PyTuple_GET_ITEM(c.rope_pair.p, 1));
    REQUIRE(cos.scalar_type() == at::kHalf && sin.scalar_type() == at::kHalf && cos.is_contiguous() && sin.is_contiguous());
    REQUIRE(cos.sizes() == sin.sizes() && cos.dim() >= 2 && cos.size(-2) == 1 && cos.size(-1) == 64);
    REQUIRE(cos.dim() == 2 || (cos.dim() == 3 && cos.size(0) == cache_B));
    c.rope = akvq_rope{static_cast<const uint16_t *>(cos.data_ptr()), static_cast<const uint16_t *>(sin.data_ptr()),
                       cos.dim() == 3 ? 64 : 0};
    c.rope_p = &c.rope;
  }
  c.stream = c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream();
}

PyObject *result(int status, Call &c) {
  Held out(THPVariable_Wrap(c.out)), lse(THPVariable_Wrap(c.lse));
  if (!out.p || !lse.p) return nullptr;
  return Py_BuildValue("iOO", status, out.p, lse.p);
}

// decode_attention(cache, q, sm_scale, n_split, flags, out, lse, rope) -> (status, out, lse)
PyObject *decode_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) {
    PyErr_SetString(PyExc_TypeError, "decode_attention takes 8 arguments");
    return nullptr;
  }
  try {
    Call c;
    gather(c, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], 0, true);
    void *const out = c.out.data_ptr();
    float *const lse = static_cast<float *>(c.lse.data_ptr());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = akvq_decode_attention_rope(&c.cache, c.fine_mask, c.win_p, c.q, c.rope_p, c.Hq, c.sm_scale, out, lse, c.n_split,
                                        c.ws, c.ws_bytes, c.flags, c.stream);
    Py_END_ALLOW_THREADS
    return result(status, c);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// decode_step(cache, k_new, v_new, q, clip, sm_scale, n_split, flags, out, lse, rope) -> (status, out, lse)
PyObject *decode_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11) {
    PyErr_SetString(PyExc_TypeError, "decode_step takes 11 arguments");
    return nullptr;
  }
  try {
    const at::Tensor &k = tensor(a[1]), &v = tensor(a[2]);
    REQUIRE(k.scalar_type() == at::kHalf && v.scalar_type() == at::kHalf);
    REQUIRE(k.is_contiguous() && v.is_contiguous());
    const int64_t shape[4] = {int_attr(a[0], names.B), int_attr(a[0], names.Hkv), 1, kHeadDim};
    REQUIRE(k.sizes() == at::IntArrayRef(shape, 4) && k.sizes() == v.sizes());
    const float clip = (float)number(a[4]);
    Call c;
    gather(c, a[0], a[3], a[5], a[6], a[7], a[8], a[9], a[10], 1, false);
    const void *const k_new = k.data_ptr(), *const v_new = v.data_ptr();
    void *const out = c.out.data_ptr();
    float *const lse = static_cast<float *>(c.lse.data_ptr());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = akvq_decode_step(&c.cache, c.fine_mask, c.win_p, k_new, v_new, c.q, c.rope_p, c.Hq, clip, c.sm_scale, out, lse,
                              c.n_split, c.ws, c.ws_bytes, c.flags, c.stream);
    Py_END_ALLOW_THREADS
    return result(status, c);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// ---- chunks: new rows of many sequences, packed token by token

// plain_paged(paged_struct, paged_type, error): as plain_cache below, for the cache in pages; what these calls raise
struct PlainPaged { PyObject *struct_ = nullptr, *type = nullptr, *error = PyExc_RuntimeError; } paged;

void need(bool ok, const char *what) {
  if (ok) return;
  PyErr_SetString(paged.error, what);
  throw Failed();
}
void need(bool ok, const char *what, const char *why) {
  if (ok) return;
  PyErr_Format(paged.error, "%s%s", what, why);
  throw Failed();
}
// The calls go to the current device's stream: a tensor of another device (or of the host) is refused.
struct Here {
  int device = -1;
  void operator()(const at::Tensor &t) {
    if (t.is_cuda() && device < 0) device = c10::hip::current_device();
    need(t.is_cuda() && t.get_device() == device, "tensors have to be on the current device");
  }
  void *stream() const { return c10::hip::getCurrentHIPStream(device).stream(); }
};
// [rows, heads, 128] fp16 whose heads lie next to each other; returns the elements from row to row.  rows, heads: -1: any
int64_t packed(const at::Tensor &t, const char *what, int64_t rows, int64_t heads) {
  need(t.scalar_type() == at::kHalf && t.dim() == 3 && t.size(2) == kHeadDim, what, " has to be fp16 [rows, heads, 128]");
  need((rows < 0 || t.size(0) == rows) && (heads < 0 || t.size(1) == heads), what, ": rows or heads do not fit");
  need(t.stride(2) == 1 && (t.size(1) == 1 || t.stride(1) == kHeadDim), what, ": the heads of a row have to lie next to each other");
  return t.size(0) > 1 ? t.stride(0) : t.size(1) * kHeadDim;
}
// The call writes into the caller's tensor, which autograd has to know of (inference tensors have no count of their changes).
void written(const at::Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// No call here records a gradient, or carries a tangent (forward-mode derivatives; none is there where they are switched off, as in inference mode).
// gradient, tangent: what is said of them
void no_gradient(const at::Tensor &t, const char *what, const char *gradient = " asks for a gradient, which this call does not record (the inverse turns it back)",
                 const char *tangent = " has a tangent, which this call does not carry (it turns as the rows do)") {
  need(!t.requires_grad() || !c10::GradMode::is_enabled(), what, gradient);
  need(!t._fw_grad(0).defined(), what, tangent);
}
at::Tensor fresh(at::IntArrayRef shape, const at::Tensor &like) { return at::empty(shape, like.options().dtype(at::kHalf).requires_grad(false)); }

template <typename Axes>
Axes axes_of(PyObject *o) {  // the description that RopeAxes or Rotary holds
  Axes axes;
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
  const bool fits = view.len == (Py_ssize_t)sizeof(axes);
  if (fits) std::memcpy(&axes, view.buf, sizeof(axes));
  PyBuffer_Release(&view);
  need(fits, "axes are described by something else");
  return axes;
}
// positions [axes, rows], or [rows] for one axis; returns the elements from axis to axis
int64_t positions(const at::Tensor &pos, int64_t rows, int axes) {
  need(pos.scalar_type() == at::kInt && (pos.dim() == 1 || pos.dim() == 2), "positions have to be int32 [axes, rows]");
  need(pos.size(-1) == rows && (pos.dim() == 2 ? pos.size(0) >= axes : axes == 1), "positions: one entry for every axis and row");
  need(rows <= 1 || pos.stride(-1) == 1, "positions: the rows of an axis have to lie next to each other");
  return pos.dim() == 2 && pos.size(0) > 1 ? pos.stride(0) : rows;
}
uint32_t flags_of(PyObject *o) {
  const long flags = integer(o);
  need(flags >= 0 && flags <= (long)UINT32_MAX, "flags do not fit 32 bits");
  return (uint32_t)flags;
}
int count(int64_t n, const char *what) {
  need(n >= 0 && n <= INT32_MAX, what, " does not fit 32 bits");
  return (int)n;
}

// Rows of a call that turns them: packed rows and where they go, which is a new tensor for None.
struct Turned {
  const void *in = nullptr;
  void *out_at = nullptr;
  int64_t stride = 0, out_stride = 0;
  int heads = 0;
  at::Tensor out;
  void take(PyObject *in_obj, PyObject *out_obj, const char *what, const char *what_out, int64_t rows, int64_t want_heads) {
    const at::Tensor &t = tensor(in_obj);
    stride = packed(t, what, rows, want_heads);
    out = out_obj == Py_None ? fresh(t.sizes(), t) : tensor(out_obj);
    out_stride = packed(out, what_out, rows, t.size(1));
    no_gradient(t, what);
    no_gradient(out, what_out);
    in = t.data_ptr();
    out_at = out.data_ptr();
    heads = count(t.size(1), "heads");
  }
  // a new reference to what the call returns for it
  PyObject *result(PyObject *in_obj, PyObject *out_obj) const {
    return in_obj == Py_None ? Py_NewRef(Py_None) : out_obj != Py_None ? Py_NewRef(out_obj) : THPVariable_Wrap(out);
  }
};

// (axes, pos, q, k, q_out, k_out, inverse) -> (status, (q_out, k_out)), of rope_axes and rotary_rows
template <typename Axes, typename Turn>
PyObject *turn_rows(PyObject *const *a, Py_ssize_t n, const char *name, Turn turn) {
  HANDLE_TH_ERRORS
  if (n != 7) {
    PyErr_Format(PyExc_TypeError, "%s takes 7 arguments", name);
    return nullptr;
  }
  try {
    need(a[2] != Py_None || a[3] != Py_None, "neither q nor k");
    const Axes axes = axes_of<Axes>(a[0]);
    const at::Tensor &pos = tensor(a[1]);
    const at::Tensor &lead = tensor(a[2] != Py_None ? a[2] : a[3]);
    need(lead.dim() == 3, a[2] != Py_None ? "q" : "k", " has to be fp16 [rows, heads, 128]");
    const int64_t rows = lead.size(0);
    Turned x[2];
    static const char *const what[2] = {"q", "k"}, *const what_out[2] = {"q_out", "k_out"}, *const without[2] = {"q_out without q", "k_out without k"};
    for (int i = 0; i < 2; ++i) {
      if (a[2 + i] == Py_None) need(a[4 + i] == Py_None, without[i]);
      else x[i].take(a[2 + i], a[4 + i], what[i], what_out[i], rows, -1);
    }
    const int64_t pos_stride = positions(pos, rows, axes.n_axes);
    Here here;
    here(pos);
    for (int i = 0; i < 2; ++i)
      if (a[2 + i] != Py_None) {
        here(tensor(a[2 + i]));
        here(x[i].out);
      }
    const int inverse = PyObject_IsTrue(a[6]);
    if (inverse < 0) return nullptr;
    int status = 0;
    if (rows > 0) {
      const int n_rows = count(rows, "rows");
      void *const stream = here.stream();
      const void *const at_pos = pos.data_ptr();
      Py_BEGIN_ALLOW_THREADS
      status = turn(&axes, static_cast<const int32_t *>(at_pos), pos_stride, n_rows, x[0].in, x[0].stride, x[0].heads, x[1].in, x[1].stride,
                    x[1].heads, x[0].out_at, x[0].out_stride, x[1].out_at, x[1].out_stride, inverse ? AKVQ_ROPE_INVERSE : 0, stream);
      Py_END_ALLOW_THREADS
      for (int i = 0; i < 2; ++i)
        if (a[4 + i] != Py_None) written(x[i].out);
    }
    Held q(x[0].result(a[2], a[4])), k(x[1].result(a[3], a[5]));
    if (!q.p || !k.p) return nullptr;
    return Py_BuildValue("i(OO)", status, q.p, k.p);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
PyObject *rope_axes(PyObject *, PyObject *const *a, Py_ssize_t n) { return turn_rows<akvq_axes>(a, n, "rope_axes", akvq_rope_axes); }
PyObject *rotary_rows(PyObject *, PyObject *const *a, Py_ssize_t n) { return turn_rows<akvq_rotary>(a, n, "rotary_rows", akvq_rotary_rows); }

// rope_axes_table(axes, pos) -> (status, (cos, sin))
PyObject *rope_axes_table(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "rope_axes_table takes 2 arguments");
    return nullptr;
  }
  try {
    const akvq_axes axes = axes_of<akvq_axes>(a[0]);
    const at::Tensor &pos = tensor(a[1]);
    need(pos.dim() == 1 || pos.dim() == 2, "positions have to be int32 [axes, rows]");
    const int64_t rows = pos.size(-1), pos_stride = positions(pos, rows, axes.n_axes);
    Here here;
    here(pos);
    const at::Tensor cos = fresh({rows, 64}, pos), sin = fresh({rows, 64}, pos);
    int status = 0;
    if (rows > 0)
      status = akvq_rope_axes_table(&axes, static_cast<const int32_t *>(pos.data_ptr()), pos_stride, count(rows, "rows"), cos.data_ptr(),
                                    sin.data_ptr(), here.stream());
    Held c(THPVariable_Wrap(cos)), s(THPVariable_Wrap(sin));
    if (!c.p || !s.p) return nullptr;
    return Py_BuildValue("i(OO)", status, c.p, s.p);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// The cache's description, and the device of its pools.
struct Pages {
  akvq_paged c;
  int bits;   // of a code
  Held held;  // keeps what the pointers come from
  Pages(PyObject *cache) : bits(bits_of(cache)) {
    if (described(cache, names.paged_struct, paged.struct_, paged.type, held, c)) {
      need(held.p != Py_None, "paged_struct() of the cache returned None");
      return;
    }
    struct { int32_t *to; PyObject *name; } ints[] = {
        {&c.B, names.B}, {&c.Hkv, names.Hkv}, {&c.G, names.G}, {&c.page_rows, names.page_rows}, {&c.n_pages, names.n_pages},
        {&c.max_pages, names.max_pages}, {&c.S_cap, names.S_cap}, {&c.max_len, names.max_len}};
    for (auto &i : ints) *i.to = (int32_t)std::min<int64_t>(std::max<int64_t>(int_attr(cache, i.name), INT32_MIN), INT32_MAX);
    c.k_codes = static_cast<uint32_t *>(ptr_attr(cache, names.k_codes));
    c.v_codes = static_cast<uint32_t *>(ptr_attr(cache, names.v_codes));
    c.k_meta = static_cast<uint32_t *>(ptr_attr(cache, names.k_meta));
    c.v_meta = static_cast<uint32_t *>(ptr_attr(cache, names.v_meta));
    c.k_sal = static_cast<uint16_t *>(ptr_attr(cache, names.k_sal));
    c.v_sal = static_cast<uint16_t *>(ptr_attr(cache, names.v_sal));
    c.sal_idx = static_cast<int32_t *>(ptr_attr(cache, names.sal_idx));
    c.sal_cnt = static_cast<int32_t *>(ptr_attr(cache, names.sal_cnt));
    c.table = static_cast<int32_t *>(ptr_attr(cache, names.table));
    c.seq_len = static_cast<int32_t *>(ptr_attr(cache, names.seq_len));
  }
  static int bits_of(PyObject *cache) {
    Held v(PyObject_GetAttr(cache, names.bits));
    if (!v.p) {  // (a cache that describes itself may know of no others)
      if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw Failed();
      PyErr_Clear();
      return 2;
    }
    const long bits = integer(v.p);
    need(bits == 2 || bits == 4, "codes have 2 or 4 bits");
    return (int)bits;
  }
  // where the pools lie; the two tensors that the caller writes may have been put there by the caller
  void on(PyObject *cache, Here &here) const {
    Held k(PyObject_GetAttr(cache, names.k_codes));
    if (!k.p) throw Failed();
    here(tensor(k.p));
    if (held.p) return;
    if (bits == 4) {  // (a pool of 2-bit codes has half the words)
      Held v(PyObject_GetAttr(cache, names.v_codes));
      if (!v.p) throw Failed();
      const int64_t words = (int64_t)c.n_pages * c.Hkv * c.page_rows * 16;
      need(tensor(k.p).numel() == words, "k_codes is no pool of 4-bit codes");
      need(tensor(v.p).numel() == words, "v_codes is no pool of 4-bit codes");
    }
    Held t(PyObject_GetAttr(cache, names.table)), s(PyObject_GetAttr(cache, names.seq_len));
    if (!t.p || !s.p) throw Failed();
    const at::Tensor &table = tensor(t.p), &len = tensor(s.p);
    need(table.scalar_type() == at::kInt && table.is_contiguous() && table.dim() == 2 && table.size(0) == c.B && table.size(1) == c.max_pages,
         "table has to be int32 [sequences, max_pages]");
    need(len.scalar_type() == at::kInt && len.is_contiguous() && len.dim() == 1 && len.size(0) == c.B, "seq_len has to be int32 [sequences]");
    here(table);
    here(len);
  }
};
akvq_chunk chunk_of(const Pages &p, const at::Tensor &row_start, int64_t rows, PyObject *max_rows) {
  need(row_start.scalar_type() == at::kInt && row_start.dim() == 1 && row_start.size(0) == p.c.B + 1 && row_start.is_contiguous(),
       "row_start has to be int32 [sequences + 1]");
  const long most = integer(max_rows);
  need(most >= 0, "max_rows has to be at least 0");
  return {static_cast<const int32_t *>(row_start.data_ptr()), count(rows, "rows"), (int32_t)std::min<long>(most, INT32_MAX)};
}

// paged_append(cache, k, v, row_start, max_rows, clip, flags) -> status
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "paged_append takes 7 arguments");
    return nullptr;
  }
  try {
    const Pages pages(a[0]);
    const at::Tensor &k = tensor(a[1]), &v = tensor(a[2]), &row_start = tensor(a[3]);
    const int64_t ks = packed(k, "k", -1, pages.c.Hkv), rows = k.size(0), vs = packed(v, "v", rows, pages.c.Hkv);
    const akvq_chunk chunk = chunk_of(pages, row_start, rows, a[4]);
    const float clip = (float)number(a[5]);
    const uint32_t flags = flags_of(a[6]);
    Here here;
    for (const at::Tensor *t : {&k, &v, &row_start}) here(*t);
    pages.on(a[0], here);
    int status = 0;
    if (rows > 0) {
      void *const stream = here.stream();
      const void *const k_at = k.data_ptr(), *const v_at = v.data_ptr();
      Py_BEGIN_ALLOW_THREADS
      status = (pages.bits == 4 ? akvq_paged_nibble_append : akvq_paged_append)(&pages.c, &chunk, k_at, ks, v_at, vs, clip, flags, stream);
      Py_END_ALLOW_THREADS
    }
    return PyLong_FromLong(status);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// paged_append_rotary(cache, rotary, pos, q, k, v, row_start, max_rows, clip, q_out, k_out, flags) -> (status, (q_out, k_out))
PyObject *paged_append_rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 12) {
    PyErr_SetString(PyExc_TypeError, "paged_append_rotary takes 12 arguments");
    return nullptr;
  }
  try {
    const Pages pages(a[0]);
    const akvq_rotary rotary = axes_of<akvq_rotary>(a[1]);
    const at::Tensor &pos = tensor(a[2]), &v = tensor(a[5]), &row_start = tensor(a[6]);
    Turned q, k;
    need(tensor(a[4]).dim() == 3, "k", " has to be fp16 [rows, heads, 128]");
    const int64_t rows = tensor(a[4]).size(0);
    k.take(a[4], a[10], "k", "k_out", rows, pages.c.Hkv);
    if (a[3] == Py_None) need(a[9] == Py_None, "q_out without q");
    else q.take(a[3], a[9], "q", "q_out", rows, -1);
    const int64_t vs = packed(v, "v", rows, pages.c.Hkv), pos_stride = positions(pos, rows, rotary.n_axes);
    const akvq_chunk chunk = chunk_of(pages, row_start, rows, a[7]);
    const float clip = (float)number(a[8]);
    const uint32_t flags = flags_of(a[11]);
    Here here;
    here(pos);
    here(tensor(a[4]));
    for (const at::Tensor *t : {static_cast<const at::Tensor *>(&k.out), &v, &row_start}) here(*t);
    if (a[3] != Py_None) {
      here(tensor(a[3]));
      here(q.out);
    }
    pages.on(a[0], here);
    int status = 0;
    if (rows > 0) {
      void *const stream = here.stream();
      const void *const v_at = v.data_ptr(), *const at_pos = pos.data_ptr();
      Py_BEGIN_ALLOW_THREADS
      status = akvq_paged_append_rotary(&pages.c, pages.bits, &chunk, &rotary, static_cast<const int32_t *>(at_pos), pos_stride, q.in, q.stride,
                                        q.heads, k.in, k.stride, v_at, vs, q.out_at, q.out_stride, k.out_at, k.out_stride, clip, flags, stream);
      Py_END_ALLOW_THREADS
      if (a[9] != Py_None) written(q.out);
      if (a[10] != Py_None) written(k.out);
    }
    Held q_out(q.result(a[3], a[9])), k_out(k.result(a[4], a[10]));
    if (!q_out.p || !k_out.p) return nullptr;
    return Py_BuildValue("i(OO)", status, q_out.p, k_out.p);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// paged_attention(cache, q, k, v, row_start, max_rows, sm_scale, n_split, flags, out, lse) -> (status, out)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11) {
    PyErr_SetString(PyExc_TypeError, "paged_attention takes 11 arguments");
    return nullptr;
  }
  try {
    const Pages pages(a[0]);
    const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]), &v = tensor(a[3]), &row_start = tensor(a[4]);
    const int64_t qs = packed(q, "q", -1, -1), rows = q.size(0), ks = packed(k, "k", rows, pages.c.Hkv), vs = packed(v, "v", rows, pages.c.Hkv);
    const int Hq = count(q.size(1), "heads");
    const akvq_chunk chunk = chunk_of(pages, row_start, rows, a[5]);
    const at::Tensor out = a[9] == Py_None ? fresh(q.sizes(), q) : tensor(a[9]);
    const int64_t os = packed(out, "out", rows, Hq);
    const at::Tensor lse = a[10] == Py_None ? at::Tensor() : tensor(a[10]);
    need(!lse.defined() || (lse.scalar_type() == at::kFloat && lse.is_contiguous() && lse.dim() == 2 && lse.size(0) == rows && lse.size(1) == Hq),
         "lse has to be fp32 [rows, Hq]");
    const float sm_scale = (float)number(a[6]);
    const long asked = integer(a[7]);
    const uint32_t flags = flags_of(a[8]);
    if (pages.bits == 4) {  // (over 2-bit codes programs have been answered without a gradient, and still are)
      static const char *const name[5] = {"q", "k", "v", "out", "lse"};
      const at::Tensor *const t[5] = {&q, &k, &v, &out, &lse};
      for (int i = 0; i < 5; ++i)
        if (t[i]->defined()) no_gradient(*t[i], name[i], " asks for a gradient, which this call does not record (torch.no_grad answers without)", " has a tangent, which this call does not carry");
    }
    Here here;
    for (const at::Tensor *t : {&q, &k, &v, &row_start, &out}) here(*t);
    if (lse.defined()) here(lse);
    pages.on(a[0], here);
    void *const lse_at = lse.defined() ? lse.data_ptr() : nullptr;
    int status = 0;
    if (rows > 0) {
      const bool four = pages.bits == 4;
      const int n_split = asked > 0 ? (int)std::min<long>(asked, INT32_MAX)
                                    : (four ? akvq_paged_nibble_default_splits : akvq_paged_default_splits)(&pages.c, Hq, std::min(chunk.max_rows, chunk.n_rows));
      const size_t bytes = n_split <= 1024 ? akvq_paged_workspace_bytes(chunk.n_rows, Hq, n_split) : 0;  // (more is refused by the call)
      at::Tensor ws;  // of its own for every call: calls on two streams, or two captured graphs, share none
      if (bytes) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte).requires_grad(false));
      void *const stream = here.stream(), *const ws_at = bytes ? ws.data_ptr() : nullptr, *const out_at = out.data_ptr();
      const void *const q_at = q.data_ptr(), *const k_at = k.data_ptr(), *const v_at = v.data_ptr();
      Py_BEGIN_ALLOW_THREADS
      status = (four ? akvq_paged_nibble_attention : akvq_paged_attention)(&pages.c, &chunk, q_at, qs, Hq, k_at, ks, v_at, vs, sm_scale, out_at, os,
                                                                     static_cast<float *>(lse_at), n_split, ws_at, bytes, flags, stream);
      Py_END_ALLOW_THREADS
      if (a[9] != Py_None) written(out);
      if (lse.defined()) written(lse);
    }
    Held o(a[9] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[9]));
    if (!o.p) return nullptr;
    return Py_BuildValue("iO", status, o.p);
  } catch (const Failed &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject *plain_paged(PyObject *, PyObject *args) {
  PlainPaged p;
  if (!PyArg_ParseTuple(args, "OOO", &p.struct_, &p.type, &p.error)) return nullptr;
  for (PyObject *o : {p.struct_, p.type, p.error}) Py_INCREF(o);
  paged = p;
  Py_RETURN_NONE;
}

// plain_cache(struct, window_struct, cache_type, window_type): the functions of the package's own cache class, and the types
// they return
PyObject *plain_cache(PyObject *, PyObject *args) {
  Plain p;
  if (!PyArg_ParseTuple(args, "OOOO", &p.struct_, &p.window_struct, &p.cache_type, &p.window_type)) return nullptr;
  for (PyObject *o : {p.struct_, p.window_struct, p.cache_type, p.window_type}) Py_INCREF(o);
  plain = p;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"plain_cache", plain_cache, METH_VARARGS, nullptr},
    {"decode_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_attention)), METH_FASTCALL, nullptr},
    {"decode_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_step)), METH_FASTCALL, nullptr},
    {"plain_paged", plain_paged, METH_VARARGS, nullptr},
    {"rope_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rope_axes)), METH_FASTCALL, nullptr},
    {"rope_axes_table", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rope_axes_table)), METH_FASTCALL, nullptr},
    {"rotary_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary_rows)), METH_FASTCALL, nullptr},
    {"paged_append_rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append_rotary)), METH_FASTCALL, nullptr},
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_akvq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__akvq_torch(void) {
  struct { PyObject **slot; const char *text; } table[] = {
      {&names.B, "B"}, {&names.Hkv, "Hkv"}, {&names.G, "G"}, {&names.T_cap, "T_cap"}, {&names.S_cap, "S_cap"},
      {&names.T_len, "T_len"}, {&names.k_codes, "k_codes"}, {&names.v_codes, "v_codes"}, {&names.k_meta, "k_meta"},
      {&names.v_meta, "v_meta"}, {&names.k_sal, "k_sal"}, {&names.v_sal, "v_sal"}, {&names.sal_idx, "sal_idx"},
      {&names.sal_cnt, "sal_cnt"}, {&names.fine_mask, "fine_mask"}, {&names.W, "W"}, {&names.k_win, "k_win"},
      {&names.v_win, "v_win"}, {&names.workspace, "workspace"}, {&names.decode, "decode"},
      {&names.struct_, "struct"}, {&names.window_struct, "window_struct"},
      {&names.page_rows, "page_rows"}, {&names.n_pages, "n_pages"}, {&names.max_pages, "max_pages"}, {&names.max_len, "max_len"},
      {&names.table, "table"}, {&names.seq_len, "seq_len"}, {&names.paged_struct, "paged_struct"}, {&names.bits, "bits"}};
  for (auto &t : table)
    if ((*t.slot = PyUnicode_InternFromString(t.text)) == nullptr) return nullptr;
  return PyModule_Create(&module);
}
