// Argument marshalling of the binding's per-call path, native: from the tensors a caller passes to one call of the C ABI.
//
// Every function takes the address of an entry point (of the library that is loaded), then the arguments of the Python
// function of the same name, and returns the entry's status -- or None where the call is not of the plain form: anything but
// exact torch tensors in device memory, of the types, layouts and sizes that the checks of the Python functions ask for.  Those
// then run, and convert or refuse as ever, so no check and no error message lives here.  No result and no address is kept
// from one call to the next.
//
// Why: at a few images a block's kernels take less time than enqueuing them, and ctypes with attribute lookups on some
// ten tensors took 2.6 us of masker_ex's 10 and 5 us of the packed block's 17.
#include <torch/csrc/autograd/python_variable.h>

#include "lasnet.h"

namespace {

PyObject *g_current_device, *g_current_stream;       // torch._C._cuda_getDevice, _cuda_getCurrentRawStream

// a tensor that is no subclass (those may override what is read here), or nullptr
inline const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

struct Plain {                                       // false from any of these: not the plain form
  bool ok = true;
  bool need(bool v) { return ok = ok && v; }

  bool map(PyObject* o, lasnet_tensor& d) {          // a feature map
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined() && t->dim() == 4 && t->is_cuda() && t->is_contiguous())) return false;
    const auto ty = t->scalar_type();
    if (!need(ty == at::kFloat || ty == at::kBFloat16)) return false;
    int32_t* sizes[4] = {&d.n, &d.h, &d.w, &d.c};
    for (int i = 0; i < 4; ++i) {
      if (!need(t->size(i) <= INT32_MAX)) return false;
      *sizes[i] = (int32_t)t->size(i);
    }
    d.data = t->data_ptr();
    d.dtype = ty == at::kFloat ? LASNET_F32 : LASNET_BF16;
    return true;
  }
  template <class T>
  T* of_type(PyObject* o, at::ScalarType ty) {
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined() && t->scalar_type() == ty && t->is_cuda() && t->is_contiguous())) return nullptr;
    return (T*)t->data_ptr();
  }
  const float* bias(PyObject* o, int64_t n) {
    const float* p = of_type<const float>(o, at::kFloat);
    return ok && need(tensor(o)->numel() == n) ? p : nullptr;
  }
  template <class T>
  T* any(PyObject* o) {                              // what the Python function passes on unchecked
    const at::Tensor* t = tensor(o);
    return need(t && t->defined()) ? (T*)t->data_ptr() : nullptr;
  }
  const void* weight(PyObject* o, const lasnet_tensor& x, std::initializer_list<int64_t> shape) {
    const at::Tensor* t = tensor(o);
    const auto ty = x.dtype == LASNET_F32 ? at::kFloat : at::kBFloat16;
    if (!need(t && t->defined() && t->scalar_type() == ty && t->is_cuda() && t->is_contiguous() && t->sizes() == at::IntArrayRef(shape))) return nullptr;
    return t->data_ptr();
  }
  int integer(PyObject* o) {
    if (!need(PyLong_CheckExact(o))) return 0;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    need(!over && v >= INT32_MIN && v <= INT32_MAX);
    return (int)v;
  }
  float real(PyObject* o) {
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    return (float)integer(o);
  }
  // rows: dense in two dimensions, apart or not; of more dimensions contiguous
  void rows(PyObject* o, lasnet_rows& d) {
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined() && t->dim() >= 2 && t->is_cuda())) return;
    const auto ty = t->scalar_type();
    if (!need(ty == at::kFloat || ty == at::kBFloat16 || ty == at::ScalarType::Float8_e4m3fn)) return;
    const int64_t cols = t->size(-1);
    if (!need(cols > 0 && cols <= INT32_MAX)) return;
    d.rows = t->numel() / cols;
    d.cols = (int32_t)cols;
    d.stride = cols;
    if (!t->is_contiguous()) {
      if (!need(t->dim() == 2 && (cols == 1 || t->stride(1) == 1))) return;
      if (d.rows > 1) {
        d.stride = t->stride(0);
        need(d.stride >= cols);
      }
    }
    d.data = t->data_ptr();
    d.dtype = ty == at::kFloat ? LASNET_F32 : ty == at::kBFloat16 ? LASNET_BF16 : LASNET_E4M3;
  }
  const lasnet_rows* rows_or_none(PyObject* o, lasnet_rows& d) {
    if (o == Py_None) return nullptr;
    rows(o, d);
    return &d;
  }
  // a dense tensor of so many elements, or None
  template <class T>
  T* dense(PyObject* o, at::ScalarType ty, int64_t n) {
    if (o == Py_None || !ok) return nullptr;
    T* t = of_type<T>(o, ty);
    return ok && need(tensor(o)->numel() == n) ? t : nullptr;
  }
  template <class T>
  T* scale(PyObject* o, int64_t n) {
    if (o == Py_None || !ok) return nullptr;
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined())) return nullptr;
    return dense<T>(o, t->scalar_type() == at::kByte ? at::kByte : at::ScalarType::Float8_e8m0fnu, n);
  }
  // bytes or truth values, or None
  const uint8_t* mask(PyObject* o, int64_t n) {
    if (o == Py_None || !ok) return nullptr;
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined())) return nullptr;
    return dense<const uint8_t>(o, t->scalar_type() == at::kBool ? at::kBool : at::kByte, n);
  }
  // [tokens, k]
  const int32_t* slots(PyObject* o, int64_t& tokens, int& k) {
    const int32_t* p = of_type<const int32_t>(o, at::kInt);
    if (!ok || !need(tensor(o)->dim() == 2 && tensor(o)->size(1) <= INT32_MAX)) return nullptr;
    tokens = tensor(o)->size(0);
    k = (int)tensor(o)->size(1);
    return p;
  }
  // [E + 1]
  const int32_t* offsets(PyObject* o, int& E) {
    const int32_t* p = of_type<const int32_t>(o, at::kInt);
    if (!ok || !need(tensor(o)->dim() == 1 && tensor(o)->numel() >= 2 && tensor(o)->numel() <= INT32_MAX)) return nullptr;
    E = (int)tensor(o)->numel() - 1;
    return p;
  }
  void* matrices(PyObject* o, int64_t E, int64_t n, int64_t k, at::ScalarType ty) {
    const at::Tensor* t = tensor(o);
    const int64_t shape[3] = {E, n, k};
    return need(t && t->defined() && t->scalar_type() == ty && t->is_cuda() && t->is_contiguous() && t->sizes() == at::IntArrayRef(shape, 3)) ? t->data_ptr() : nullptr;
  }
  // None, or a dense tensor of any type on the device of another argument
  void* workspace(PyObject* o, PyObject* beside, size_t& bytes) {
    bytes = 0;
    if (o == Py_None || !ok) return nullptr;
    const at::Tensor* t = tensor(o);
    if (!need(t && t->defined() && t->is_cuda() && t->device() == tensor(beside)->device() && t->is_contiguous())) return nullptr;
    bytes = t->nbytes();
    return t->data_ptr();
  }
  // the list: storage for every cell of the map (the kernels may read entries past the count)
  void list(PyObject* idx, PyObject* count, const lasnet_tensor& x, int S, const int32_t*& i, const int32_t*& c) {
    i = c = nullptr;
    if (count != Py_None) c = of_type<const int32_t>(count, at::kInt);
    if (idx != Py_None) {
      i = of_type<const int32_t>(idx, at::kInt);
      if (ok) need(S > 0 && x.h % S == 0 && x.w % S == 0 && tensor(idx)->numel() >= (int64_t)x.n * (x.h / S) * (x.w / S));
    }
  }
};

void* current_stream() {
  PyObject* device = PyObject_CallNoArgs(g_current_device);
  if (!device) return nullptr;
  PyObject* stream = PyObject_CallOneArg(g_current_stream, device);
  Py_DECREF(device);
  if (!stream) return nullptr;
  void* st = PyLong_AsVoidPtr(stream);
  Py_DECREF(stream);
  return st;
}

// body(plain) marshals and, where plain.ok, calls the entry
template <class Body>
PyObject* call(Py_ssize_t n, Py_ssize_t want, Body&& body) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  int status = 0;
  Plain p;
  try {
    status = body(p);
  } catch (const std::exception&) {                  // a tensor without storage, for instance
    p.ok = false;
  }
  if (PyErr_Occurred()) return nullptr;
  if (!p.ok) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}
template <class F>
F* entry(PyObject* address) { return (F*)PyLong_AsVoidPtr(address); }

#define ENQUEUE(...)              \
  void* st = current_stream();    \
  if (PyErr_Occurred()) return 0; \
  int status;                     \
  Py_BEGIN_ALLOW_THREADS          \
  status = __VA_ARGS__;           \
  Py_END_ALLOW_THREADS            \
  return status

// (x, Wm, bm, S, thr, mask, idx, count, pass_out)
PyObject* masker_ex(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&](Plain& p) {
    lasnet_tensor x, o;
    p.map(a[1], x);
    const float* Wm = p.of_type<const float>(a[2], at::kFloat);
    const float bm = p.real(a[3]), thr = p.real(a[5]);
    const int S = p.integer(a[4]);
    uint8_t* mask = p.any<uint8_t>(a[6]);
    int32_t *idx = p.any<int32_t>(a[7]), *count = p.any<int32_t>(a[8]);
    if (a[9] != Py_None) p.map(a[9], o);
    if (!p.ok || !p.need(S > 0 && x.h % S == 0 && x.w % S == 0)) return 0;
    lasnet_tensor* out = a[9] != Py_None ? &o : nullptr;
    auto* f = entry<decltype(lasnet_masker_ex)>(a[0]);
    ENQUEUE(f(&x, Wm, bm, S, thr, mask, idx, count, out, st));
  });
}

// (x, idx, count, S, M, packed, need, b1, b2, b3, out, flags); need: bytes that `packed` must hold, 0 if the shape has none
PyObject* block_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 13, [&](Plain& p) {
    lasnet_tensor x, o;
    p.map(a[1], x);
    const int S = p.integer(a[4]), M = p.integer(a[5]), flags = p.integer(a[12]);
    const int32_t *idx, *count;
    p.list(a[2], a[3], x, S, idx, count);
    const void* packed = p.any<const void>(a[6]);
    if (!p.ok) return 0;
    const size_t need = entry<decltype(lasnet_packed_weights_bytes)>(a[7])(LASNET_BF16, x.c, M, S);
    p.need((size_t)tensor(a[6])->nbytes() >= need);
    const float *b1 = p.bias(a[8], M), *b2 = p.bias(a[9], M), *b3 = p.bias(a[10], x.c);
    p.map(a[11], o);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_sparse_bottleneck_packed)>(a[0]);
    ENQUEUE(f(&x, idx, count, S, M, packed, b1, b2, b3, &o, (uint32_t)flags, st));
  });
}

// (x, idx, count, mask, S, M, packed, b1, b2, b3, out, workspace, flags)
PyObject* block_planned(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 14, [&](Plain& p) {
    lasnet_tensor x, o;
    p.map(a[1], x);
    const int S = p.integer(a[5]), M = p.integer(a[6]), flags = p.integer(a[13]);
    const int32_t *idx, *count;
    p.list(a[2], a[3], x, S, idx, count);
    const uint8_t* mask = a[4] == Py_None ? nullptr : p.of_type<const uint8_t>(a[4], at::kByte);
    const void* packed = p.any<const void>(a[7]);
    if (!p.ok) return 0;
    const float *b1 = p.bias(a[8], M), *b2 = p.bias(a[9], M), *b3 = p.bias(a[10], x.c);
    p.map(a[11], o);
    void* workspace = a[12] == Py_None ? nullptr : p.any<void>(a[12]);
    if (!p.ok) return 0;
    const size_t bytes = a[12] == Py_None ? 0 : tensor(a[12])->nbytes();
    auto* f = entry<decltype(lasnet_sparse_bottleneck_planned)>(a[0]);
    ENQUEUE(f(&x, idx, count, mask, S, M, packed, b1, b2, b3, &o, (uint32_t)flags, workspace, bytes, st));
  });
}

struct Weights { const void *W1, *W2, *W3; const float *b1, *b2, *b3; int M; };
// w: W1, b1, W2, b2, W3, b3
inline void weights(Plain& p, PyObject* const* w, const lasnet_tensor& x, Weights& r) {
  const at::Tensor* W1 = tensor(w[0]);
  if (!p.need(W1 && W1->defined() && W1->dim() == 2 && W1->size(0) <= INT32_MAX)) return;
  const int64_t M = W1->size(0);
  r.M = (int)M;
  r.W1 = p.weight(w[0], x, {M, x.c});
  r.b1 = p.bias(w[1], M);
  r.W2 = p.weight(w[2], x, {M, 3, 3, M});
  r.b2 = p.bias(w[3], M);
  r.W3 = p.weight(w[4], x, {x.c, M});
  r.b3 = p.bias(w[5], x.c);
}

// (x, idx, count, S, W1, b1, W2, b2, W3, b3, out, flags)
PyObject* block_ex(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 13, [&](Plain& p) {
    lasnet_tensor x, o;
    if (!p.map(a[1], x)) return 0;
    const int S = p.integer(a[4]), flags = p.integer(a[12]);
    const int32_t *idx, *count;
    p.list(a[2], a[3], x, S, idx, count);
    Weights w;
    weights(p, a + 5, x, w);
    p.map(a[11], o);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_sparse_bottleneck_ex)>(a[0]);
    ENQUEUE(f(&x, idx, count, S, w.M, w.W1, w.b1, w.W2, w.b2, w.W3, w.b3, &o, (uint32_t)flags, st));
  });
}

// (x, W1, b1, W2, b2, W3, b3, out, flags)
PyObject* block_dense(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&](Plain& p) {
    lasnet_tensor x, o;
    if (!p.map(a[1], x)) return 0;
    const int flags = p.integer(a[9]);
    Weights w;
    weights(p, a + 2, x, w);
    p.map(a[8], o);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_dense_bottleneck)>(a[0]);
    ENQUEUE(f(&x, w.M, w.W1, w.b1, w.W2, w.b2, w.W3, w.b3, &o, (uint32_t)flags, st));
  });
}

// (x, weight, eps, residual, out, scale, sum_out, rstd)
PyObject* norm_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 9, [&](Plain& p) {
    lasnet_rows x, res, out, sum;
    p.rows(a[1], x);
    if (!p.ok) return 0;
    const float* weight = p.dense<const float>(a[2], at::kFloat, x.cols);
    const float eps = p.real(a[3]);
    const lasnet_rows *r = p.rows_or_none(a[4], res), *s = p.rows_or_none(a[7], sum);
    p.rows(a[5], out);
    uint8_t* scale = p.scale<uint8_t>(a[6], x.rows);
    float* rstd = p.dense<float>(a[8], at::kFloat, x.rows);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_norm_rows)>(a[0]);
    ENQUEUE(f(&x, r, weight, eps, s, &out, scale, rstd, st));
  });
}

// (dy, s, weight, rstd, dsum, dx, dweight, workspace)
PyObject* norm_rows_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 9, [&](Plain& p) {
    lasnet_rows dy, s, sum, dx;
    p.rows(a[1], dy);
    p.rows(a[2], s);
    if (!p.ok) return 0;
    const float* weight = p.dense<const float>(a[3], at::kFloat, s.cols);
    const float* rstd = p.dense<const float>(a[4], at::kFloat, s.rows);
    const lasnet_rows* dsum = p.rows_or_none(a[5], sum);
    p.rows(a[6], dx);
    float* dweight = p.dense<float>(a[7], at::kFloat, s.cols);
    size_t bytes;
    void* workspace = p.workspace(a[8], a[2], bytes);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_norm_rows_backward)>(a[0]);
    ENQUEUE(f(&dy, &s, weight, rstd, dsum, &dx, dweight, workspace, bytes, st));
  });
}

// (experts, E, offsets, order, position, workspace)
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&](Plain& p) {
    int64_t tokens;
    int k;
    const int32_t* experts = p.slots(a[1], tokens, k);
    const int E = p.integer(a[2]);
    if (!p.ok) return 0;
    int32_t* offsets = p.dense<int32_t>(a[3], at::kInt, (int64_t)E + 1);
    int32_t* order = p.dense<int32_t>(a[4], at::kInt, tokens * k);
    int32_t* position = p.dense<int32_t>(a[5], at::kInt, tokens * k);
    size_t bytes;
    void* workspace = p.workspace(a[6], a[1], bytes);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_route)>(a[0]);
    ENQUEUE(f(experts, tokens, k, E, offsets, order, position, workspace, bytes, st));
  });
}

// (x, position, offsets, scale, out, out_scale)
PyObject* dispatch_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&](Plain& p) {
    lasnet_rows x, out;
    int64_t tokens;
    int k, E;
    p.rows(a[1], x);
    const int32_t* position = p.slots(a[2], tokens, k);
    const int32_t* offsets = p.offsets(a[3], E);
    p.rows(a[5], out);
    if (!p.ok || !p.need(x.rows == tokens)) return 0;
    const uint8_t* scale = p.scale<const uint8_t>(a[4], tokens);
    uint8_t* out_scale = p.scale<uint8_t>(a[6], tokens * k);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_dispatch_rows)>(a[0]);
    ENQUEUE(f(&x, scale, position, offsets, k, E, &out, out_scale, st));
  });
}

// (y, position, weights, base, out)
PyObject* combine_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&](Plain& p) {
    lasnet_rows y, b, out;
    int64_t tokens;
    int k;
    p.rows(a[1], y);
    const int32_t* position = p.slots(a[2], tokens, k);
    const lasnet_rows* base = p.rows_or_none(a[4], b);
    p.rows(a[5], out);
    if (!p.ok || !p.need(out.rows == tokens)) return 0;
    const float* weights = p.dense<const float>(a[3], at::kFloat, tokens * k);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_combine_rows)>(a[0]);
    ENQUEUE(f(&y, weights, position, k, base, &out, st));
  });
}

// (dout, y, position, offsets, weights, dy, dweights)
PyObject* combine_rows_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&](Plain& p) {
    lasnet_rows dout, y, dy;
    int64_t tokens;
    int k, E;
    p.rows(a[1], dout);
    p.rows(a[2], y);
    const int32_t* position = p.slots(a[3], tokens, k);
    const int32_t* offsets = p.offsets(a[4], E);
    p.rows(a[6], dy);
    if (!p.ok || !p.need(dout.rows == tokens)) return 0;
    const float* weights = p.dense<const float>(a[5], at::kFloat, tokens * k);
    float* dweights = p.dense<float>(a[7], at::kFloat, tokens * k);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_combine_rows_backward)>(a[0]);
    ENQUEUE(f(&dout, &y, weights, position, offsets, k, E, &dy, dweights, st));
  });
}

inline at::ScalarType row_type(int dtype) {
  return dtype == LASNET_F32 ? at::kFloat : dtype == LASNET_BF16 ? at::kBFloat16 : at::ScalarType::Float8_e4m3fn;
}

// (x, offsets, W, scale, wscale, out, flags)
PyObject* expert_product(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&](Plain& p) {
    lasnet_rows x, out;
    int E;
    p.rows(a[1], x);
    const int32_t* offsets = p.offsets(a[2], E);
    p.rows(a[6], out);
    const int flags = p.integer(a[7]);
    if (!p.ok) return 0;
    const void* W = p.matrices(a[3], E, out.cols, x.cols, row_type(x.dtype));
    const uint8_t* scale = p.scale<const uint8_t>(a[4], x.rows);
    const float* wscale = p.dense<const float>(a[5], at::kFloat, (int64_t)E * out.cols);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_expert_product)>(a[0]);
    ENQUEUE(f(&x, scale, offsets, E, W, wscale, &out, (uint32_t)flags, st));
  });
}

// (dy, offsets, W, dx)
PyObject* expert_product_dx(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 5, [&](Plain& p) {
    lasnet_rows dy, dx;
    int E;
    p.rows(a[1], dy);
    const int32_t* offsets = p.offsets(a[2], E);
    p.rows(a[4], dx);
    if (!p.ok) return 0;
    const void* W = p.matrices(a[3], E, dy.cols, dx.cols, row_type(dy.dtype));
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_expert_product_dx)>(a[0]);
    ENQUEUE(f(&dy, offsets, E, W, &dx, st));
  });
}

// (dy, x, offsets, dW, workspace)
PyObject* expert_product_dw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&](Plain& p) {
    lasnet_rows dy, x;
    int E;
    p.rows(a[1], dy);
    p.rows(a[2], x);
    const int32_t* offsets = p.offsets(a[3], E);
    const at::Tensor* dW = tensor(a[4]);
    if (!p.ok || !p.need(dW && dW->defined())) return 0;
    const auto ty = dW->scalar_type();
    p.need(ty == at::kFloat || ty == at::kBFloat16);
    void* to = p.matrices(a[4], E, dy.cols, x.cols, ty);
    size_t bytes;
    void* workspace = p.workspace(a[5], a[2], bytes);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_expert_product_dw_ex)>(a[0]);
    ENQUEUE(f(&dy, &x, offsets, E, to, ty == at::kFloat ? LASNET_F32 : LASNET_BF16, workspace, bytes, st));
  });
}

// (logits, mask, k, experts, weights, lse, flags)
PyObject* choose_experts(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&](Plain& p) {
    lasnet_rows logits;
    p.rows(a[1], logits);
    const int k = p.integer(a[3]), flags = p.integer(a[7]);
    if (!p.ok) return 0;
    const uint8_t* mask = p.mask(a[2], logits.rows);
    int32_t* experts = p.dense<int32_t>(a[4], at::kInt, logits.rows * k);
    float* weights = p.dense<float>(a[5], at::kFloat, logits.rows * k);
    float* lse = p.dense<float>(a[6], at::kFloat, logits.rows);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_choose_experts)>(a[0]);
    ENQUEUE(f(&logits, mask, k, experts, weights, lse, (uint32_t)flags, st));
  });
}

// (logits, lse, experts, counts, share, loss, workspace)
PyObject* balance(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&](Plain& p) {
    lasnet_rows logits;
    int64_t tokens;
    int k;
    p.rows(a[1], logits);
    const int32_t* experts = p.slots(a[3], tokens, k);
    if (!p.ok || !p.need(tokens == logits.rows)) return 0;
    const float* lse = p.dense<const float>(a[2], at::kFloat, logits.rows);
    int32_t* counts = p.dense<int32_t>(a[4], at::kInt, (int64_t)logits.cols + 1);
    float* share = p.dense<float>(a[5], at::kFloat, logits.cols);
    float* loss = p.dense<float>(a[6], at::kFloat, 2);
    size_t bytes;
    void* workspace = p.workspace(a[7], a[1], bytes);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_balance)>(a[0]);
    ENQUEUE(f(&logits, lse, experts, k, counts, share, loss, workspace, bytes, st));
  });
}

// (logits, lse, experts, weights, dweights, counts, dloss, dlogits, flags)
PyObject* choose_experts_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&](Plain& p) {
    lasnet_rows logits, dlogits;
    int64_t tokens;
    int k;
    p.rows(a[1], logits);
    const int32_t* experts = p.slots(a[3], tokens, k);
    p.rows(a[8], dlogits);
    const int flags = p.integer(a[9]);
    if (!p.ok || !p.need(tokens == logits.rows)) return 0;
    const float* lse = p.dense<const float>(a[2], at::kFloat, logits.rows);
    const float* weights = p.dense<const float>(a[4], at::kFloat, tokens * k);
    const float* dweights = p.dense<const float>(a[5], at::kFloat, tokens * k);
    const int32_t* counts = p.dense<const int32_t>(a[6], at::kInt, (int64_t)logits.cols + 1);
    const float* dloss = p.dense<const float>(a[7], at::kFloat, 2);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_choose_experts_backward)>(a[0]);
    ENQUEUE(f(&logits, lse, experts, weights, k, dweights, counts, dloss, &dlogits, (uint32_t)flags, st));
  });
}

inline int64_t blocks(int64_t n) { return (n + 127) / 128; }

// (x, position, offsets, out, scale)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&](Plain& p) {
    lasnet_rows x, out;
    int64_t tokens = 0;
    int k = 1, E = 1;
    p.rows(a[1], x);
    p.rows(a[4], out);
    const int32_t *position = nullptr, *offsets = nullptr;
    if (!p.ok || !p.need((a[2] == Py_None) == (a[3] == Py_None))) return 0;
    if (a[2] != Py_None) {
      position = p.slots(a[2], tokens, k);
      offsets = p.offsets(a[3], E);
      if (!p.ok || !p.need(tokens == x.rows)) return 0;
    }
    uint8_t* scale = p.scale<uint8_t>(a[5], x.rows * k * blocks(x.cols));
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_quantize_rows)>(a[0]);
    ENQUEUE(f(&x, position, offsets, k, E, &out, scale, st));
  });
}

// (W, out, scale, out_t, scale_t)
PyObject* quantize_matrices(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&](Plain& p) {
    const at::Tensor* W = tensor(a[1]);
    if (!p.need(W && W->defined() && W->dim() == 3 && W->size(0) <= INT32_MAX && W->size(1) <= INT32_MAX && W->size(2) <= INT32_MAX)) return 0;
    const auto ty = W->scalar_type();
    if (!p.need((ty == at::kFloat || ty == at::kBFloat16) && (a[4] == Py_None) == (a[5] == Py_None))) return 0;
    const int64_t E = W->size(0), rows = W->size(1), k = W->size(2), cells = E * blocks(rows) * blocks(k);
    const void* from = p.matrices(a[1], E, rows, k, ty);
    void* out = p.matrices(a[2], E, rows, k, at::ScalarType::Float8_e4m3fn);
    uint8_t* scale = p.scale<uint8_t>(a[3], cells);
    void* out_t = a[4] == Py_None ? nullptr : p.matrices(a[4], E, k, rows, at::ScalarType::Float8_e4m3fn);
    uint8_t* scale_t = p.scale<uint8_t>(a[5], cells);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_quantize_matrices)>(a[0]);
    ENQUEUE(f(from, ty == at::kFloat ? LASNET_F32 : LASNET_BF16, (int)E, (int)rows, (int)k, out, scale, out_t, scale_t, st));
  });
}

// (x, scale, offsets, W, wscale, out, flags)
PyObject* block_product(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&](Plain& p) {
    lasnet_rows x, out;
    int E;
    p.rows(a[1], x);
    const int32_t* offsets = p.offsets(a[3], E);
    p.rows(a[6], out);
    const int flags = p.integer(a[7]);
    const at::Tensor* ws = tensor(a[5]);
    if (!p.ok || !p.need(ws && ws->defined())) return 0;
    const bool floats = ws->scalar_type() == at::kFloat;
    const int64_t cells = E * blocks(out.cols) * blocks(x.cols);
    const void* W = p.matrices(a[4], E, out.cols, x.cols, row_type(x.dtype));
    const uint8_t* scale = p.scale<const uint8_t>(a[2], x.rows * blocks(x.cols));
    const void* wscale = floats ? (const void*)p.dense<const float>(a[5], at::kFloat, cells) : p.scale<const uint8_t>(a[5], cells);
    if (!p.ok) return 0;
    auto* f = entry<decltype(lasnet_block_product)>(a[0]);
    ENQUEUE(f(&x, scale, offsets, E, W, wscale, floats ? LASNET_F32 : LASNET_E8M0, &out, (uint32_t)flags, st));
  });
}

PyMethodDef methods[] = {
    {"choose_experts", (PyCFunction)(void*)choose_experts, METH_FASTCALL, nullptr},
    {"choose_experts_backward", (PyCFunction)(void*)choose_experts_backward, METH_FASTCALL, nullptr},
    {"balance", (PyCFunction)(void*)balance, METH_FASTCALL, nullptr},
    {"quantize_rows", (PyCFunction)(void*)quantize_rows, METH_FASTCALL, nullptr},
    {"quantize_matrices", (PyCFunction)(void*)quantize_matrices, METH_FASTCALL, nullptr},
    {"block_product", (PyCFunction)(void*)block_product, METH_FASTCALL, nullptr},
    {"norm_rows", (PyCFunction)(void*)norm_rows, METH_FASTCALL, nullptr},
    {"norm_rows_backward", (PyCFunction)(void*)norm_rows_backward, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void*)route, METH_FASTCALL, nullptr},
    {"dispatch_rows", (PyCFunction)(void*)dispatch_rows, METH_FASTCALL, nullptr},
    {"combine_rows", (PyCFunction)(void*)combine_rows, METH_FASTCALL, nullptr},
    {"combine_rows_backward", (PyCFunction)(void*)combine_rows_backward, METH_FASTCALL, nullptr},
    {"expert_product", (PyCFunction)(void*)expert_product, METH_FASTCALL, nullptr},
    {"expert_product_dx", (PyCFunction)(void*)expert_product_dx, METH_FASTCALL, nullptr},
    {"expert_product_dw", (PyCFunction)(void*)expert_product_dw, METH_FASTCALL, nullptr},
    {"masker_ex", (PyCFunction)(void*)masker_ex, METH_FASTCALL, nullptr},
    {"block_packed", (PyCFunction)(void*)block_packed, METH_FASTCALL, nullptr},
    {"block_planned", (PyCFunction)(void*)block_planned, METH_FASTCALL, nullptr},
    {"block_ex", (PyCFunction)(void*)block_ex, METH_FASTCALL, nullptr},
    {"block_dense", (PyCFunction)(void*)block_dense, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  PyObject* torch = PyImport_ImportModule("torch._C");
  if (!torch) return nullptr;
  g_current_device = PyObject_GetAttrString(torch, "_cuda_getDevice");
  g_current_stream = PyObject_GetAttrString(torch, "_cuda_getCurrentRawStream");
  Py_DECREF(torch);
  if (!g_current_device || !g_current_stream) return nullptr;
  return PyModule_Create(&module);
}
