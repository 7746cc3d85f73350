// The short way from Python to the library for the calls that take a dozen microseconds on the device:
// outputs are made and arguments marshalled here instead of in Python (a buffer made from Python takes
// 2 us, a call with its checks some 10).
//
// Nothing is decided here.  A function returns None where anything is not as the plain call has it (a
// dtype, a shape, a stride, another device than the current one, a refusal of the library); its caller
// then goes the long way, which says what is wrong.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "thanos.h"

namespace {

using at::Tensor;

// The library's entry points, given as addresses by bind().
#define ENTRIES(X)                                                                     \
  X(thanos_token_logprobs) X(thanos_token_logprobs_backward) X(thanos_pack_weights)    \
  X(thanos_unpack_weights) X(thanos_pack_activations) X(thanos_unpack_activations)     \
  X(thanos_adapter_forward) X(thanos_adapter_backward) X(thanos_adapter_forward_packed) \
  X(thanos_adapter_backward_packed) X(thanos_adapter_workspace_bytes)                  \
  X(thanos_adapter_packed_workspace_bytes)
#define DECLARE(name) decltype(&::name) p_##name = nullptr;
ENTRIES(DECLARE)
#undef DECLARE

PyObject* packed_weights_type = nullptr;
PyObject* packed_activations_type = nullptr;

constexpr at::ScalarType F32 = at::kFloat, BF16 = at::kBFloat16, I64 = at::kLong, I32 = at::kInt,
                         U8 = at::kByte, I8 = at::kChar;

// One call: the current device, and whether everything so far is as it should be.
struct Call {
  bool ok = true;
  int dev = -1;  // asked for with the first CUDA tensor: without one there may be no device

  const Tensor* tensor(PyObject* o) {
    if (!ok || !THPVariable_Check(o)) {
      ok = false;
      return nullptr;
    }
    const Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && dev < 0) dev = c10::cuda::current_device();
    if (!t.is_cuda() || t.get_device() != dev) ok = false;
    return ok ? &t : nullptr;
  }
  const Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : tensor(o); }
  // a contiguous tensor of this type and shape, as an address
  void* dense(const Tensor* t, at::ScalarType type, at::IntArrayRef shape) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) ok = false;
    return ok ? t->data_ptr() : nullptr;
  }
  // a matrix of `cols` columns and unit inner stride; its leading dimension
  int64_t rows(const Tensor* t, int64_t cols, at::ScalarType type) {
    if (!t || t->dim() != 2 || t->scalar_type() != type || t->size(1) != cols ||
        (t->stride(1) != 1 && cols > 1)) {
      ok = false;
      return 0;
    }
    return t->size(0) > 1 ? t->stride(0) : (cols + 7) / 8 * 8;
  }
  int dtype(const Tensor* t) {
    if (t && t->scalar_type() == F32) return THANOS_F32;
    if (t && t->scalar_type() == BF16) return THANOS_BF16;
    ok = false;
    return 0;
  }
  int64_t number(PyObject* o) {
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  Tensor make(at::IntArrayRef shape, at::ScalarType type) const {
    return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)dev),
                                  std::nullopt);
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }
};

// Makes outputs and launches, without the interpreter's lock: an allocation may wait for the device and a
// launch for room in the stream's queue, which may be for a thread that wants the lock.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
bool done(const F& call) {
  const Unlocked unlocked;
  return call() == THANOS_OK;
}

void* at_or_null(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
PyObject* wrap(const Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }

PyObject* tuple_of(std::initializer_list<Tensor> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  Py_ssize_t i = 0;
  for (const Tensor& t : ts) {
    PyObject* o = r ? wrap(t) : nullptr;
    if (!o) {
      Py_XDECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

#define LONG_WAY() Py_RETURN_NONE
#define ARGUMENTS(n) \
  if (given != (n)) LONG_WAY()

// ------------------------------------------------------------------------------ log probabilities
// Z, target, k
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(3);
  Call c;
  const Tensor *Z = c.tensor(a[0]), *target = c.maybe(a[1]);
  const int64_t k = c.number(a[2]);
  const int dt = c.dtype(Z);
  if (!c.ok || Z->dim() != 2 || k < 0 || k > 64 || (Z->stride(1) != 1 && Z->size(1) > 1)) LONG_WAY();
  const int64_t T = Z->size(0), V = Z->size(1), ld = T > 1 ? Z->stride(0) : std::max<int64_t>(V, 1);
  const void* tp = c.dense(target, I64, {T});
  if (!c.ok) LONG_WAY();
  Tensor logp, top_index, top_logp, stats, entropy;
  if (!done([&] {
        stats = c.make({T, 2}, F32);
        entropy = c.make({T}, F32);
        if (target) logp = c.make({T}, F32);
        if (k > 0) {
          top_index = c.make({T, k}, I64);
          top_logp = c.make({T, k}, F32);
        }
        return p_thanos_token_logprobs(
            (float*)at_or_null(logp), (float*)entropy.data_ptr(), (float*)stats.data_ptr(),
            (int64_t*)at_or_null(top_index), (float*)at_or_null(top_logp), Z->data_ptr(), ld,
            (thanos_dtype_t)dt, (const int64_t*)tp, T, V, (int32_t)k, c.stream());
      }))
    LONG_WAY();
  return tuple_of({logp, entropy, stats, top_index, top_logp});
  END_HANDLE_TH_ERRORS
}

// Z, stats, target, dlogp, entropy, dentropy, top_index, dtop
PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(8);
  Call c;
  const Tensor *Z = c.tensor(a[0]), *stats = c.tensor(a[1]), *target = c.maybe(a[2]),
               *dlogp = c.maybe(a[3]), *entropy = c.maybe(a[4]), *dentropy = c.maybe(a[5]),
               *top = c.maybe(a[6]), *dtop = c.maybe(a[7]);
  const int dt = c.dtype(Z);
  if (!c.ok || Z->dim() != 2 || (Z->stride(1) != 1 && Z->size(1) > 1) || !target != !dlogp ||
      (dentropy && !entropy) || (dtop && (!top || dtop->dim() != 2 || dtop->size(1) == 0)))
    LONG_WAY();
  const int64_t T = Z->size(0), V = Z->size(1), ld = T > 1 ? Z->stride(0) : std::max<int64_t>(V, 1);
  const int64_t k = dtop ? dtop->size(1) : 0;
  const void* ps = c.dense(stats, F32, {T, 2});
  const void* pt = c.dense(target, I64, {T});
  const void* pl = c.dense(dlogp, F32, {T});
  const void* ph = dentropy ? c.dense(entropy, F32, {T}) : nullptr;
  const void* pdh = c.dense(dentropy, F32, {T});
  const void* pi = dtop ? c.dense(top, I64, {T, k}) : nullptr;
  const void* pd = c.dense(dtop, F32, {T, k});
  if (!c.ok) LONG_WAY();
  Tensor out;
  if (!done([&] {
        out = c.make({T, V}, Z->scalar_type());
        return p_thanos_token_logprobs_backward(
            out.data_ptr(), std::max<int64_t>(V, 1), Z->data_ptr(), ld, (thanos_dtype_t)dt,
            (const float*)ps, (const int64_t*)pt, (const float*)pl, (const float*)ph,
            (const float*)pdh, (const int64_t*)pi, (const float*)pd, T, V, (int32_t)k, c.stream());
      }))
    LONG_WAY();
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// ----------------------------------------------------------------------------------------- packing
struct Weights {
  const Tensor *codes = nullptr, *scales = nullptr;
  int64_t group = 0, b = 0, c = 0, ldq = 0;
  // PackedWeights
  void read(Call& k, PyObject* o) {
    if (!k.ok || PyTuple_GET_SIZE(o) != 4) {
      k.ok = false;
      return;
    }
    codes = k.tensor(PyTuple_GET_ITEM(o, 0));
    scales = k.tensor(PyTuple_GET_ITEM(o, 1));
    group = k.number(PyTuple_GET_ITEM(o, 2));
    b = k.number(PyTuple_GET_ITEM(o, 3));
    if (!k.ok) return;
    k.ok = codes->scalar_type() == U8 && codes->dim() == 2 && codes->stride(1) == 1 && b > 0 && b < (1 << 30) &&
           codes->size(1) >= (b + 63) / 64 * 32 && (group == 64 || group == 128);
    if (!k.ok) return;
    c = codes->size(0);
    ldq = c > 1 ? codes->stride(0) : (codes->size(1) + 15) / 16 * 16;
    k.dense(scales, BF16, {(b + group - 1) / group, c});
  }
};
struct Activations {
  const Tensor *codes = nullptr, *exps = nullptr;
  int64_t T = 0, ldc = 0, lde = 0;
  // PackedActivations of b columns
  void read(Call& k, PyObject* o, int64_t b) {
    if (!k.ok || PyTuple_GET_SIZE(o) != 2) {
      k.ok = false;
      return;
    }
    codes = k.tensor(PyTuple_GET_ITEM(o, 0));
    exps = k.tensor(PyTuple_GET_ITEM(o, 1));
    ldc = k.rows(codes, b, I8);
    lde = k.rows(exps, (b + 31) / 32, U8);
    if (!k.ok) return;
    T = codes->size(0);
    k.ok = exps->size(0) == T;
    if (T <= 1) {
      ldc = (b + 15) / 16 * 16;
      lde = (lde + 3) / 4 * 4;
    }
  }
};

// W, group -> codes, scales
PyObject* pack_weights(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(2);
  Call k;
  const Tensor* W = k.tensor(a[0]);
  const int64_t group = k.number(a[1]);
  const int dt = k.dtype(W);
  if (!k.ok || W->dim() != 2 || (group != 64 && group != 128)) LONG_WAY();
  const int64_t c = W->size(0), b = W->size(1), ldw = k.rows(W, b, W->scalar_type());
  if (!k.ok) LONG_WAY();
  const int64_t ldq = (b + 63) / 64 * 32;
  Tensor codes, scales;
  if (!done([&] {
        codes = k.make({c, ldq}, U8);
        scales = k.make({(b + group - 1) / group, c}, BF16);
        return p_thanos_pack_weights((uint8_t*)codes.data_ptr(), ldq, scales.data_ptr(),
                                     W->data_ptr(), ldw, (thanos_dtype_t)dt, c, b, (int32_t)group,
                                     k.stream());
      }))
    LONG_WAY();
  return tuple_of({codes, scales});
  END_HANDLE_TH_ERRORS
}

bool dtype_of(PyObject* o, at::ScalarType& type) {
  if (!THPDtype_Check(o)) return false;
  type = reinterpret_cast<THPDtype*>(o)->scalar_type;
  return type == F32 || type == BF16;
}

// PackedWeights, dtype
PyObject* unpack_weights(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(2);
  Call k;
  at::ScalarType type;
  if ((PyObject*)Py_TYPE(a[0]) != packed_weights_type || !dtype_of(a[1], type)) LONG_WAY();
  Weights w;
  w.read(k, a[0]);
  if (!k.ok) LONG_WAY();
  Tensor out;
  if (!done([&] {
        out = k.make({w.c, w.b}, type);
        return p_thanos_unpack_weights(out.data_ptr(), (w.b + 7) / 8 * 8,
                                       type == F32 ? THANOS_F32 : THANOS_BF16,
                                       (const uint8_t*)w.codes->data_ptr(), w.ldq,
                                       w.scales->data_ptr(), w.c, w.b, (int32_t)w.group, k.stream());
      }))
    LONG_WAY();
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// X -> codes, exps
PyObject* pack_activations(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(1);
  Call k;
  const Tensor* X = k.tensor(a[0]);
  const int dt = k.dtype(X);
  if (!k.ok || X->dim() != 2) LONG_WAY();
  const int64_t T = X->size(0), b = X->size(1), ldx = k.rows(X, b, X->scalar_type());
  if (!k.ok) LONG_WAY();
  const int64_t groups = (b + 31) / 32, ldc = (b + 15) / 16 * 16, lde = (groups + 3) / 4 * 4;
  Tensor codes, exps;
  if (!done([&] {
        codes = k.make({T, ldc}, I8);
        exps = k.make({T, lde}, U8);
        return p_thanos_pack_activations((int8_t*)codes.data_ptr(), ldc, (uint8_t*)exps.data_ptr(),
                                         lde, X->data_ptr(), ldx, (thanos_dtype_t)dt, T, b,
                                         k.stream());
      }))
    LONG_WAY();
  return tuple_of({ldc == b ? codes : codes.narrow(1, 0, b),
                   lde == groups ? exps : exps.narrow(1, 0, groups)});
  END_HANDLE_TH_ERRORS
}

// PackedActivations, dtype
PyObject* unpack_activations(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(2);
  Call k;
  at::ScalarType type;
  if ((PyObject*)Py_TYPE(a[0]) != packed_activations_type || !dtype_of(a[1], type)) LONG_WAY();
  const Tensor* codes = PyTuple_GET_SIZE(a[0]) == 2 ? k.tensor(PyTuple_GET_ITEM(a[0], 0)) : nullptr;
  if (!codes || codes->dim() != 2) LONG_WAY();
  const int64_t b = codes->size(1);
  Activations x;
  x.read(k, a[0], b);
  if (!k.ok) LONG_WAY();
  Tensor out;
  if (!done([&] {
        out = k.make({x.T, b}, type);
        return p_thanos_unpack_activations(out.data_ptr(), (b + 7) / 8 * 8,
                                           type == F32 ? THANOS_F32 : THANOS_BF16,
                                           (const int8_t*)x.codes->data_ptr(), x.ldc,
                                           (const uint8_t*)x.exps->data_ptr(), x.lde, x.T, b,
                                           k.stream());
      }))
    LONG_WAY();
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------ adapted projection
struct Projection {
  const Tensor* W = nullptr;
  Weights packed;
  bool is_packed = false;
  const void *A = nullptr, *B = nullptr, *index = nullptr, *scale = nullptr;
  int64_t T = 0, c = 0, b = 0, n = 0, r = 0, ldw = 0;
  int dt = 0;
  // X (or dY), W or PackedWeights, A, B, index, scale
  void read(Call& k, const Tensor* X, PyObject* const* a) {
    dt = k.dtype(X);
    if (!k.ok) return;
    T = X->size(0);
    is_packed = (PyObject*)Py_TYPE(a[0]) == packed_weights_type;
    if (is_packed) {
      packed.read(k, a[0]);
      c = packed.c;
      b = packed.b;
      ldw = packed.ldq;
    } else {
      W = k.tensor(a[0]);
      if (!k.ok || W->dim() != 2) {
        k.ok = false;
        return;
      }
      c = W->size(0);
      b = W->size(1);
      ldw = k.rows(W, b, X->scalar_type());
    }
    const Tensor *tA = k.maybe(a[1]), *tB = k.maybe(a[2]), *ti = k.maybe(a[3]), *ts = k.maybe(a[4]);
    if (!k.ok) return;
    if (!tA) {
      k.ok = !tB && !ti && !ts;
      return;
    }
    if (tA->dim() != 3 || !tB || !ti || !ts) {
      k.ok = false;
      return;
    }
    n = tA->size(0);
    r = tA->size(1);
    A = k.dense(tA, X->scalar_type(), {n, r, b});
    B = k.dense(tB, X->scalar_type(), {n, c, r});
    index = k.dense(ti, I32, {T});
    scale = k.dense(ts, F32, {n});
  }
  void* weights() const { return is_packed ? packed.codes->data_ptr() : W->data_ptr(); }
};

// X, W, A, B, index, scale -> Y, V
PyObject* adapter_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(6);
  Call k;
  const Tensor* X = k.tensor(a[0]);
  if (!k.ok || X->dim() != 2) LONG_WAY();
  Projection p;
  p.read(k, X, a + 1);
  if (!k.ok) LONG_WAY();
  const int64_t ldx = k.rows(X, p.b, X->scalar_type());
  if (!k.ok) LONG_WAY();
  const thanos_dtype_t dt = (thanos_dtype_t)p.dt;
  const size_t need =
      p.is_packed
          ? p_thanos_adapter_packed_workspace_bytes(0, 1, 0, p.T, p.c, p.b, p.n, (int32_t)p.r, dt)
          : p_thanos_adapter_workspace_bytes(0, p.T, p.c, p.b, p.n, (int32_t)p.r, dt);
  if (need == 0) LONG_WAY();
  Tensor Y, V;
  const int64_t ldy = p.T > 1 ? p.c : (p.c + 7) / 8 * 8;
  if (!done([&] {
        Y = k.make({p.T, p.c}, X->scalar_type());
        if (p.n > 0) V = k.make({p.T, p.r}, F32);
        const Tensor ws = k.make({(int64_t)need}, U8);
        return p.is_packed
                   ? p_thanos_adapter_forward_packed(
                         Y.data_ptr(), ldy, (float*)at_or_null(V), X->data_ptr(), ldx,
                         (const uint8_t*)p.weights(), p.ldw, p.packed.scales->data_ptr(),
                         (int32_t)p.packed.group, p.A, p.B, (const int32_t*)p.index,
                         (const float*)p.scale, dt, p.T, p.c, p.b, p.n, (int32_t)p.r, ws.data_ptr(),
                         need, k.stream())
                   : p_thanos_adapter_forward(Y.data_ptr(), ldy, (float*)at_or_null(V),
                                              X->data_ptr(), ldx, p.weights(), p.ldw, p.A, p.B,
                                              (const int32_t*)p.index, (const float*)p.scale, dt,
                                              p.T, p.c, p.b, p.n, (int32_t)p.r, ws.data_ptr(), need,
                                              k.stream());
      }))
    LONG_WAY();
  return tuple_of({Y, V});
  END_HANDLE_TH_ERRORS
}

// dY, X, V, W, A, B, index, scale, need_dx, need_grads -> dX, dA, dB
PyObject* adapter_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
  HANDLE_TH_ERRORS
  ARGUMENTS(10);
  Call k;
  const Tensor* dY = k.tensor(a[0]);
  if (!k.ok || dY->dim() != 2) LONG_WAY();
  Projection p;
  p.read(k, dY, a + 3);
  if (!k.ok) LONG_WAY();
  const int64_t lddy = k.rows(dY, p.c, dY->scalar_type());
  const bool need_dx = a[8] == Py_True, grads = a[9] == Py_True && p.n > 0;
  const Tensor* X = nullptr;
  const void* V = nullptr;
  Activations x;
  int64_t ldx = 0;
  const bool x_packed = grads && (PyObject*)Py_TYPE(a[1]) == packed_activations_type;
  if (grads) {
    if (x_packed) {
      x.read(k, a[1], p.b);
      if (k.ok && x.T != p.T) k.ok = false;
      ldx = x.ldc;
    } else {
      X = k.tensor(a[1]);
      ldx = k.rows(X, p.b, dY->scalar_type());
      if (k.ok && X->size(0) != p.T) k.ok = false;
    }
    V = k.dense(k.tensor(a[2]), F32, {p.T, p.r});
  }
  if (!k.ok) LONG_WAY();
  const thanos_dtype_t dt = (thanos_dtype_t)p.dt;
  const bool packed = p.is_packed || x_packed;
  const size_t need =
      packed ? p_thanos_adapter_packed_workspace_bytes(1, p.is_packed && (need_dx || dt == THANOS_F32),
                                                       x_packed, p.T, p.c, p.b, p.n, (int32_t)p.r, dt)
             : p_thanos_adapter_workspace_bytes(1, p.T, p.c, p.b, p.n, (int32_t)p.r, dt);
  if (need == 0) LONG_WAY();
  Tensor dX, dA, dB;
  const int64_t lddx = need_dx ? (p.T > 1 ? p.b : (p.b + 7) / 8 * 8) : 0;
  void* xp = x_packed ? x.codes->data_ptr() : X ? X->data_ptr() : nullptr;
  if (!done([&] {
        if (need_dx) dX = k.make({p.T, p.b}, dY->scalar_type());
        if (grads) {
          dA = k.make({p.n, p.r, p.b}, F32);
          dB = k.make({p.n, p.c, p.r}, F32);
        }
        const Tensor ws = k.make({(int64_t)need}, U8);
        return packed
                   ? p_thanos_adapter_backward_packed(
                         at_or_null(dX), lddx, (float*)at_or_null(dA), (float*)at_or_null(dB), 0,
                         dY->data_ptr(), lddy, xp, ldx,
                         x_packed ? (const uint8_t*)x.exps->data_ptr() : nullptr, x.lde,
                         (const float*)V, p.weights(), p.ldw,
                         p.is_packed ? p.packed.scales->data_ptr() : nullptr,
                         (int32_t)p.packed.group, p.A, p.B, (const int32_t*)p.index,
                         (const float*)p.scale, dt, p.T, p.c, p.b, p.n, (int32_t)p.r, ws.data_ptr(),
                         need, k.stream())
                   : p_thanos_adapter_backward(
                         at_or_null(dX), lddx, (float*)at_or_null(dA), (float*)at_or_null(dB), 0,
                         dY->data_ptr(), lddy, xp, ldx, (const float*)V, p.weights(), p.ldw, p.A,
                         p.B, (const int32_t*)p.index, (const float*)p.scale, dt, p.T, p.c, p.b, p.n,
                         (int32_t)p.r, ws.data_ptr(), need, k.stream());
      }))
    LONG_WAY();
  return tuple_of({dX, dA, dB});
  END_HANDLE_TH_ERRORS
}

// bind(PackedWeights, PackedActivations, {entry: address})
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t given) {
  if (given != 3 || !PyDict_Check(a[2])) {
    PyErr_SetString(PyExc_TypeError, "bind(PackedWeights, PackedActivations, addresses)");
    return nullptr;
  }
#define TAKE(name)                                                            \
  {                                                                           \
    PyObject* v = PyDict_GetItemString(a[2], #name);                          \
    void* p = v ? PyLong_AsVoidPtr(v) : nullptr;                              \
    if (!p) {                                                                 \
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, #name);          \
      return nullptr;                                                         \
    }                                                                         \
    p_##name = reinterpret_cast<decltype(&::name)>(p);                        \
  }
  ENTRIES(TAKE)
#undef TAKE
  packed_weights_type = Py_NewRef(a[0]);
  packed_activations_type = Py_NewRef(a[1]);
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(token_logprobs), METHOD(token_logprobs_backward),
                         METHOD(pack_weights), METHOD(unpack_weights), METHOD(pack_activations),
                         METHOD(unpack_activations), METHOD(adapter_forward),
                         METHOD(adapter_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr,
                      nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  PyObject* m = PyModule_Create(&module);
  // classes of another torch have other layouts, though their symbols may be found
  if (m && PyModule_AddStringConstant(m, "built_for", THANOS_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
