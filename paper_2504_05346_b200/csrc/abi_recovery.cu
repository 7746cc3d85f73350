// extern "C" entry points of the recovery operators: argument checks and dispatch.
#include <math.h>

#include "packed.cuh"
#include "recovery.cuh"

using namespace thanos;

namespace {

constexpr int64_t MAX_FEATURES_IN = 65536;
constexpr int64_t MAX_FEATURES_OUT = 1 << 20;
constexpr int64_t MAX_TOKENS = 1 << 24;
constexpr int64_t MAX_ADAPTERS = 1 << 20;
constexpr int MAX_RANK = 128;
constexpr int64_t MAX_TILES = 1 << 27;

// index and scale are read one value at a time: a slice of a batch's index is taken as it is
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool known_dtype(thanos_dtype_t d) { return d == THANOS_F32 || d == THANOS_BF16; }

thanos_status_t adapter_shape(int64_t T, int64_t c, int64_t b, int64_t n, int32_t r,
                              thanos_dtype_t dtype) {
  if (!known_dtype(dtype)) return THANOS_ERR_DTYPE;
  if (b < 8 || b > MAX_FEATURES_IN || b % 8 != 0 || c < 1 || c > MAX_FEATURES_OUT || T < 0 ||
      T > MAX_TOKENS || n < 0 || n > MAX_ADAPTERS)
    return THANOS_ERR_SHAPE;
  if (n > 0 && (r < 1 || r > MAX_RANK)) return THANOS_ERR_SHAPE;
  // what a launch's grid holds, with the narrowest tiles
  int64_t rows = c > b ? c : b;
  if (n > 0 && n * r > rows) rows = n * r;
  if (ceil_div(rows, 128) * ceil_div(T, 32) > MAX_TILES) return THANOS_ERR_SHAPE;
  return THANOS_OK;
}

thanos_status_t orthogonal_shape(int64_t batch, int64_t m, int64_t n) {
  if (batch < 0 || batch > 65535 || m < 1 || m > 65536 || n < 1 || n > 65536)
    return THANOS_ERR_SHAPE;
  return THANOS_OK;
}

thanos_status_t orthogonal_common(OrthogonalArgs& a, const void* G, thanos_dtype_t gdtype,
                                  int64_t batch, int64_t m, int64_t n, const float* coef,
                                  int32_t steps, float eps) {
  if ((!G && batch != 0) || !coef) return THANOS_ERR_INVALID_ARG;
  if (!known_dtype(gdtype)) return THANOS_ERR_DTYPE;
  THANOS_TRY(orthogonal_shape(batch, m, n));
  if (steps < 1 || steps > 32 || !(eps >= 0.f) || !isfinite(eps)) return THANOS_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i) {
    if (!isfinite(coef[i])) return THANOS_ERR_INVALID_ARG;
    a.coef[i] = coef[i];
  }
  if (!aligned16(G)) return THANOS_ERR_ALIGNMENT;
  a.G = G;
  a.gdtype = gdtype;
  a.batch = batch;
  a.m = m;
  a.n = n;
  a.steps = steps;
  a.eps = eps;
  return THANOS_OK;
}

thanos_status_t orthogonal_run(const OrthogonalArgs& a, void* workspace, size_t ws_bytes,
                               void* stream) {
  if (!aligned16(workspace)) return THANOS_ERR_ALIGNMENT;
  if (!workspace || ws_bytes < orthogonal_workspace_bytes(a.batch, a.m, a.n))
    return THANOS_ERR_WORKSPACE;
  if (a.batch == 0) return THANOS_OK;
  return orthogonal_impl(a, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

// ---- packed operands
constexpr int64_t PACKED_LINE = 64;   // columns: rows of what is unpacked start on whole lines

thanos_status_t packed_weights_ok(const PackedWeights& w, int64_t b) {
  if (w.group != 64 && w.group != 128) return THANOS_ERR_SHAPE;
  if (w.ldq < (int64_t)round_up((size_t)b, 64) / 2) return THANOS_ERR_SHAPE;
  if (w.ldq % 16 || !aligned16(w.codes) || (reinterpret_cast<uintptr_t>(w.scales) & 1u))
    return THANOS_ERR_ALIGNMENT;
  return THANOS_OK;
}

thanos_status_t packed_activations_ok(const PackedActivations& x, int64_t b) {
  if (x.ldc < b || x.lde < ceil_div(b, ACT_GROUP)) return THANOS_ERR_SHAPE;
  if (x.ldc % 16 || x.lde % 4 || !aligned16(x.codes) || !aligned4(x.exps))
    return THANOS_ERR_ALIGNMENT;
  return THANOS_OK;
}

// Room for packed weights in bf16, behind what the call needs itself (fp32 calls have room for a plane).
size_t packed_extra_bytes(int64_t c, int64_t b, thanos_dtype_t dtype) {
  return dtype == THANOS_BF16 ? round_up((size_t)c * round_up((size_t)b, PACKED_LINE) * 2, 256) : 0;
}

// Where W is: as it is, or packed (W null).
struct Weights {
  const void* W;
  int64_t ldw;
  PackedWeights packed;
  bool is_packed;
};

thanos_status_t weights_ok(const Weights& w, int64_t b) {
  if (w.is_packed) return packed_weights_ok(w.packed, b);
  if (w.ldw < b) return THANOS_ERR_SHAPE;
  if (w.ldw % 8 || !aligned16(w.W)) return THANOS_ERR_ALIGNMENT;
  return THANOS_OK;
}

bool weights_there(const Weights& w) {
  return w.is_packed ? w.packed.codes && w.packed.scales : w.W != nullptr;
}

thanos_status_t forward_call(void* Y, int64_t ldy, float* V, const void* X, int64_t ldx,
                             const Weights& w, const void* A, const void* B, const int32_t* index,
                             const float* scale, thanos_dtype_t dtype, int64_t n_tok, int64_t c,
                             int64_t b, int64_t n_adapters, int32_t r, void* workspace,
                             size_t ws_bytes, cudaStream_t stream) {
  if (!weights_there(w) || (n_tok > 0 && (!Y || !X))) return THANOS_ERR_INVALID_ARG;
  if (n_adapters > 0 && (!A || !B || !scale || (n_tok > 0 && !index)))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, c, b, n_adapters, r, dtype));
  if (ldy < c || ldx < b || (!w.is_packed && w.ldw < b)) return THANOS_ERR_SHAPE;
  if (ldx % 8) return THANOS_ERR_ALIGNMENT;
  THANOS_TRY(weights_ok(w, b));
  if (!aligned16(Y) || !aligned16(V) || !aligned16(X) || !aligned16(A) || !aligned16(B) ||
      !aligned4(index) || !aligned4(scale) || !aligned16(workspace))
    return THANOS_ERR_ALIGNMENT;
  const size_t need =
      w.is_packed ? thanos_adapter_packed_workspace_bytes(0, 1, 0, n_tok, c, b, n_adapters, r, dtype)
                  : thanos_adapter_workspace_bytes(0, n_tok, c, b, n_adapters, r, dtype);
  if (!workspace || ws_bytes < need) return THANOS_ERR_WORKSPACE;
  if (n_tok == 0) {
    THANOS_CUDA(cudaMemsetAsync(workspace, 0, 16, stream));
    return THANOS_OK;
  }
  AdapterArgs a;
  a.out = Y;
  a.ldo = ldy;
  a.in = X;
  a.ldi = ldx;
  a.W = w.W;
  a.ldw = w.ldw;
  a.A = A;
  a.B = B;
  a.index = index;
  a.scale = scale;
  a.V = n_adapters > 0 ? V : nullptr;
  a.dtype = dtype;
  a.T = n_tok;
  a.c = c;
  a.b = b;
  a.n = n_adapters;
  a.r = n_adapters > 0 ? r : 1;
  if (w.is_packed) {
    if (packed_few_tokens(a)) return packed_forward_few(a, w.packed, workspace, stream);
    // many tokens: the weights are unpacked once, the product is theirs
    a.packed = &w.packed;
    ws_bytes = need - packed_extra_bytes(c, b, dtype);
    a.unpacked = static_cast<char*>(workspace) + ws_bytes;
    a.ldw = (int64_t)round_up((size_t)b, PACKED_LINE);
  }
  return adapter_forward_impl(a, workspace, ws_bytes, stream);
}

thanos_status_t backward_call(void* dX, int64_t lddx, float* dA, float* dB, int32_t accumulate,
                              const void* dY, int64_t lddy, const void* X, int64_t ldx,
                              const PackedActivations& x8, bool x_packed, const float* V,
                              const Weights& w, const void* A, const void* B, const int32_t* index,
                              const float* scale, thanos_dtype_t dtype, int64_t n_tok, int64_t c,
                              int64_t b, int64_t n_adapters, int32_t r, void* workspace,
                              size_t ws_bytes, cudaStream_t stream) {
  const bool grads = dA != nullptr || dB != nullptr;
  const bool x_there = x_packed ? x8.codes && x8.exps : X != nullptr;
  if (!weights_there(w) || (n_tok > 0 && !dY)) return THANOS_ERR_INVALID_ARG;
  if (grads && (!dA || !dB || n_adapters == 0 || (n_tok > 0 && (!x_there || !V))))
    return THANOS_ERR_INVALID_ARG;
  if (n_adapters > 0 && (!A || !B || !scale || (n_tok > 0 && !index)))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, c, b, n_adapters, r, dtype));
  if (lddy < c || (!w.is_packed && w.ldw < b) || (dX && lddx < b) || (grads && !x_packed && ldx < b))
    return THANOS_ERR_SHAPE;
  if (grads && !x_packed && ldx % 8) return THANOS_ERR_ALIGNMENT;
  if (grads && x_packed) THANOS_TRY(packed_activations_ok(x8, b));
  THANOS_TRY(weights_ok(w, b));
  if (!aligned16(dX) || !aligned16(dA) || !aligned16(dB) || !aligned16(dY) || !aligned16(V) ||
      !aligned16(X) || !aligned16(A) || !aligned16(B) || !aligned4(index) || !aligned4(scale) ||
      !aligned16(workspace))
    return THANOS_ERR_ALIGNMENT;
  const size_t need =
      w.is_packed
          ? thanos_adapter_packed_workspace_bytes(1, 1, x_packed, n_tok, c, b, n_adapters, r, dtype) -
                (dX ? 0 : packed_extra_bytes(c, b, dtype))  // without dX nothing is unpacked
          : thanos_adapter_workspace_bytes(1, n_tok, c, b, n_adapters, r, dtype);
  if (!workspace || ws_bytes < need) return THANOS_ERR_WORKSPACE;
  if (n_tok == 0) {
    THANOS_CUDA(cudaMemsetAsync(workspace, 0, 16, stream));
    if (grads && !accumulate) {
      const size_t nr = (size_t)n_adapters * (size_t)r;
      THANOS_CUDA(cudaMemsetAsync(dA, 0, nr * (size_t)b * 4, stream));
      THANOS_CUDA(cudaMemsetAsync(dB, 0, nr * (size_t)c * 4, stream));
    }
    return THANOS_OK;
  }
  AdapterArgs a;
  a.out = dX;
  a.ldo = lddx;
  a.in = dY;
  a.ldi = lddy;
  a.X = X;
  a.ldx = ldx;
  a.W = w.W;
  a.ldw = w.ldw;
  a.A = A;
  a.B = B;
  a.index = index;
  a.scale = scale;
  a.Vin = V;
  a.dA = dA;
  a.dB = dB;
  a.accumulate = accumulate ? 1 : 0;
  a.dtype = dtype;
  a.T = n_tok;
  a.c = c;
  a.b = b;
  a.n = n_adapters;
  a.r = n_adapters > 0 ? r : 1;
  if (x_packed) {
    a.X8 = x8.codes;
    a.ldx8 = x8.ldc;
    a.exps = x8.exps;
    a.lde = x8.lde;
  }
  if (w.is_packed) {
    a.packed = &w.packed;
    ws_bytes = need;
    if (dX) {
      ws_bytes -= packed_extra_bytes(c, b, dtype);
      a.unpacked = static_cast<char*>(workspace) + ws_bytes;
    }
    a.ldw = (int64_t)round_up((size_t)b, PACKED_LINE);
  }
  return adapter_backward_impl(a, workspace, ws_bytes, stream);
}

}  // namespace

extern "C" {

size_t thanos_adapter_workspace_bytes(int32_t backward, int64_t n_tok, int64_t c, int64_t b,
                                      int64_t n_adapters, int32_t r, thanos_dtype_t dtype) {
  if (adapter_shape(n_tok, c, b, n_adapters, r, dtype) != THANOS_OK) return 0;
  return adapter_workspace_bytes(backward != 0, n_tok, c, b, n_adapters, n_adapters > 0 ? r : 1,
                                 dtype, false);
}

thanos_status_t thanos_adapter_forward(void* Y, int64_t ldy, float* V, const void* X, int64_t ldx,
                                       const void* W, int64_t ldw, const void* A, const void* B,
                                       const int32_t* index, const float* scale,
                                       thanos_dtype_t dtype, int64_t n_tok, int64_t c, int64_t b,
                                       int64_t n_adapters, int32_t r, void* workspace,
                                       size_t ws_bytes, void* stream) {
  return forward_call(Y, ldy, V, X, ldx, Weights{W, ldw, PackedWeights{}, false}, A, B, index, scale,
                      dtype, n_tok, c, b, n_adapters, r, workspace, ws_bytes,
                      static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_adapter_backward(void* dX, int64_t lddx, float* dA, float* dB,
                                        int32_t accumulate, const void* dY, int64_t lddy,
                                        const void* X, int64_t ldx, const float* V, const void* W,
                                        int64_t ldw, const void* A, const void* B,
                                        const int32_t* index, const float* scale,
                                        thanos_dtype_t dtype, int64_t n_tok, int64_t c, int64_t b,
                                        int64_t n_adapters, int32_t r, void* workspace,
                                        size_t ws_bytes, void* stream) {
  return backward_call(dX, lddx, dA, dB, accumulate, dY, lddy, X, ldx, PackedActivations{}, false, V,
                       Weights{W, ldw, PackedWeights{}, false}, A, B, index, scale, dtype, n_tok, c, b,
                       n_adapters, r, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

size_t thanos_adapter_packed_workspace_bytes(int32_t backward, int32_t packed_w, int32_t,
                                             int64_t n_tok, int64_t c, int64_t b,
                                             int64_t n_adapters, int32_t r, thanos_dtype_t dtype) {
  if (adapter_shape(n_tok, c, b, n_adapters, r, dtype) != THANOS_OK) return 0;
  AdapterArgs a;
  a.T = n_tok;
  a.c = c;
  a.b = b;
  a.n = n_adapters;
  a.r = n_adapters > 0 ? r : 1;
  a.dtype = dtype;
  if (!backward && packed_w && packed_few_tokens(a)) return packed_few_workspace_bytes(n_tok, a.r);
  return round_up(adapter_workspace_bytes(backward != 0, n_tok, c, b, n_adapters, a.r, dtype, packed_w != 0),
                  256) +
         (packed_w ? packed_extra_bytes(c, b, dtype) : 0);
}

thanos_status_t thanos_adapter_forward_packed(void* Y, int64_t ldy, float* V, const void* X,
                                              int64_t ldx, const uint8_t* w_codes, int64_t ldq,
                                              const void* w_scales, int32_t group, const void* A,
                                              const void* B, const int32_t* index,
                                              const float* scale, thanos_dtype_t dtype,
                                              int64_t n_tok, int64_t c, int64_t b,
                                              int64_t n_adapters, int32_t r, void* workspace,
                                              size_t ws_bytes, void* stream) {
  const PackedWeights w{w_codes, ldq, static_cast<const __nv_bfloat16*>(w_scales), group};
  return forward_call(Y, ldy, V, X, ldx, Weights{nullptr, 0, w, true}, A, B, index, scale, dtype,
                      n_tok, c, b, n_adapters, r, workspace, ws_bytes,
                      static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_adapter_backward_packed(void* dX, int64_t lddx, float* dA, float* dB,
                                               int32_t accumulate, const void* dY, int64_t lddy,
                                               const void* X, int64_t ldx, const uint8_t* x_exps,
                                               int64_t lde, const float* V, const void* W,
                                               int64_t ldw, const void* w_scales, int32_t group,
                                               const void* A, const void* B, const int32_t* index,
                                               const float* scale, thanos_dtype_t dtype,
                                               int64_t n_tok, int64_t c, int64_t b,
                                               int64_t n_adapters, int32_t r, void* workspace,
                                               size_t ws_bytes, void* stream) {
  Weights w{W, ldw, PackedWeights{}, false};
  if (w_scales)
    w = Weights{nullptr, 0,
                PackedWeights{static_cast<const uint8_t*>(W), ldw,
                              static_cast<const __nv_bfloat16*>(w_scales), group},
                true};
  PackedActivations x8;
  if (x_exps) x8 = PackedActivations{static_cast<const int8_t*>(X), ldx, x_exps, lde};
  return backward_call(dX, lddx, dA, dB, accumulate, dY, lddy, x_exps ? nullptr : X, ldx, x8,
                       x_exps != nullptr, V, w, A, B, index, scale, dtype, n_tok, c, b, n_adapters, r,
                       workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_pack_weights(uint8_t* codes, int64_t ldq, void* scales, const void* W,
                                    int64_t ldw, thanos_dtype_t dtype, int64_t c, int64_t b,
                                    int32_t group, void* stream) {
  if (!codes || !scales || !W) return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(0, c, b, 0, 0, dtype));
  const PackedWeights w{codes, ldq, static_cast<const __nv_bfloat16*>(scales), group};
  if (ldw < b) return THANOS_ERR_SHAPE;
  THANOS_TRY(packed_weights_ok(w, b));
  if (ldw % 8 || !aligned16(W)) return THANOS_ERR_ALIGNMENT;
  return pack_weights(codes, ldq, static_cast<__nv_bfloat16*>(scales), W, ldw, dtype, c, b, group,
                      static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_unpack_weights(void* W, int64_t ldw, thanos_dtype_t dtype,
                                      const uint8_t* codes, int64_t ldq, const void* scales,
                                      int64_t c, int64_t b, int32_t group, void* stream) {
  if (!codes || !scales || !W) return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(0, c, b, 0, 0, dtype));
  const PackedWeights w{codes, ldq, static_cast<const __nv_bfloat16*>(scales), group};
  if (ldw < b) return THANOS_ERR_SHAPE;
  THANOS_TRY(packed_weights_ok(w, b));
  if (ldw % 8 || !aligned16(W)) return THANOS_ERR_ALIGNMENT;
  return unpack_weights(W, ldw, dtype, w, c, b, static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_pack_activations(int8_t* codes, int64_t ldc, uint8_t* exps, int64_t lde,
                                        const void* X, int64_t ldx, thanos_dtype_t dtype,
                                        int64_t n_tok, int64_t b, void* stream) {
  if (n_tok > 0 && (!codes || !exps || !X)) return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, 1, b, 0, 0, dtype));
  if (ldx < b) return THANOS_ERR_SHAPE;
  THANOS_TRY(packed_activations_ok(PackedActivations{codes, ldc, exps, lde}, b));
  if (ldx % 8 || !aligned16(X)) return THANOS_ERR_ALIGNMENT;
  if (n_tok == 0) return THANOS_OK;
  return pack_activations(codes, ldc, exps, lde, X, ldx, dtype, n_tok, b,
                          static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_unpack_activations(void* X, int64_t ldx, thanos_dtype_t dtype,
                                          const int8_t* codes, int64_t ldc, const uint8_t* exps,
                                          int64_t lde, int64_t n_tok, int64_t b, void* stream) {
  if (n_tok > 0 && (!codes || !exps || !X)) return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, 1, b, 0, 0, dtype));
  if (ldx < b) return THANOS_ERR_SHAPE;
  THANOS_TRY(packed_activations_ok(PackedActivations{codes, ldc, exps, lde}, b));
  if (ldx % 8 || !aligned16(X)) return THANOS_ERR_ALIGNMENT;
  if (n_tok == 0) return THANOS_OK;
  return unpack_activations(X, ldx, dtype, codes, ldc, exps, lde, n_tok, b,
                            static_cast<cudaStream_t>(stream));
}

size_t thanos_orthogonal_workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  if (orthogonal_shape(batch, m, n) != THANOS_OK) return 0;
  return orthogonal_workspace_bytes(batch, m, n);
}

thanos_status_t thanos_orthogonalise(void* O, const void* G, thanos_dtype_t gdtype, int64_t batch,
                                     int64_t m, int64_t n, const float* coef, int32_t steps,
                                     float eps, void* workspace, size_t ws_bytes, void* stream) {
  OrthogonalArgs a;
  if (!O && batch != 0) return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(orthogonal_common(a, G, gdtype, batch, m, n, coef, steps, eps));
  if (!aligned16(O)) return THANOS_ERR_ALIGNMENT;
  a.O = static_cast<__nv_bfloat16*>(O);
  return orthogonal_run(a, workspace, ws_bytes, stream);
}

thanos_status_t thanos_orthogonal_step(void* W_out, const void* W_in, thanos_dtype_t wdtype,
                                       float* M_out, const float* M_in, const void* G,
                                       thanos_dtype_t gdtype, const uint8_t* mask, int64_t batch,
                                       int64_t m, int64_t n, float lr, float gain, float momentum,
                                       int32_t nesterov, float weight_decay, const float* coef,
                                       int32_t steps, float eps, void* workspace, size_t ws_bytes,
                                       void* stream) {
  OrthogonalArgs a;
  if (batch != 0 && (!W_out || !W_in || !M_out || !M_in)) return THANOS_ERR_INVALID_ARG;
  if (!known_dtype(wdtype)) return THANOS_ERR_DTYPE;
  THANOS_TRY(orthogonal_common(a, G, gdtype, batch, m, n, coef, steps, eps));
  if (!isfinite(lr) || !isfinite(gain) || !isfinite(momentum) || !isfinite(weight_decay))
    return THANOS_ERR_INVALID_ARG;
  if (!aligned16(W_out) || !aligned16(W_in) || !aligned16(M_out) || !aligned16(M_in) ||
      !aligned16(mask))
    return THANOS_ERR_ALIGNMENT;
  a.W_out = W_out;
  a.W_in = W_in;
  a.wdtype = wdtype;
  a.M_out = M_out;
  a.M_in = M_in;
  a.mask = mask;
  a.keep = (float)(1.0 - (double)lr * (double)weight_decay);
  a.rate = (float)((double)lr * (double)gain);
  a.momentum = momentum;
  a.nesterov = nesterov ? 1 : 0;
  return orthogonal_run(a, workspace, ws_bytes, stream);
}

}  // extern "C"
