// extern "C" entry points of the recovery operators: argument checks and dispatch.
#include <math.h>

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

}  // namespace

extern "C" {

size_t thanos_adapter_workspace_bytes(int32_t backward, int64_t n_tok, int64_t c, int64_t b,
                                      int64_t n_adapters, int32_t r, thanos_dtype_t dtype) {
  if (adapter_shape(n_tok, c, b, n_adapters, r, dtype) != THANOS_OK) return 0;
  return adapter_workspace_bytes(backward != 0, n_tok, c, b, n_adapters, n_adapters > 0 ? r : 1,
                                 dtype);
}

thanos_status_t thanos_adapter_forward(void* Y, int64_t ldy, float* V, const void* X, int64_t ldx,
                                       const void* W, int64_t ldw, const void* A, const void* B,
                                       const int32_t* index, const float* scale,
                                       thanos_dtype_t dtype, int64_t n_tok, int64_t c, int64_t b,
                                       int64_t n_adapters, int32_t r, void* workspace,
                                       size_t ws_bytes, void* stream) {
  if (!W || (n_tok > 0 && (!Y || !X))) return THANOS_ERR_INVALID_ARG;
  if (n_adapters > 0 && (!A || !B || !scale || (n_tok > 0 && !index)))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, c, b, n_adapters, r, dtype));
  if (ldy < c || ldx < b || ldw < b) return THANOS_ERR_SHAPE;
  if (ldx % 8 || ldw % 8) return THANOS_ERR_ALIGNMENT;
  if (!aligned16(Y) || !aligned16(V) || !aligned16(X) || !aligned16(W) || !aligned16(A) ||
      !aligned16(B) || !aligned4(index) || !aligned4(scale) || !aligned16(workspace))
    return THANOS_ERR_ALIGNMENT;
  if (!workspace ||
      ws_bytes < thanos_adapter_workspace_bytes(0, n_tok, c, b, n_adapters, r, dtype))
    return THANOS_ERR_WORKSPACE;
  if (n_tok == 0) {
    THANOS_CUDA(cudaMemsetAsync(workspace, 0, 16, static_cast<cudaStream_t>(stream)));
    return THANOS_OK;
  }
  AdapterArgs a;
  a.out = Y;
  a.ldo = ldy;
  a.in = X;
  a.ldi = ldx;
  a.W = W;
  a.ldw = ldw;
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
  return adapter_forward_impl(a, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_adapter_backward(void* dX, int64_t lddx, float* dA, float* dB,
                                        int32_t accumulate, const void* dY, int64_t lddy,
                                        const void* X, int64_t ldx, const float* V, const void* W,
                                        int64_t ldw, const void* A, const void* B,
                                        const int32_t* index, const float* scale,
                                        thanos_dtype_t dtype, int64_t n_tok, int64_t c, int64_t b,
                                        int64_t n_adapters, int32_t r, void* workspace,
                                        size_t ws_bytes, void* stream) {
  const bool grads = dA != nullptr || dB != nullptr;
  if (!W || (n_tok > 0 && !dY)) return THANOS_ERR_INVALID_ARG;
  if (grads && (!dA || !dB || n_adapters == 0 || (n_tok > 0 && (!X || !V))))
    return THANOS_ERR_INVALID_ARG;
  if (n_adapters > 0 && (!A || !B || !scale || (n_tok > 0 && !index)))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(adapter_shape(n_tok, c, b, n_adapters, r, dtype));
  if (lddy < c || ldw < b || (dX && lddx < b) || (grads && ldx < b)) return THANOS_ERR_SHAPE;
  if (ldw % 8 || (grads && ldx % 8)) return THANOS_ERR_ALIGNMENT;
  if (!aligned16(dX) || !aligned16(dA) || !aligned16(dB) || !aligned16(dY) || !aligned16(V) ||
      !aligned16(X) || !aligned16(W) || !aligned16(A) || !aligned16(B) || !aligned4(index) ||
      !aligned4(scale) || !aligned16(workspace))
    return THANOS_ERR_ALIGNMENT;
  if (!workspace ||
      ws_bytes < thanos_adapter_workspace_bytes(1, n_tok, c, b, n_adapters, r, dtype))
    return THANOS_ERR_WORKSPACE;
  if (n_tok == 0) {
    THANOS_CUDA(cudaMemsetAsync(workspace, 0, 16, static_cast<cudaStream_t>(stream)));
    if (grads && !accumulate) {
      const size_t nr = (size_t)n_adapters * (size_t)r;
      THANOS_CUDA(cudaMemsetAsync(dA, 0, nr * (size_t)b * 4, static_cast<cudaStream_t>(stream)));
      THANOS_CUDA(cudaMemsetAsync(dB, 0, nr * (size_t)c * 4, static_cast<cudaStream_t>(stream)));
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
  a.W = W;
  a.ldw = ldw;
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
  return adapter_backward_impl(a, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
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
