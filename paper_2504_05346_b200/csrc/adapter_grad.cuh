// Gradients of the adapters from 16-bit activations (see adapter_grad.cu).
#pragma once

#include "common.cuh"

namespace thanos {

// Tokens by adapter: order[off[i] .. off[i + 1]) are the tokens of adapter i in ascending order.
// One CTA, which runs beside the launch before it in the stream (it reads nothing but index, which has
// to be there when that launch starts); also reports an index that names no adapter.
thanos_status_t sort_tokens(const int32_t* index, int64_t T, int64_t n, int32_t* order,
                            int32_t* spare, int32_t* off, int32_t* status, cudaStream_t stream);

struct AdapterGradSide {
  const __nv_bfloat16* Z = nullptr;  // [T, F], leading dimension ldz (multiple of 8)
  int64_t ldz = 0;
  const __nv_bfloat16* R = nullptr;  // [T, 2 r16] with r16 = r rounded up to 16: R[t] as two bf16
                                     // planes hi | lo, zeros beyond r
  const float* scale = nullptr;      // factor by adapter, or null
  float* out = nullptr;              // [n, r, F], or [n, F, r] if by_feature
  int F = 0;
  int by_feature = 0;
};

// out_i = scale_i sum over the adapter's tokens of R[t]^T Z[t], for both sides in one launch.
thanos_status_t adapter_grads(const AdapterGradSide& a, const AdapterGradSide& b,
                              const int32_t* order, const int32_t* off, int64_t T, int64_t n, int r,
                              int accumulate, int32_t* status, cudaStream_t stream);

// x = hi + lo to 16 significant bits; what is not finite is in hi alone.
__device__ __forceinline__ void split2(float x, __nv_bfloat16& hi, __nv_bfloat16& lo) {
  hi = __float2bfloat16_rn(x);
  const float h = __bfloat162float(hi);
  lo = __float2bfloat16_rn(isfinite(h) ? x - h : 0.f);
}

}  // namespace thanos
