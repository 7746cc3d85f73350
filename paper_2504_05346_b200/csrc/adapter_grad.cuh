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
  const __nv_bfloat16* R = nullptr;  // [T, 3 r16] with r16 = r rounded up to 16: R[t] as three bf16
                                     // planes side by side, zeros beyond r
  const float* scale = nullptr;      // factor by adapter, or null
  float* out = nullptr;              // [n, r, F], or [n, F, r] if by_feature
  int F = 0;
  int by_feature = 0;
};

// out_i = scale_i sum over the adapter's tokens of R[t]^T Z[t], for both sides in one launch.
thanos_status_t adapter_grads(const AdapterGradSide& a, const AdapterGradSide& b,
                              const int32_t* order, const int32_t* off, int64_t T, int64_t n, int r,
                              int accumulate, int32_t* status, cudaStream_t stream);

// x = h + m + l, all 24 bits, cut and not rounded: all three have x's sign, and none is zero beside
// another, so that an infinite factor of x meets three numbers of x's sign (a zero would make a NaN
// of it; what stands in for one is 2^-40 of x).  What is not finite is in l, beside two ones: a finite
// factor meets it once.
__device__ __forceinline__ void split3(float x, __nv_bfloat16& h, __nv_bfloat16& m,
                                       __nv_bfloat16& l) {
  const bool odd = !isfinite(x);
  const float hf = odd ? copysignf(1.f, x) : __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
  const float rest = odd ? 0.f : x - hf;
  const float mf = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u), lf = rest - mf;
  const float stand_in = hf * 0x1p-40f;
  h = __float2bfloat16_rn(hf);
  m = __float2bfloat16_rn(odd ? hf : mf != 0.f ? mf : stand_in);
  l = __float2bfloat16_rn(odd ? x : lf != 0.f ? lf : stand_in);
}

}  // namespace thanos
