// Shared by the kernels of the adapted projection of few tokens on 4-bit weights (packed_gemv.cu,
// packed_tc.cu).
#pragma once

#include "packed.cuh"
#include "proj_gemm.cuh"
#include "tc_common.cuh"

namespace thanos {

struct FewParams {
  void* Y;
  int64_t ldy;
  const void* X;
  int64_t ldx;
  const uint8_t* codes;
  int64_t ldq;
  const __nv_bfloat16* scales;
  const void* A;
  const void* B;
  const int32_t* index;
  const float* scale;
  float* V;
  int32_t* status;
  int c, b, T, n, r, shift;  // group = 2^shift columns
};

namespace {

using namespace tc;
using bf16 = __nv_bfloat16;


// y of one row and token: the adapter's part is added here.
template <typename T>
__device__ __forceinline__ void finish(const FewParams& p, int row, int at, float v) {
  if (p.n > 0) {
    const int i = p.index[at];
    if (i >= 0 && i < p.n) {
      const T* bw = static_cast<const T*>(p.B) + ((int64_t)i * p.c + row) * p.r;
      const float* vt = p.V + (int64_t)at * p.r;
      float d = 0.f;
      if (p.r % 8 == 0) {  // rows of B_i and of V on whole 16-byte lines
#pragma unroll 2
        for (int j = 0; j < p.r; j += 8) {
          const float4 v0 = *reinterpret_cast<const float4*>(vt + j);
          const float4 v1 = *reinterpret_cast<const float4*>(vt + j + 4);
          const uint4* q = reinterpret_cast<const uint4*>(bw + j);
          if constexpr (sizeof(T) == 2) {
            const float f[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
            const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              d = fmaf(f[2 * e], __uint_as_float(w[e] << 16), d);
              d = fmaf(f[2 * e + 1], __uint_as_float(w[e] & 0xFFFF0000u), d);
            }
          } else {
            const float4 b0 = reinterpret_cast<const float4*>(q)[0];
            const float4 b1 = reinterpret_cast<const float4*>(q)[1];
            d = fmaf(v0.x, b0.x, d), d = fmaf(v0.y, b0.y, d);
            d = fmaf(v0.z, b0.z, d), d = fmaf(v0.w, b0.w, d);
            d = fmaf(v1.x, b1.x, d), d = fmaf(v1.y, b1.y, d);
            d = fmaf(v1.z, b1.z, d), d = fmaf(v1.w, b1.w, d);
          }
        }
      } else {
        for (int j = 0; j < p.r; ++j) d = fmaf(vt[j], to_float(bw[j]), d);
      }
      v = fmaf(p.scale[i], d, v);
    } else if (i != -1 && row == 0) {
      atomicCAS(p.status, 0, (int)THANOS_ERR_INVALID_ARG);
    }
  }
  T* y = static_cast<T*>(p.Y) + (int64_t)at * p.ldy + row;
  if constexpr (sizeof(T) == 2) *y = __float2bfloat16_rn(v);
  else *y = v;
}

}  // namespace

// bf16 activations on the tensor cores' tiles of 128 rows (packed_tc.cu).
thanos_status_t packed_tiles(const FewParams& p, cudaStream_t stream);

}  // namespace thanos
