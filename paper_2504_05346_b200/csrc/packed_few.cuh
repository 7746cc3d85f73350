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
      constexpr int VEC = 16 / sizeof(T);
      float d = 0.f;
      if (p.r % VEC == 0) {
#pragma unroll 2
        for (int j = 0; j < p.r; j += VEC) {
          const uint4 q = *reinterpret_cast<const uint4*>(bw + j);
          const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (VEC == 8) {
              d = fmaf(vt[j + 2 * e], __uint_as_float(w[e] << 16), d);
              d = fmaf(vt[j + 2 * e + 1], __uint_as_float(w[e] & 0xFFFF0000u), d);
            } else {
              d = fmaf(vt[j + e], __uint_as_float(w[e]), d);
            }
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
