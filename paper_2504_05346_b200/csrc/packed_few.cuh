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


__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1, bool first) {
  if (first) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    return;
  }
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// y of O rows and tokens (row -1: none): the adapters' parts are added here.  The rows of B of all O are in
// flight together (128 tokens of 11008 x 4096 with 16 adapters of rank 16: 43 us, one by one 47).
template <typename T, int O, bool ADAPTERS = true>
__device__ __forceinline__ void finish(const FewParams& p, const int (&row)[O], const int (&at)[O],
                                       float (&v)[O]) {
  if (ADAPTERS && p.n > 0) {
    constexpr int VEC = 16 / sizeof(T);
    int i[O];
#pragma unroll
    for (int u = 0; u < O; ++u) i[u] = row[u] >= 0 ? p.index[at[u]] : -1;
    const T* bw[O];
    const float* vt[O];
    float d[O] = {};
#pragma unroll
    for (int u = 0; u < O; ++u) {
      if (i[u] < -1 || i[u] >= p.n) {
        if (row[u] == 0) atomicCAS(p.status, 0, (int)THANOS_ERR_INVALID_ARG);
        i[u] = -1;
      }
      // without an adapter: read what is there, and leave the sum out
      bw[u] = static_cast<const T*>(p.B) + (i[u] >= 0 ? ((int64_t)i[u] * p.c + row[u]) * p.r : 0);
      vt[u] = p.V + (i[u] >= 0 ? (int64_t)at[u] * p.r : 0);
    }
    if (p.r % VEC == 0) {  // rows of B_i and of V on whole 16-byte lines
#pragma unroll(O == 1 ? 2 : 1)
      for (int j = 0; j < p.r; j += VEC) {
        uint4 q[O];
        float f[O][VEC];
#pragma unroll
        for (int u = 0; u < O; ++u) q[u] = *reinterpret_cast<const uint4*>(bw[u] + j);
#pragma unroll
        for (int u = 0; u < O; ++u) {
#pragma unroll
          for (int e = 0; e < VEC; e += 4) {
            const float4 w = *reinterpret_cast<const float4*>(vt[u] + j + e);
            f[u][e] = w.x, f[u][e + 1] = w.y, f[u][e + 2] = w.z, f[u][e + 3] = w.w;
          }
        }
#pragma unroll
        for (int u = 0; u < O; ++u) {
          const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (VEC == 8) {
              d[u] = fmaf(f[u][2 * e], __uint_as_float(w[e] << 16), d[u]);
              d[u] = fmaf(f[u][2 * e + 1], __uint_as_float(w[e] & 0xFFFF0000u), d[u]);
            } else {
              d[u] = fmaf(f[u][e], __uint_as_float(w[e]), d[u]);
            }
          }
        }
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < p.r; ++j)
#pragma unroll
        for (int u = 0; u < O; ++u) d[u] = fmaf(vt[u][j], to_float(bw[u][j]), d[u]);
    }
#pragma unroll
    for (int u = 0; u < O; ++u)
      if (i[u] >= 0) v[u] = fmaf(p.scale[i[u]], d[u], v[u]);
  }
#pragma unroll
  for (int u = 0; u < O; ++u) {
    if (row[u] < 0) continue;
    T* y = static_cast<T*>(p.Y) + (int64_t)at[u] * p.ldy + row[u];
    if constexpr (sizeof(T) == 2) *y = __float2bfloat16_rn(v[u]);
    else *y = v[u];
  }
}

}  // namespace

// bf16 activations on the tensor cores' tiles of 128 rows (packed_tc.cu).
thanos_status_t packed_tiles(const FewParams& p, cudaStream_t stream);

}  // namespace thanos
