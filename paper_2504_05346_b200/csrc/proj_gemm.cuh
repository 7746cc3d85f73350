// 16-bit products on tcgen05 for the recovery operators: the adapted projection, its skinny
// companion (V = X A^T) and the products of the Newton-Schulz iteration.
//
//   D[m, n] = sum_k A(m, k) B(n, k)     A [M, K] K-major, or stored [K, M] (MN-major); B [N, K]
//
// with m along the lanes of tensor memory.  Consecutive m are consecutive in memory for every
// output (y[n, m] for token n and feature m), so a warp's stores are coalesced without a
// transposition, and few tokens are simply a small n (down to 16 columns of the instruction).
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace thanos {

enum ProjEpilogue {
  PROJ_OUT = 0,     // out[n, m] = bf16(D + adapter part)
  PROJ_SHRINK = 1,  // m = (adapter, rank): V[n, rank] where the token's adapter is the row's
  PROJ_GRAM = 2,    // S = alpha D, fp16, symmetric: upper tiles computed, mirror written; with
                    // s_diag the diagonal goes there in fp32 and is zero in S
  PROJ_GRAM_ADD = 3,  // the same, added to both planes of the S that is there (a form of its own: the
                    // code for it costs PROJ_GRAM 3 us of 110 where its products are small)
  PROJ_POLY = 4,    // P = beta S + alpha S S, fp16, symmetric, its diagonal in p_diag likewise
  PROJ_NEXT = 5,    // X' = beta (hi + lo) + alpha P X, as two fp16 planes
  PROJ_FINAL = 6,   // the same value, unscaled, into O (bf16) or the new weights
  PROJ_OUT32 = 7,   // PROJ_OUT with fp32 accuracy: A and B are three bf16 planes (a_batch, b_batch
                    // apart), out and P are fp32
  PROJ_SHRINK32 = 8 // PROJ_SHRINK with fp32 accuracy, planes as in OUT32
};

struct ProjArgs {
  int M = 0, N = 0, K = 0, batch = 1;
  const void* A = nullptr;
  int64_t lda = 0, a_batch = 0;
  int a_mn = 0;                  // A stored [K, M]
  const void* B = nullptr;
  int64_t ldb = 0, b_batch = 0;
  int f16 = 0;                   // operands fp16 instead of bf16
  int epi = PROJ_OUT;
  int early = 0;                 // operands do not depend on the previous launch of the stream
  int first = 0;                 // first launch of its call: plain, and clears the status word
  const void* skinny = nullptr;  // PROJ_OUT of a few tokens: A [n, r, K], V is computed on the way (and
                                 // written, if wanted)
  int32_t* status = nullptr;
  // PROJ_OUT, PROJ_SHRINK and their fp32 forms
  void* out = nullptr;           // [N, ldo], bf16 (OUT32: fp32)
  int64_t ldo = 0;
  int add = 0;                   // OUT32: to what is there
  int one_plane = 0;             // OUT32: A is bf16, one plane, and three products are enough
  float* V = nullptr;            // [N, r]: PROJ_OUT reads it (forward: V, backward: U); SHRINK writes
  __nv_bfloat16* planes = nullptr;  // SHRINK: V also as three bf16 planes, [N, 3 r16] (or null)
  const int32_t* index = nullptr;
  const float* scale = nullptr;  // factor of a row of V by its adapter, or null
  int n_adapters = 0, r = 0;
  // distinct adapters of every token tile of proj_pair_tile() tokens, [tiles] and [tiles, width]
  const int32_t* tile_count = nullptr;
  const int32_t* tile_list = nullptr;
  const void* P = nullptr;       // the adapters' wide factor, bf16 (OUT32: fp32)
  int64_t ldp = 0, p_adapter = 0;       // a_mn == 0: [n][M][ldp]; else [n][r][ldp].  On CTA pairs
                                        // ldp and p_adapter are multiples of 8
  // PROJ_GRAM .. PROJ_FINAL
  int fine = 0;                  // A, B, S and P have a second plane of what fp16 leaves over, batch
                                 // matrices behind the first; three products of planes
  float alpha = 1.f, beta = 0.f;
  __half* S = nullptr;           // GRAM: written, POLY: read
  int64_t lds = 0, s_batch = 0;
  __half* Pm = nullptr;          // POLY: written (strides as S)
  float* s_diag = nullptr;       // [batch, lds], or both null
  float* p_diag = nullptr;
  const __half* Xh = nullptr;
  const __half* Xl = nullptr;
  __half* Yh = nullptr;
  __half* Yl = nullptr;
  int64_t ldx = 0, x_batch = 0;
  __nv_bfloat16* O = nullptr;
  void* W_out = nullptr;
  const void* W_in = nullptr;
  const uint8_t* mask = nullptr;
  int w_bf16 = 0, tall = 0;
  float keep = 1.f, rate = 0.f;
};

// Width of the token tiles for which PROJ_OUT needs the lists of distinct adapters; 0 if the product
// (N tokens, M features) does not run on CTA pairs and needs none.
int proj_pair_tile(int64_t N, int64_t M);

thanos_status_t proj_gemm(const ProjArgs& a, cudaStream_t stream);

// Programmatic launch: the kernel may start while its predecessor in the stream still runs; it
// waits (griddepcontrol.wait) before it touches anything the predecessor writes.
__device__ __forceinline__ void grid_dependency_wait() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void grid_dependents_launch() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

}  // namespace thanos
