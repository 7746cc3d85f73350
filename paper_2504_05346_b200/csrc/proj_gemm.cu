// See proj_gemm.cuh.  Two kernels share the operand layouts and the epilogues.
//
// tile_kernel: one CTA per 128 x nt output tile and slice of k.  A cluster of up to eight CTAs
// splits the k range of a tile when there are fewer tiles than SMs and adds the partial sums over
// distributed shared memory in rank order (same inputs, same bits).  Roles of its 320 threads:
//   warp 0      TMA producer: per 64-wide k step the A tile (128 x 64, 128-byte swizzle; K-major, or
//               two MN-major boxes of 64 m x 64 k) and the B tile (nt x 64, K-major)
//   warp 1      tcgen05.mma issuer, 128 x nt x 16 each
//   warps 2..9  first the adapter part of the outputs they will write, in fp32 on the ALUs while the
//               weights stream in (2 r flops per output, next to 2 K in the product), then the
//               epilogue: a quarter of the TMEM lanes and half of the columns each
// pair_kernel: large products, see there.
// Few tokens are bound by reading the weights, and short of that by one wave of CTAs: 64 tokens, 11008
// x 4096, 64 adapters of rank 16 (123 MB): 31 us, 4.0 TB/s; 1 token, 4096 x 4096 (34 MB): 12.6 us,
// 2.7 TB/s, of which start and the partial sums are half.
// Every wait is bounded (see tc_common.cuh); on expiry the status word gets THANOS_ERR_TIMEOUT.
#include "proj_gemm.cuh"

#include <math.h>

#include "adapter_grad.cuh"
#include "tc_common.cuh"

namespace thanos {

namespace {

using namespace tc;

constexpr int TM = 128;
constexpr int BK = 64;
constexpr int A_BYTES = TM * BK * 2;
constexpr int MAX_STAGES = 10;
constexpr int TILE_THREADS = 320;
constexpr int DRAIN_STEPS = 8;
constexpr int FACTOR_BYTES = 128 * 16 * 4;    // 16 ranks of up to 128 tokens, fp32

struct Params {
  int M, N, K, tiles_m, tiles_n, nt, stages, splits, batch_z, ring_bytes, tmem_cols;
  int products;                  // of planes: six, or three where A is one plane
  int symmetric, f16, early, first, fine, add;
  int32_t* status;
  // adapter part
  void* out;
  int64_t ldo;
  float* V;
  __nv_bfloat16* planes;
  const __nv_bfloat16* skinny;        // A, for V on the way; the tokens are at x, ld_tok apart
  const __nv_bfloat16* x;
  int64_t ld_tok;
  const int32_t* index;
  const float* scale;
  int n_adapters, r, chunks;          // chunks of 16 per adapter
  const int32_t* tile_count;
  const int32_t* tile_list;
  const __nv_bfloat16* P;             // OUT32: fp32 values
  int64_t ldp, p_adapter;
  // iteration
  float alpha, beta;
  __half* S;
  int64_t lds, s_batch;
  __half* Pm;
  float* s_diag;
  float* p_diag;
  const __half* Xh;
  const __half* Xl;
  __half* Yh;
  __half* Yl;
  int64_t ldx, x_batch;
  __nv_bfloat16* O;
  void* W_out;
  const void* W_in;
  const uint8_t* mask;
  int w_bf16, tall;
  float keep, rate;
};

__device__ __forceinline__ uint64_t make_desc(uint32_t addr, uint32_t lbo, uint32_t sbo,
                                              uint32_t layout) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)layout << 61;
  return d;
}
constexpr uint32_t SW128 = 2, SW32 = 6;

// The four products of a 64-wide k step whose operands start at the descriptors ad, bd.  Only the
// start address (16-byte units, in the low bits) moves between them.
template <bool AMN, bool PAIR>
__device__ __forceinline__ void mma_step(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc,
                                         uint32_t first) {
#pragma unroll
  for (int k4 = 0; k4 < BK / 16; ++k4) {
    const uint64_t a = ad + (uint64_t)(k4 * (AMN ? 2048 : 32) >> 4);
    const uint64_t b = bd + (uint64_t)(k4 * 32 >> 4);
    if (PAIR) tc_mma_bf16_pair(d, a, b, idesc, k4 == 0 ? first : 1u);
    else tc_mma_bf16(d, a, b, idesc, k4 == 0 ? first : 1u);
  }
}

__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ void tc_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t u[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]),
        "=r"(u[7])
      : "r"(taddr)
      : "memory");
  tc_wait_ld();
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(u[e]);
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, float (&v)[16]) {
  uint32_t u[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]),
        "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]),
        "=r"(u[14]), "=r"(u[15])
      : "r"(taddr)
      : "memory");
  tc_wait_ld();
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(u[e]);
}
__device__ __forceinline__ float tc_ld1(uint32_t taddr) {
  uint32_t u;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(u) : "r"(taddr) : "memory");
  tc_wait_ld();
  return __uint_as_float(u);
}
__device__ __forceinline__ void tc_st1(uint32_t taddr, float v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr),
               "r"(__float_as_uint(v))
               : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
      "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
      "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
      : "memory");
}
__device__ __forceinline__ void tc_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ bool bf16_nonfinite(uint32_t h) { return (h & 0x7F80u) == 0x7F80u; }
// any non-finite bf16 in a 16-byte vector
__device__ __forceinline__ bool any_nonfinite(const uint4& q) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    bad = bad || bf16_nonfinite(w[e]) || bf16_nonfinite(w[e] >> 16);
  return bad;
}
__device__ __forceinline__ uint32_t drop_nonfinite(uint32_t w) {
  if (bf16_nonfinite(w)) w &= 0xFFFF0000u;
  if (bf16_nonfinite(w >> 16)) w &= 0x0000FFFFu;
  return w;
}

__device__ __forceinline__ int valid_adapter(const Params& p, int t) {
  const int i = p.index[t];
  return i >= 0 && i < p.n_adapters ? i : -1;
}

// The 16 columns j0.. of a token's factor, sc V[t, j], zeros beyond the rank.
__device__ __forceinline__ void token_factor(const Params& p, int t, float sc, int j0, float (&v)[16]) {
  const float* src = p.V + (int64_t)t * p.r + j0;
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] = 0.f;
  if (p.r % 4 == 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j0 + 4 * e < p.r) {
        const float4 f = *reinterpret_cast<const float4*>(src + 4 * e);
        v[4 * e] = sc * f.x;
        v[4 * e + 1] = sc * f.y;
        v[4 * e + 2] = sc * f.z;
        v[4 * e + 3] = sc * f.w;
      }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j0 + j < p.r) v[j] = sc * src[j];
  }
}

// Sixteen values as two planes of packed bf16: what the first cuts off (nothing of an infinity or NaN)
// is rounded in the second, 2^-16 of the value, far below the rounding of the result.
__device__ __forceinline__ void factor_planes(const float (&v)[16], uint32_t (&hi)[8],
                                              uint32_t (&lo)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t h[2], l[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float x = v[2 * e + k];
      const bool odd = !isfinite(x);
      h[k] = odd ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __float_as_uint(x) >> 16;
      const float rest = odd ? 0.f : x - __uint_as_float(h[k] << 16);
      l[k] = __bfloat16_as_ushort(__float2bfloat16_rn(rest));
    }
    hi[e] = h[0] | h[1] << 16;
    lo[e] = l[0] | l[1] << 16;
  }
}

__device__ __forceinline__ void clean_vector(uint4* at, int* poison) {
  uint4 w = *at;
  if (any_nonfinite(w)) {
    w.x = drop_nonfinite(w.x);
    w.y = drop_nonfinite(w.y);
    w.z = drop_nonfinite(w.z);
    w.w = drop_nonfinite(w.w);
    *at = w;
    *poison = 1;
  }
}

template <bool AMN>
__device__ __noinline__ float poison_terms(const Params& p, int m, int t) {
  const int i = valid_adapter(p, t);
  float s = 0.f;
  if (i < 0) return s;
  for (int j = 0; j < p.r; ++j) {
    const __nv_bfloat16 w =
        p.P[(int64_t)i * p.p_adapter + (AMN ? (int64_t)j * p.ldp + m : (int64_t)m * p.ldp + j)];
    if (bf16_nonfinite(__bfloat16_as_ushort(w))) {
      const float v = p.V[(int64_t)t * p.r + j];
      s += (p.scale ? p.scale[i] * v : v) * __bfloat162float(w);
    }
  }
  return s;
}

__device__ __forceinline__ uint4 pack8_half(const float (&v)[8]) {
  uint4 q;
  uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 h = __floats2half2_rn(v[2 * e], v[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return q;
}

// Diagonal entries of NC columns; rows of lds (a multiple of eight) hold them, so whole eights exist.
template <int NC>
__device__ __forceinline__ void load_diag(const float* d, int nc, float (&v)[NC]) {
#pragma unroll
  for (int e = 0; e < NC; e += 4) {
    const float4 q = *reinterpret_cast<const float4*>(d + (e / 8 * 8 < nc ? e : 0));
    v[e] = q.x;
    v[e + 1] = q.y;
    v[e + 2] = q.z;
    v[e + 3] = q.w;
  }
}

// NC consecutive n of one m (a lane); n0 is a multiple of 8.
template <bool AMN, int EPI, int NC>
__device__ __forceinline__ void emit(const Params& p, int z, int m, int n0, float (&v)[NC],
                                     bool mirror, bool poisoned) {
  if (m >= p.M || n0 >= p.N) return;
  const int nc = p.N - n0;  // columns that exist
  if constexpr (EPI == PROJ_OUT32) {
    float* out = static_cast<float*>(p.out) + (int64_t)n0 * p.ldo + m;
    if (p.add) {
      float old[NC];
#pragma unroll
      for (int e = 0; e < NC; ++e) old[e] = out[(int64_t)(e < nc ? e : 0) * p.ldo];
#pragma unroll
      for (int e = 0; e < NC; ++e) v[e] += old[e];
    }
#pragma unroll
    for (int e = 0; e < NC; ++e)
      if (e < nc) out[(int64_t)e * p.ldo] = v[e];
  } else if constexpr (EPI == PROJ_OUT) {
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + (int64_t)n0 * p.ldo + m;
    if (poisoned) {
#pragma unroll
      for (int e = 0; e < NC; ++e)
        if (e < nc) v[e] += poison_terms<AMN>(p, m, n0 + e);
    }
#pragma unroll
    for (int e = 0; e < NC; ++e)
      if (e < nc) out[(int64_t)e * p.ldo] = __float2bfloat16_rn(v[e]);
  } else if constexpr (EPI == PROJ_SHRINK || EPI == PROJ_SHRINK32) {
    const int i = m / p.r, j = m - i * p.r;
#pragma unroll
    for (int e = 0; e < NC; ++e) {
      const int t = n0 + e;
      if (e >= nc) break;
      const int own = valid_adapter(p, t);
      if (own == i) {
        const float x = p.scale ? p.scale[i] * v[e] : v[e];
        p.V[(int64_t)t * p.r + j] = x;
        if (p.planes) {
          const int r16 = 16 * p.chunks;
          __nv_bfloat16* row = p.planes + (int64_t)t * 3 * r16 + j;
          split3(x, row[0], row[r16], row[2 * r16]);
        }
      } else if (own < 0 && i == 0) p.V[(int64_t)t * p.r + j] = 0.f;
    }
  } else if constexpr (EPI == PROJ_GRAM || EPI == PROJ_GRAM_ADD || EPI == PROJ_POLY) {
    __half* D = (EPI == PROJ_POLY ? p.Pm : p.S) + (int64_t)z * p.s_batch;
    if constexpr (EPI == PROJ_POLY) {
      const __half* S = p.S + (int64_t)z * p.s_batch + (int64_t)n0 * p.lds + m;
      // columns beyond the last read the first one again: a load under a condition is not issued ahead
      __half old[NC], rest[NC];
#pragma unroll
      for (int e = 0; e < NC; ++e) old[e] = S[(int64_t)(e < nc ? e : 0) * p.lds];
#pragma unroll
      for (int e = 0; e < NC; ++e) rest[e] = __half(0.f);
      if (p.fine) {
        const __half* S2 = S + (int64_t)p.batch_z * p.s_batch;
#pragma unroll
        for (int e = 0; e < NC; ++e) rest[e] = S2[(int64_t)(e < nc ? e : 0) * p.lds];
      }
      if (p.s_diag) {
        // S = S' + diag(d): S S = S' S' + (d_m + d_n) S' + diag(d^2), of which the product gave the
        // first
        const float* d = p.s_diag + (int64_t)z * p.lds;
        float dn[NC];
        load_diag<NC>(d + n0, nc, dn);
        const float dm = d[m];
#pragma unroll
        for (int e = 0; e < NC; ++e) {
          const float x = n0 + e == m ? dm : __half2float(old[e]) + __half2float(rest[e]);
          const float y = n0 + e == m ? dm : dm + dn[e];
          v[e] = fmaf(fmaf(p.alpha, y, p.beta), x, p.alpha * v[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < NC; ++e)
          v[e] = fmaf(p.beta, __half2float(old[e]) + __half2float(rest[e]), p.alpha * v[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < NC; ++e) v[e] *= p.alpha;
      if constexpr (EPI == PROJ_GRAM_ADD) {
#pragma unroll 1
        for (int pl = 0; pl < 2; ++pl) {
          const __half* S = D + (int64_t)(pl * p.batch_z) * p.s_batch + (int64_t)n0 * p.lds + m;
          __half old[NC];
#pragma unroll
          for (int e = 0; e < NC; ++e) old[e] = S[(int64_t)(e < nc ? e : 0) * p.lds];
#pragma unroll
          for (int e = 0; e < NC; ++e) v[e] += __half2float(old[e]);
        }
      }
    }
    if (p.s_diag && m >= n0 && m < n0 + NC) {
      float* diag = EPI == PROJ_POLY ? p.p_diag : p.s_diag;
#pragma unroll
      for (int e = 0; e < NC; ++e)
        if (n0 + e == m) {
          if (EPI == PROJ_GRAM_ADD) v[e] += diag[(int64_t)z * p.lds + m];
          diag[(int64_t)z * p.lds + m] = v[e];
          v[e] = 0.f;
        }
    }
#pragma unroll 1
    for (int plane = 0;; ++plane) {
      __half* col = D + (int64_t)n0 * p.lds + m;
#pragma unroll
      for (int e = 0; e < NC; ++e)
        if (e < nc) col[(int64_t)e * p.lds] = __float2half_rn(v[e]);
      if (mirror) {
        __half* row = D + (int64_t)m * p.lds + n0;
#pragma unroll
        for (int e8 = 0; e8 < NC; e8 += 8) {
          if (e8 + 8 <= nc) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = v[e8 + e];
            *reinterpret_cast<uint4*>(row + e8) = pack8_half(f);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e8 + e < nc) row[e8 + e] = __float2half_rn(v[e8 + e]);
          }
        }
      }
      if (plane == 1 || !p.fine) break;
      D += (int64_t)p.batch_z * p.s_batch;
#pragma unroll
      for (int e = 0; e < NC; ++e) v[e] -= __half2float(__float2half_rn(v[e]));
    }
  } else {
    const int64_t at = (int64_t)z * p.x_batch + (int64_t)n0 * p.ldx + m;
    __half hi[NC], lo[NC];
#pragma unroll
    for (int e = 0; e < NC; ++e) {
      hi[e] = p.Xh[at + (int64_t)(e < nc ? e : 0) * p.ldx];
      lo[e] = p.Xl[at + (int64_t)(e < nc ? e : 0) * p.ldx];
    }
    if (p.p_diag) {
      // with what the product read of X: P acts on nearly parallel rows of X then as a whole
      float dn[NC];
      load_diag<NC>(p.p_diag + (int64_t)z * p.lds + n0, nc, dn);
#pragma unroll
      for (int e = 0; e < NC; ++e)
        v[e] = fmaf(dn[e], __half2float(hi[e]) + (p.fine ? __half2float(lo[e]) : 0.f), v[e]);
    }
#pragma unroll
    for (int e = 0; e < NC; ++e)
      v[e] = fmaf(p.beta, __half2float(hi[e]) + __half2float(lo[e]), p.alpha * v[e]);
    if constexpr (EPI == PROJ_NEXT) {
#pragma unroll
      for (int e = 0; e < NC; ++e) {
        if (e >= nc) break;
        const __half h = __float2half_rn(v[e]);
        p.Yh[at + (int64_t)e * p.ldx] = h;
        p.Yl[at + (int64_t)e * p.ldx] = __float2half_rn(v[e] - __half2float(h));
      }
    } else {
      const int64_t base = (int64_t)z * (int64_t)p.M * p.N;
      const int64_t step = p.tall ? 1 : p.M;
      const int64_t at0 = base + (p.tall ? (int64_t)m * p.N + n0 : (int64_t)n0 * p.M + m);
      if (p.O) {
        if (p.tall && p.N % 8 == 0) {
#pragma unroll
          for (int e8 = 0; e8 < NC; e8 += 8) {
            if (e8 >= nc) break;
            uint4 q;
            uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              w[e] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[e8 + 2 * e])) |
                     ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[e8 + 2 * e + 1])) << 16);
            *reinterpret_cast<uint4*>(p.O + at0 + e8) = q;
          }
        } else {
#pragma unroll
          for (int e = 0; e < NC; ++e)
            if (e < nc) p.O[at0 + e * step] = __float2bfloat16_rn(v[e]);
        }
      } else {
        // loads first: W_in may be W_out, so the compiler cannot move them over the stores
        float w[NC];
        uint32_t gone = 0;  // bit e: removed
        if (p.tall && p.N % 8 == 0) {
          // the thread's columns are consecutive in memory, and whole groups of eight exist or not
#pragma unroll
          for (int e8 = 0; e8 < NC; e8 += 8) {
            if (e8 >= nc) break;
            if (p.w_bf16) {
              const uint4 q = *reinterpret_cast<const uint4*>(
                  static_cast<const __nv_bfloat16*>(p.W_in) + at0 + e8);
              const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w[e8 + 2 * e] = __uint_as_float(u[e] << 16);
                w[e8 + 2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
              }
            } else {
#pragma unroll
              for (int e4 = 0; e4 < 8; e4 += 4) {
                const float4 q = *reinterpret_cast<const float4*>(
                    static_cast<const float*>(p.W_in) + at0 + e8 + e4);
                w[e8 + e4] = q.x;
                w[e8 + e4 + 1] = q.y;
                w[e8 + e4 + 2] = q.z;
                w[e8 + e4 + 3] = q.w;
              }
            }
            if (p.mask) {
              const uint2 q = *reinterpret_cast<const uint2*>(p.mask + at0 + e8);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((q.x >> (8 * e)) & 0xFFu) gone |= 1u << (e8 + e);
                if ((q.y >> (8 * e)) & 0xFFu) gone |= 1u << (e8 + 4 + e);
              }
            }
          }
#pragma unroll
          for (int e = 0; e < NC; ++e)
            v[e] = (gone >> e) & 1u ? 0.f : fmaf(-p.rate, v[e], p.keep * w[e]);
#pragma unroll
          for (int e8 = 0; e8 < NC; e8 += 8) {
            if (e8 >= nc) break;
            if (p.w_bf16) {
              uint4 q;
              uint32_t* u = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                u[e] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[e8 + 2 * e])) |
                       ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[e8 + 2 * e + 1])) << 16);
              *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.W_out) + at0 + e8) = q;
            } else {
#pragma unroll
              for (int e4 = 0; e4 < 8; e4 += 4)
                *reinterpret_cast<float4*>(static_cast<float*>(p.W_out) + at0 + e8 + e4) =
                    make_float4(v[e8 + e4], v[e8 + e4 + 1], v[e8 + e4 + 2], v[e8 + e4 + 3]);
            }
          }
        } else {
          // the type is asked once, not per element: a branch between two loads would keep them from
          // being in flight together
          if (p.w_bf16) {
            const __nv_bfloat16* W = static_cast<const __nv_bfloat16*>(p.W_in) + at0;
            __nv_bfloat16 h[NC];
#pragma unroll
            for (int e = 0; e < NC; ++e) h[e] = e < nc ? W[e * step] : __float2bfloat16_rn(0.f);
#pragma unroll
            for (int e = 0; e < NC; ++e) w[e] = __bfloat162float(h[e]);
          } else {
            const float* W = static_cast<const float*>(p.W_in) + at0;
#pragma unroll
            for (int e = 0; e < NC; ++e) w[e] = e < nc ? W[e * step] : 0.f;
          }
          if (p.mask && !p.tall && p.M % 16 == 0 && m - (int)(threadIdx.x & 31) + 32 <= p.M &&
              nc >= NC) {
            // 32 mask bytes of each of the NC columns, 16 by a lane in one load; one bit per byte is
            // then handed to the lane that it belongs to (a byte load per column took twice the time
            // of everything else here)
            const int lane = threadIdx.x & 31;
            uint32_t bits = 0;
            if (lane < 2 * NC) {
              const uint4 q = *reinterpret_cast<const uint4*>(
                  p.mask + at0 - lane + (int64_t)(lane >> 1) * step + 16 * (lane & 1));
              const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                  if ((u[e] >> (8 * b)) & 0xFFu) bits |= 1u << (4 * e + b);
            }
#pragma unroll
            for (int e = 0; e < NC; ++e) {
              const uint32_t of = __shfl_sync(0xffffffffu, bits, 2 * e + (lane >> 4));
              gone |= ((of >> (lane & 15)) & 1u) << e;
            }
          } else if (p.mask) {
            uint8_t k[NC];
#pragma unroll
            for (int e = 0; e < NC; ++e) k[e] = e < nc ? p.mask[at0 + e * step] : (uint8_t)0;
#pragma unroll
            for (int e = 0; e < NC; ++e) gone |= (k[e] ? 1u : 0u) << e;
          }
#pragma unroll
          for (int e = 0; e < NC; ++e)
            v[e] = (gone >> e) & 1u ? 0.f : fmaf(-p.rate, v[e], p.keep * w[e]);
          if (p.w_bf16) {
            __nv_bfloat16* W = static_cast<__nv_bfloat16*>(p.W_out) + at0;
#pragma unroll
            for (int e = 0; e < NC; ++e)
              if (e < nc) W[e * step] = __float2bfloat16_rn(v[e]);
          } else {
            float* W = static_cast<float*>(p.W_out) + at0;
#pragma unroll
            for (int e = 0; e < NC; ++e)
              if (e < nc) W[e * step] = v[e];
          }
        }
      }
    }
  }
}

// First column of the q-th group of eight that a thread of tile_kernel writes: every second group,
// or every 2 S-th with a split.
__device__ __forceinline__ int tile_column(int S, int rank, int half, int q) {
  return 8 * (rank + S * (half + 2 * q));
}

__device__ __forceinline__ void prefetch_l2(const void* p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}
__device__ __forceinline__ void epilogue_sync() {  // the eight epilogue warps of tile_kernel
  __syncwarp();
  asm volatile("bar.sync 1, 256;" ::: "memory");
}
__device__ __forceinline__ bool epilogue_any(bool mine) {  // whether any of the 256 says yes
  int r;
  __syncwarp();
  asm volatile(
      "{\n.reg .pred a, b;\nsetp.ne.u32 a, %1, 0;\n"
      "barrier.cta.red.or.aligned.pred b, 1, 256, a;\nselp.u32 %0, 1, 0, b;\n}"
      : "=r"(r)
      : "r"((int)mine)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

// Sixteen ranks of one adapter's row of the wide factor (feature m), packed bf16; zeros beyond r.
template <bool AMN>
__device__ __forceinline__ void wide_row(const Params& p, int i, int m, int j0, uint32_t (&w)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = 0u;
  if (i < 0) return;
  if constexpr (AMN) {
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p.P) +
                              (int64_t)i * p.p_adapter + (int64_t)j0 * p.ldp + m;
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j0 + j < p.r) w[j >> 1] |= (uint32_t)q[(int64_t)j * p.ldp] << (16 * (j & 1));
  } else {
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p.P) +
                              (int64_t)i * p.p_adapter + (int64_t)m * p.ldp + j0;
    if (p.r % 8 == 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (j0 + 8 * h < p.r) {
          const uint4 v = *reinterpret_cast<const uint4*>(q + 8 * h);
          w[4 * h] = v.x;
          w[4 * h + 1] = v.y;
          w[4 * h + 2] = v.z;
          w[4 * h + 3] = v.w;
        }
    } else if (p.r % 2 == 0) {
#pragma unroll
      for (int h = 0; h < 8; ++h)
        if (j0 + 2 * h < p.r) w[h] = *reinterpret_cast<const uint32_t*>(q + 2 * h);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j0 + j < p.r) w[j >> 1] |= (uint32_t)q[j] << (16 * (j & 1));
    }
  }
}

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 u = unpack2(x[e]), v = unpack2(y[e]);
    s = fmaf(u.x, v.x, s);
    s = fmaf(u.y, v.y, s);
  }
  return s;
}

__device__ __forceinline__ void unpack16(const uint32_t (&w)[8], float (&f)[16]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 u = unpack2(w[e]);
    f[2 * e] = u.x;
    f[2 * e + 1] = u.y;
  }
}
__device__ __forceinline__ float dot16(const float (&w)[16], const float* __restrict__ v) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 f = reinterpret_cast<const float4*>(v)[e];
    s = fmaf(w[4 * e], f.x, s);
    s = fmaf(w[4 * e + 1], f.y, s);
    s = fmaf(w[4 * e + 2], f.z, s);
    s = fmaf(w[4 * e + 3], f.w, s);
  }
  return s;
}

// The same in fp32.
template <bool AMN>
__device__ __forceinline__ void wide_row_f32(const Params& p, int i, int m, int j0, float (&w)[16]) {
  const float* P = reinterpret_cast<const float*>(p.P) + (int64_t)(i < 0 ? 0 : i) * p.p_adapter;
  const int last = p.r - 1 - j0;  // ranks beyond it are read again there, and not used
  if (!AMN && p.r % 4 == 0) {
    const float* q = P + (int64_t)m * p.ldp + j0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 f = *reinterpret_cast<const float4*>(q + min(4 * e, last & ~3));
      w[4 * e] = f.x;
      w[4 * e + 1] = f.y;
      w[4 * e + 2] = f.z;
      w[4 * e + 3] = f.w;
    }
  } else {
    const float* q = P + (AMN ? (int64_t)j0 * p.ldp + m : (int64_t)m * p.ldp + j0);
    const int64_t dj = AMN ? p.ldp : 1;
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = q[min(j, last) * dj];
  }
  if (last < 15) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j > last) w[j] = 0.f;
  }
}

// Planes of the six products that make up an fp32 product, the smallest first: the tensor cores cut
// what they add to an accumulator, by up to 2^-23 of it each time, so the products that are 2^-9 and
// 2^-18 of the whole go in before the accumulator has its size.
__device__ __forceinline__ void plane_pair(int combo, int& a, int& b) {
  a = (0x010201 >> (4 * combo)) & 15;  // nibbles from the right: mm, hl, lh, hm, mh, hh
  b = (0x001021 >> (4 * combo)) & 15;
}

__host__ __device__ constexpr bool two_per_sm(int epi) {
  return epi <= PROJ_SHRINK || epi >= PROJ_OUT32;
}

template <bool AMN, int EPI>
__global__ void __launch_bounds__(TILE_THREADS, two_per_sm(EPI) ? 2 : 1)
tile_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
            const Params p) {
  constexpr bool F32 = EPI == PROJ_OUT32, OUT = EPI == PROJ_OUT || F32;
  constexpr bool DRAIN = EPI == PROJ_SHRINK || EPI == PROJ_SHRINK32;
  constexpr bool PLANES = F32 || EPI == PROJ_SHRINK32;
  constexpr bool ITER = EPI >= PROJ_GRAM && EPI <= PROJ_FINAL;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* factor = reinterpret_cast<float*>(smem + p.ring_bytes);             // [nt][16]
  int* ids = reinterpret_cast<int*>(smem + p.ring_bytes + FACTOR_BYTES);     // [nt]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.ring_bytes + FACTOR_BYTES + 512);
  // full [MAX_STAGES], empty [MAX_STAGES], accumulator ready; SHRINK: accumulator full and empty (2)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * MAX_STAGES + 5);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 2 * MAX_STAGES + 6);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem);
  const uint32_t bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (MAX_STAGES + s); };
  const uint32_t done_bar = bar_base + 8u * (2 * MAX_STAGES);
  auto tfull_bar = [&](int q) { return bar_base + 8u * (2 * MAX_STAGES + 1 + q); };
  auto tempty_bar = [&](int q) { return bar_base + 8u * (2 * MAX_STAGES + 3 + q); };

  const int S = p.splits;
  const int rank = S > 1 ? (int)cluster_ctarank() : 0;
  const int tile = (int)(blockIdx.x / S);
  const int tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m;
  const int m0 = tm * TM, n0 = tn * p.nt;
  const int z = blockIdx.y;
  const int stage_bytes = A_BYTES + p.nt * BK * 2;

  if (p.first && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0;
  // symmetric results: tiles left of the diagonal blocks are the mirror of those right of them
  // (nt divides TM)
  if (p.symmetric && n0 < m0) return;
  const bool mirror = n0 >= m0 + TM;
  if constexpr (DRAIN) {
    // rows of adapters that no token of the tile uses are not needed (tile row 0 also writes the
    // zeros of tokens without adapter)
    grid_dependency_wait();
    grid_dependents_launch();
    if (tm > 0) {
      const int lo = m0 / p.r, hi = (min(m0 + TM, p.M) - 1) / p.r;
      bool hit = false;
      for (int t = n0 + lane; t < min(n0 + p.nt, p.N); t += 32) {
        const int i = p.index[t];
        hit = hit || (i >= lo && i <= hi);
      }
      if (!__any_sync(0xffffffffu, hit)) return;  // the same answer in every warp of the cluster
    }
  }

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(done_bar, 1);
    for (int q = 0; q < 2; ++q) {
      mbar_init(tfull_bar(q), 1);
      mbar_init(tempty_bar(q), 8);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(p.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if constexpr (!DRAIN) grid_dependents_launch();

  const int nk1 = (p.K + BK - 1) / BK;
  const int planes = ITER && p.fine ? 2 : 1;  // stages of a k step: hi planes, then lo planes
  // this CTA's k blocks; three planes: all six products of planes of each, one product after another
  const int b0 = (int)((int64_t)nk1 * rank / S), b1 = (int)((int64_t)nk1 * (rank + 1) / S);
  const int ks0 = PLANES ? p.products * b0 : b0, ks1 = PLANES ? p.products * b1 : b1;
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (!p.early) grid_dependency_wait();
    if (elect_one()) {
    int s = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int q = planes * ks0; q < planes * ks1 && ok; ++q) {
      const int ks = planes == 2 ? q >> 1 : q, second = planes == 2 && (q & 1) ? p.batch_z : 0;
      ok = mbar_wait(empty_bar(s), phase ^ 1u, abort_flag);
      if (ok) {
        const uint32_t dst = smem_base + (uint32_t)s * stage_bytes;
        int k0 = ks * BK, za = z + second, zb = z + second;
        if (PLANES) {
          const int combo = (ks - ks0) / (b1 - b0);
          k0 = (b0 + ks - ks0 - combo * (b1 - b0)) * BK;
          plane_pair(p.products == 6 ? combo : 2 * combo + 1, za, zb);  // hl, hm, hh of the six
        }
        mbar_expect_tx(full_bar(s), stage_bytes);
        if (AMN) {
          tma_load_3d(dst, &mapA, full_bar(s), m0, k0, za);
          tma_load_3d(dst + A_BYTES / 2, &mapA, full_bar(s), m0 + 64, k0, za);
        } else {
          tma_load_3d(dst, &mapA, full_bar(s), k0, m0, za);
        }
        tma_load_3d(dst + A_BYTES, &mapB, full_bar(s), k0, n0, zb);
      }
      if (++s == p.stages) {
        s = 0;
        phase ^= 1u;
      }
    }
    // let copies that are still in flight land before the CTA's shared memory goes away
    if (!ok) {
      for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    // its bounded waits begin when the operands can come, however long the launch before takes
    if (!p.early) grid_dependency_wait();
    if (elect_one()) {
    uint32_t idesc = 0;
    idesc |= 1u << 4;  // D fp32
    if (!p.f16) idesc |= (1u << 7) | (1u << 10);  // both operands bf16 (0: both fp16)
    if (AMN) idesc |= 1u << 15;
    idesc |= (uint32_t)(p.nt >> 3) << 17;
    idesc |= (uint32_t)(TM >> 4) << 24;
    const uint64_t ad0 = AMN ? make_desc(smem_base, A_BYTES / 2, 1024, SW128)
                             : make_desc(smem_base, 16, 1024, SW128);
    const uint64_t bd0 = make_desc(smem_base + A_BYTES, 16, 1024, SW128);
    const uint64_t hop = (uint64_t)(stage_bytes >> 4);
    int s = 0;
    uint32_t phase = 0;
    uint64_t at = 0;  // stage s in descriptor units
    bool ok = true;
    int q = 0;
    uint32_t tphase = 0;
    for (int ks = ks0; ks < ks1 && ok; ++ks) {
      const bool start = DRAIN ? (ks - ks0) % DRAIN_STEPS == 0 : ks == ks0;
      if (DRAIN && start) {
        ok = mbar_wait(tempty_bar(q), tphase ^ 1u, abort_flag);
        tc_fence_after();
      }
      ok = ok && mbar_wait(full_bar(s), phase, abort_flag);
      tc_fence_after();
      const uint32_t d = tmem_base + (uint32_t)(q * p.nt);
      if (ITER && planes == 2) {
        // hi and lo planes lie in this stage and the next: hi lo + lo hi + hi hi
        const uint64_t hi = at;
        const int s_hi = s;
        at += hop;
        if (++s == p.stages) {
          s = 0;
          at = 0;
          phase ^= 1u;
        }
        ok = ok && mbar_wait(full_bar(s), phase, abort_flag);
        tc_fence_after();
        if (ok) {
          mma_step<AMN, false>(d, ad0 + hi, bd0 + at, idesc, start ? 0u : 1u);
          mma_step<AMN, false>(d, ad0 + at, bd0 + hi, idesc, 1u);
          mma_step<AMN, false>(d, ad0 + hi, bd0 + hi, idesc, 1u);
          tc_commit(empty_bar(s_hi));
          tc_commit(empty_bar(s));
        }
      } else if (ok) {
        mma_step<AMN, false>(d, ad0 + at, bd0 + at, idesc, start ? 0u : 1u);
        tc_commit(empty_bar(s));
      }
      if (DRAIN && ((ks - ks0) % DRAIN_STEPS == DRAIN_STEPS - 1 || ks + 1 == ks1)) {
        if (ok) tc_commit(tfull_bar(q));
        tphase ^= (uint32_t)q;
        q ^= 1;
      }
      at += hop;
      if (++s == p.stages) {
        s = 0;
        at = 0;
        phase ^= 1u;
      }
    }
    if (ok) tc_commit(done_bar);
    }
    __syncwarp();
  } else {
    const int g = warp & 3, half = (warp - 2) >> 2;
    const int row = 32 * g + lane, m = m0 + row;
    const uint32_t taddr = tmem_base + ((uint32_t)(32 * g) << 16);
    // All loops below are kept rolled: the code runs once per CTA, and straight-line code of a few
    // thousand instructions costs more in instruction fetches than it saves.
    // Instructions of tensor memory want the whole warp, so its lanes take the same way: a lane
    // beyond the last row does what the last row does, and only emit() leaves it out.
    const bool live_warp = m0 + 32 * g < p.M;
    const int mr = min(m, p.M - 1);
    bool used = false;
    if constexpr (OUT) {
      // ---------------------------------------------------------- adapter part
      const int tid = threadIdx.x - 64;
      if (p.n_adapters > 0) {
        bool any = false;
        if (tid < p.nt) {
          const int t = n0 + tid;
          const int i = t < p.N ? valid_adapter(p, t) : -1;
          ids[tid] = i;
          any = i >= 0;
        }
        used = epilogue_any(any);
      }
      int ldf = 16;                      // row of `factor`
      if (!used && !F32 && p.skinny && p.V && tm == 0 && rank == 0) {
        // no token of the tile has an adapter: there is nothing to compute, but V is an output
        const int e1 = min(n0 + p.nt, p.N) * p.r;
        for (int e = n0 * p.r + tid; e < e1; e += 256) p.V[e] = 0.f;
      }
      if (used && !F32 && p.skinny) {
        // V of the few tokens, by the CTAs that write their outputs: a warp per pair of ranks
        ldf = (p.r + 15) & ~15;
        const int live = min(p.nt, p.N - n0);
        const bool mine = tile_column(S, rank, 0, 0) < live;
#pragma unroll 1
        for (int e = 2 * (warp - 2); mine && e < live * ldf; e += 16) {
          const int c = e / ldf, j = e - c * ldf, i = ids[c];
          float s0 = 0.f, s1 = 0.f;
          if (i >= 0 && j < p.r) {
            const __nv_bfloat16* xr = p.x + (int64_t)(n0 + c) * p.ld_tok;
            const __nv_bfloat16* a0 = p.skinny + ((int64_t)i * p.r + j) * p.K;
            const __nv_bfloat16* a1 = a0 + (j + 1 < p.r ? p.K : 0);
#pragma unroll 8
            for (int k = lane * 8; k < p.K; k += 256) {
              const uint4 x = *reinterpret_cast<const uint4*>(xr + k);
              s0 = dot8(x, *reinterpret_cast<const uint4*>(a0 + k), s0);
              s1 = dot8(x, *reinterpret_cast<const uint4*>(a1 + k), s1);
            }
            for (int o = 16; o > 0; o >>= 1) {
              s0 += __shfl_xor_sync(0xffffffffu, s0, o);
              s1 += __shfl_xor_sync(0xffffffffu, s1, o);
            }
            if (j + 1 >= p.r) s1 = 0.f;
          }
          if (lane < 2 && j + lane < ldf) {
            const float v = lane ? s1 : s0;
            if (tm == 0 && p.V && j + lane < p.r) p.V[(int64_t)(n0 + c) * p.r + j + lane] = v;
            factor[e + lane] = i >= 0 && p.scale ? p.scale[i] * v : v;
          }
        }
      }
      if (used && !F32 && p.early) {
        // while the launch before this one still computes V, the rows of the wide factors that this
        // thread will read are on their way to L2
#pragma unroll 1
        for (int q = 0; live_warp; ++q) {
          const int c = tile_column(S, rank, half, q);
          if (c >= p.nt || n0 + c >= p.N) break;
#pragma unroll 1
          for (int e = 0; e < 8; ++e) {
            const int i = ids[c + e];
            if (i < 0 || (e > 0 && ids[c + e - 1] == i)) continue;
            const __nv_bfloat16* a =
                p.P + (int64_t)i * p.p_adapter + (AMN ? (int64_t)mr : (int64_t)mr * p.ldp);
            for (int jj = 0; jj < p.r; jj += AMN ? 1 : 16) prefetch_l2(a + jj * (AMN ? p.ldp : 1));
          }
        }
      }
      grid_dependency_wait();
#pragma unroll 1
      for (int j0 = 0; used && j0 < p.r; j0 += 16) {
        const float* fac = factor;
        if (!F32 && p.skinny) {
          fac += j0;
          if (j0 == 0) epilogue_sync();
        } else {
          epilogue_sync();
#pragma unroll 4
          for (int e = tid; e < p.nt * 16; e += 256) {
            const int i = ids[e >> 4], j = j0 + (e & 15);
            const bool live = i >= 0 && j < p.r;
            const float v = live ? p.V[(int64_t)(n0 + (e >> 4)) * p.r + j] : 0.f;
            const float f = live && p.scale ? p.scale[i] : 1.f;
            factor[e] = f * v;
          }
          epilogue_sync();
        }
        float w[16];
        int held = -1;  // the adapter whose row w is
#pragma unroll 1
        for (int q = 0; live_warp; ++q) {
          const int c = tile_column(S, rank, half, q);
          if (c >= p.nt || n0 + c >= p.N) break;
          // eight tokens of one request, some perhaps without adapter, share a row
          int one = -1;
          bool same = true;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = ids[c + e];
            same = same && (i < 0 || one < 0 || i == one);
            one = max(one, i);
          }
          if (F32 || same) {
            // the row stays in registers from one eight to the next while the request stays the same
            if (same && one >= 0 && one != held) {
              if constexpr (F32) {
                wide_row_f32<AMN>(p, one, mr, j0, w);
              } else {
                uint32_t u[8];
                wide_row<AMN>(p, one, mr, j0, u);
                unpack16(u, w);
              }
              held = one;
            }
            if (same && j0 > 0) {
              // further ranks: eight columns of sums are fetched, added to and put back together
              float d[8];
              tc_ld8(taddr + p.nt + c, d);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (ids[c + e] >= 0) d[e] += dot16(w, fac + (c + e) * ldf);
              tc_st8(taddr + p.nt + c, d);
            } else {
#pragma unroll 1
              for (int e = 0; e < 8; ++e) {
                const int i = ids[c + e];
                if constexpr (F32) {
                  if (!same && i >= 0) wide_row_f32<AMN>(p, i, mr, j0, w);
                }
                float d = i >= 0 ? dot16(w, fac + (c + e) * ldf) : 0.f;
                if (F32 && j0 > 0) d += tc_ld1(taddr + p.nt + c + e);
                tc_st1(taddr + p.nt + c + e, d);
              }
              if (!same) held = -1;
            }
          } else {
#pragma unroll 1
            for (int e4 = 0; e4 < 8; e4 += 4) {
              uint32_t u[4][8];  // four rows in flight
#pragma unroll
              for (int e = 0; e < 4; ++e)
                wide_row<AMN>(p, ids[c + e4 + e], mr, j0, u[e]);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float f[16];
                unpack16(u[e], f);
                float d = ids[c + e4 + e] >= 0 ? dot16(f, fac + (c + e4 + e) * ldf) : 0.f;
                if (j0 > 0) d += tc_ld1(taddr + p.nt + c + e4 + e);
                tc_st1(taddr + p.nt + c + e4 + e, d);
              }
            }
          }
        }
        // the sums are kept in tensor memory beside the accumulator, at the columns they belong to
        tc_wait_st();
      }
    } else {
      grid_dependency_wait();
    }
    // ------------------------------------------------------------ epilogue, one slice of k
    bool ok = true;
    if constexpr (DRAIN) {
      // The tensor cores cut what they add to an accumulator, so a long chain of them drifts (128 of
      // them: 2e-6 of V); after every DRAIN_STEPS steps the sums move on in registers, rounded.
      float own[8][8] = {};
      int q = 0;
      uint32_t tphase = 0;
      for (int ks = ks0; ks < ks1 && ok; ks += DRAIN_STEPS) {
        ok = mbar_wait_warp(tfull_bar(q), tphase, abort_flag);
        tc_fence_after();
        if (!ok) break;
#pragma unroll
        for (int g8 = 0; g8 < 8; ++g8) {
          const int c = 8 * (half + 2 * g8);
          if (c >= p.nt) break;
          float v[8];
          tc_ld8(taddr + q * p.nt + c, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) own[g8][e] += v[e];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(q));
        tphase ^= (uint32_t)q;
        q ^= 1;
      }
      // all products are done: the first accumulator takes the totals
      if (ok) {
#pragma unroll
        for (int g8 = 0; g8 < 8; ++g8) {
          const int c = 8 * (half + 2 * g8);
          if (c < p.nt) tc_st8(taddr + c, own[g8]);
        }
        tc_wait_st();
      }
    } else {
      ok = mbar_wait_warp(done_bar, 0, abort_flag);
      tc_fence_after();
    }
    if (ok && S == 1) {
#pragma unroll 1
      for (int q = 0;; ++q) {
        const int c = tile_column(1, 0, half, q);
        if (c >= p.nt || n0 + c >= p.N) break;
        float v[8];
        tc_ld8(taddr + c, v);
        if (used) {
          float own[8];
          tc_ld8(taddr + p.nt + c, own);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += own[e];
        }
        emit<AMN, EPI, 8>(p, z, m, n0 + c, v, mirror, false);
        __syncwarp();
      }
    }
    if (S > 1) {
      // Every CTA writes the sums of a group of eight columns to the CTA that owns it, into the ring
      // there: [CTA][group][column][m].  The first barrier says that all rings are free.
      cluster_sync_all();
      bool bad = false;
#pragma unroll 1
      for (int q = 0; q < S; ++q)
        bad = bad || ld_cluster_u32(map_to_cta(smem_u32((const void*)abort_flag), q)) != 0;
      const int G = (p.nt / 8 + S - 1) / S;
#pragma unroll 1
      for (int c = 8 * half; c < p.nt && !bad; c += 16) {
        float v[8];
        tc_ld8(taddr + c, v);
        const uint32_t dst = map_to_cta(smem_base, (c >> 3) % S) +
                             (uint32_t)((((rank * G + (c >> 3) / S) * 8) * TM + row) * 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) st_cluster(dst + e * TM * 4, v[e]);
      }
      cluster_sync_all();
#pragma unroll 1
      for (int q = 0; !bad; ++q) {
        const int c = tile_column(S, rank, half, q);
        if (c >= p.nt || n0 + c >= p.N) break;
        float f[8] = {};
        if (used) tc_ld8(taddr + p.nt + c, f);
        const float* part = reinterpret_cast<const float*>(smem) + ((c >> 3) / S * 8) * TM + row;
#pragma unroll 2
        for (int k = 0; k < S; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += part[(k * G * 8 + e) * TM];
        emit<AMN, EPI, 8>(p, z, m, n0 + c, f, mirror, false);
        __syncwarp();
      }
    }
    if constexpr (OUT) {
      // an index that names no adapter (the status word has long been cleared)
      const int t = n0 + (int)threadIdx.x - 64;
      if (p.n_adapters > 0 && tm == 0 && rank == 0 && t < min(n0 + p.nt, p.N) && p.index[t] != -1 &&
          valid_adapter(p, t) < 0)
        atomicCAS(p.status, 0, (int)THANOS_ERR_INVALID_ARG);
    }
  }
  if (S > 1 && warp < 2) {
    __syncwarp();
    cluster_sync_all();
    cluster_sync_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                 "r"(p.tmem_cols)
                 : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(p.status, 0, (int)THANOS_ERR_TIMEOUT);
}

// ------------------------------------------------------------------------------- CTA pairs
// The same product on a persistent cluster of two CTAs with tcgen05.mma.cta_group::2: tiles of 256 x
// nt, CTA r holds rows 128 r .. +127 in its tensor memory and loads only those and half of the n
// rows, so an SM moves 32 KB instead of 48 KB through shared memory per 64-wide k step of a 256-wide
// tile.  Two accumulators: the epilogue of a tile runs beside the next tile's products.
//
// Adapter part (PROJ_OUT): for every adapter that occurs in the token tile, k is extended by its rank
// in chunks of 16, two to a stage, in a ring of their own that four more warps fill a tile
// ahead: the wide factor's rows come by TMA (32-byte swizzle; MN-major: 128-byte), the factor of the
// tokens, s_i V[t], is built as two bf16 planes with zero rows for tokens of other adapters.  (One
// plane would give a token a result in a large batch that is 2^-9 of the adapter part off what it gets
// in a small one.  The second costs 1 to 2 % where a tile has few adapters, 8 % with 16 adapters mixed
// token by token, 12 % at rank 128.)  0 times a
// non-finite weight would reach those tokens, so the chunk is scanned, non-finite weights become
// zeros and the epilogue adds their products to the adapter's own tokens.
//
// Bound by the tensor cores and the power cap.  4096 tokens, 4096 x 4096, 7 adapters of rank 32: 117 us
// with the skinny product, 1.19 PFLOP/s (256 tiles are 3.46 rounds of 74 pairs; 107 us and 69 % of the
// tensor cycles in this kernel alone, cold).  8192 x 11008 x 4096: 1.3 PFLOP/s of 1.43 sustained.
constexpr int PTM = 256;
constexpr int PSTAGE_BYTES = 2 * A_BYTES;
constexpr int CHUNK_BYTES = TM * 16 * 2;      // a 16-wide chunk of an adapter's wide factor
constexpr int EPLANE_BYTES = 128 * 16 * 2;    // a plane of the tokens' factors
constexpr int CHUNKS = 2;                     // chunks per stage
constexpr int ESTAGES = 2;
constexpr int FACTORS = CHUNKS * CHUNK_BYTES; // offset of the factors in a stage
__host__ __device__ constexpr int pair_stages(int epi) { return epi == PROJ_OUT ? 5 : 7; }
__host__ __device__ constexpr int pair_threads(int epi) { return epi == PROJ_OUT ? 448 : 320; }
constexpr size_t PSMEM_BYTES = (size_t)7 * PSTAGE_BYTES + 1024 + 512;
static_assert(pair_stages(PROJ_OUT) + ESTAGES == 7 &&
                  FACTORS + 2 * CHUNKS * EPLANE_BYTES <= PSTAGE_BYTES,
              "shared memory of the rings");

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map,
                                                 uint32_t lead_bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(lead_bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}

struct PairTile {
  int z, tm, tn;
};
// Tiles by groups of eight columns, rows inside: the pairs that run at the same time share the
// operands of about 8 x 9 tiles, which L2 holds.
__device__ __forceinline__ PairTile pair_tile(const Params& p, int t) {
  PairTile r;
  if (p.symmetric) {
    const int per = p.tiles_m * (p.tiles_m + 1) / 2;
    r.z = t / per;
    int u = t - r.z * per, col = 0;
    while (u > col) {  // column col of the triangle has col + 1 tiles
      u -= col + 1;
      ++col;
    }
    r.tm = u;
    r.tn = col;
    return r;
  }
  const int per = p.tiles_m * p.tiles_n;
  r.z = t / per;
  int u = t - r.z * per;
  const int group = u / (8 * p.tiles_m);
  u -= group * 8 * p.tiles_m;
  const int wide = min(8, p.tiles_n - 8 * group);
  r.tm = u / wide;
  r.tn = 8 * group + (u - r.tm * wide);
  return r;
}

template <bool AMN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(EPI), 1)
pair_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
            const __grid_constant__ CUtensorMap mapP, const Params p, const int n_tiles) {
  constexpr bool EXT = EPI == PROJ_OUT;
  constexpr int STAGES = pair_stages(EPI);
  constexpr int EPI_WARP = EXT ? 6 : 2;       // first of the eight epilogue warps
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ering = smem + (size_t)STAGES * PSTAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)7 * PSTAGE_BYTES);
  // full (used in the first CTA), empty (STAGES each); accumulator full, accumulator empty (first
  // CTA); adapter stage: chunks landed, ready (first CTA), empty
  constexpr int B_TFULL = 2 * STAGES, B_EXT = B_TFULL + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + B_EXT + 3 * ESTAGES);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + B_EXT + 3 * ESTAGES + 1);
  int* poison = reinterpret_cast<int*>(bars + B_EXT + 3 * ESTAGES + 2);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const uint32_t smem_base = smem_u32(smem);
  const uint32_t ering_base = smem_u32(ering);
  const uint32_t bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  auto tfull_bar = [&](int q) { return bar_base + 8u * (B_TFULL + q); };
  auto tempty_bar = [&](int q) { return bar_base + 8u * (B_TFULL + 2 + q); };
  auto land_bar = [&](int e) { return bar_base + 8u * (B_EXT + e); };
  auto ready_bar = [&](int e) { return bar_base + 8u * (B_EXT + ESTAGES + e); };
  auto eempty_bar = [&](int e) { return bar_base + 8u * (B_EXT + 2 * ESTAGES + e); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int q = 0; q < 2; ++q) {
      mbar_init(tfull_bar(q), 1);
      mbar_init(tempty_bar(q), 16);  // eight epilogue warps in each CTA
    }
    for (int e = 0; e < ESTAGES; ++e) {
      mbar_init(land_bar(e), 1);
      mbar_init(ready_bar(e), 8);    // four warps in each CTA
      mbar_init(eempty_bar(e), 1);
    }
    *abort_flag = 0;
    *poison = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // both CTAs' barriers are initialised before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (!p.early) grid_dependency_wait();
  grid_dependents_launch();

  const int nk = (p.K + BK - 1) / BK;
  const int planes = !EXT && p.fine ? 2 : 1;  // stages of a k step: hi planes, then lo planes
  const int half = p.nt / 2;  // n rows that this CTA loads
  const bool ext = EXT && p.n_adapters > 0;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (elect_one()) {
    int s = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += npairs) {
      const PairTile tl = pair_tile(p, t);
      const int m0 = tl.tm * PTM + 128 * (int)rank, n0 = tl.tn * p.nt + half * (int)rank;
      for (int u = 0; u < planes * nk && ok; ++u) {
        ok = mbar_wait(empty_bar(s), phase ^ 1u, abort_flag);
        if (ok) {
          const int kb = (planes == 2 ? u >> 1 : u) * BK;
          const int slab = tl.z + (planes == 2 && (u & 1) ? p.batch_z : 0);
          const uint32_t dst = smem_base + (uint32_t)s * PSTAGE_BYTES;
          const uint32_t lead = map_to_cta(full_bar(s), 0);
          if (rank == 0) mbar_expect_tx(full_bar(s), 2 * (A_BYTES + half * BK * 2));
          if (AMN) {
            tma_load_3d_pair(dst, &mapA, lead, m0, kb, slab);
            tma_load_3d_pair(dst + A_BYTES / 2, &mapA, lead, m0 + 64, kb, slab);
          } else {
            tma_load_3d_pair(dst, &mapA, lead, kb, m0, slab);
          }
          tma_load_3d_pair(dst + A_BYTES, &mapB, lead, kb, n0, slab);
        }
        if (++s == STAGES) {
          s = 0;
          phase ^= 1u;
        }
      }
      // The products of the next tile wait for this one's adapter stages, and those for the launch
      // before, which may take long (the sort of all tokens, on one CTA): no bounded wait spans it.
      if (ext && t == pair) grid_dependency_wait();
    }
    // let copies that are still in flight land before the CTA's shared memory goes away
    if (!ok) {
      for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (first CTA only)
    if (rank == 0 && elect_one()) {
      uint32_t idesc = 0;
      idesc |= 1u << 4;  // D fp32
      if (!p.f16) idesc |= (1u << 7) | (1u << 10);
      if (AMN) idesc |= 1u << 15;
      idesc |= (uint32_t)(p.nt >> 3) << 17;
      idesc |= (uint32_t)(PTM >> 4) << 24;
      const uint64_t ad0 = AMN ? make_desc(smem_base, A_BYTES / 2, 1024, SW128)
                               : make_desc(smem_base, 16, 1024, SW128);
      const uint64_t bd0 = make_desc(smem_base + A_BYTES, 16, 1024, SW128);
      int s = 0, q = 0, e = 0;
      uint32_t phase = 0, tphase = 0, ephase = 0;
      bool ok = true, waited = false;
      for (int t = pair; t < n_tiles && ok; t += npairs) {
        const PairTile tl = pair_tile(p, t);
        ok = mbar_wait(tempty_bar(q), tphase ^ 1u, abort_flag);
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)q * 256;
        for (int ks = 0; ks < nk && ok; ++ks) {
          ok = mbar_wait(full_bar(s), phase, abort_flag);
          tc_fence_after();
          const uint64_t at = (uint64_t)s * (PSTAGE_BYTES >> 4);
          const uint32_t add = ks > 0 ? 1u : 0u;
          if (!EXT && planes == 2) {
            const int s_hi = s;
            if (++s == STAGES) {
              s = 0;
              phase ^= 1u;
            }
            ok = ok && mbar_wait(full_bar(s), phase, abort_flag);
            tc_fence_after();
            if (ok) {
              const uint64_t lo = (uint64_t)s * (PSTAGE_BYTES >> 4);
              mma_step<AMN, true>(d, ad0 + at, bd0 + lo, idesc, add);
              mma_step<AMN, true>(d, ad0 + lo, bd0 + at, idesc, 1u);
              mma_step<AMN, true>(d, ad0 + at, bd0 + at, idesc, 1u);
              tc_commit_pair(empty_bar(s_hi));
              tc_commit_pair(empty_bar(s));
            }
          } else if (ok) {
            mma_step<AMN, true>(d, ad0 + at, bd0 + at, idesc, add);
            tc_commit_pair(empty_bar(s));
          }
          if (++s == STAGES) {
            s = 0;
            phase ^= 1u;
          }
        }
        if (ext && ok) {
          if (!waited) grid_dependency_wait();
          waited = true;
          const int total = p.tile_count[tl.tn] * p.chunks;
          for (int c0 = 0; c0 < total && ok; c0 += CHUNKS) {
            ok = mbar_wait(ready_bar(e), ephase, abort_flag);
            tc_fence_after();
            if (ok) {
              const uint32_t st = ering_base + (uint32_t)e * PSTAGE_BYTES;
              const int nc = min(CHUNKS, total - c0);
              for (int c = 0; c < nc; ++c) {
                const uint32_t sa = st + c * CHUNK_BYTES, sb = st + FACTORS + 2 * c * EPLANE_BYTES;
                const uint64_t ad = AMN ? make_desc(sa, CHUNK_BYTES / 2, 1024, SW128)
                                        : make_desc(sa, 16, 256, SW32);
                tc_mma_bf16_pair(d, ad, make_desc(sb, 16, 256, SW32), idesc, 1u);
                tc_mma_bf16_pair(d, ad, make_desc(sb + EPLANE_BYTES, 16, 256, SW32), idesc, 1u);
              }
              tc_commit_pair(eempty_bar(e));
            }
            if (++e == ESTAGES) {
              e = 0;
              ephase ^= 1u;
            }
          }
        }
        if (ok) tc_commit_pair(tfull_bar(q));
        if (++q == 2) {
          q = 0;
          tphase ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp < EPI_WARP) {
    // ------------------------------------------------------------ adapter stages
    if (ext) {
      grid_dependency_wait();
      const int row = threadIdx.x - 64;  // the token row of this thread, warps 2..5
      int e = 0;
      uint32_t ephase = 0;
      bool ok = true;
      // Thread 64 brings the wide factors, ahead of the stage that is worked on as far as the ring is
      // free: what follows ranks ij.. of the iat-th adapter of tile it goes to slot ie next.
      int ahead = 0, it = pair, iat = 0, ij = 0, icount = 0, im0 = 0, ie = 0;
      const int32_t* ilist = nullptr;
      uint32_t iphase = 0;
      auto open_tile = [&]() {  // the next tile with adapters, from `it` on
        for (; it < n_tiles; it += npairs) {
          const PairTile tl = pair_tile(p, it);
          icount = p.tile_count[tl.tn];
          if (icount == 0) continue;
          im0 = tl.tm * PTM + 128 * (int)rank;
          ilist = p.tile_list + (int64_t)tl.tn * p.nt;
          return;
        }
      };
      auto bring = [&](bool is_free) {
        if (it >= n_tiles || !(is_free || mbar_test(eempty_bar(ie), iphase ^ 1u))) return false;
        const int nc = min(CHUNKS, (icount - iat) * p.chunks - (ij >> 4));
        mbar_expect_tx(land_bar(ie), nc * CHUNK_BYTES);
        uint32_t dst = ering_base + (uint32_t)ie * PSTAGE_BYTES;
        for (int q = 0; q < nc; ++q, dst += CHUNK_BYTES) {
          const int who = ilist[iat];
          if (AMN) {
            tma_load_3d(dst, &mapP, land_bar(ie), im0, ij, who);
            tma_load_3d(dst + CHUNK_BYTES / 2, &mapP, land_bar(ie), im0 + 64, ij, who);
          } else {
            tma_load_3d(dst, &mapP, land_bar(ie), ij, im0, who);
          }
          ij += 16;
          if (ij >= p.r) {
            ij = 0;
            ++iat;
          }
        }
        if (++ie == ESTAGES) {
          ie = 0;
          iphase ^= 1u;
        }
        if (iat == icount) {
          iat = 0;
          it += npairs;
          open_tile();
        }
        return true;
      };
      if (threadIdx.x == 64) open_tile();
      __syncwarp();
      for (int t = pair; t < n_tiles && ok; t += npairs) {
        const PairTile tl = pair_tile(p, t);
        const int tok = tl.tn * p.nt + half * (int)rank + row;
        const int mine = row < half && tok < p.N ? valid_adapter(p, tok) : -1;
        const float sc = mine >= 0 && p.scale ? p.scale[mine] : 1.f;
        const int count = p.tile_count[tl.tn], total = count * p.chunks;
        const int32_t* list = p.tile_list + (int64_t)tl.tn * p.nt;
        float v0[16];                    // the token's first sixteen ranks, all of them up to rank 16
        if (count > 0 && mine >= 0) token_factor(p, tok, sc, 0, v0);
        int j0 = 0, at = 0, seen = 0;    // the next chunk: ranks j0.. of the at-th adapter of the tile
        for (int c0 = 0; c0 < total; c0 += CHUNKS) {
          const int nc = min(CHUNKS, total - c0);
          // the factors of the stage's chunks, loaded while the stage before is on its way
          uint32_t hi[CHUNKS][8] = {}, lo[CHUNKS][8] = {};
#pragma unroll
          for (int q = 0; q < CHUNKS; ++q) {
            if (j0 == 0 && (at & 31) == 0) seen = at + lane < count ? list[at + lane] : -1;
            const int who = __shfl_sync(0xffffffffu, seen, at & 31);
            if (q < nc && who == mine) {
              if (j0 == 0) {
                factor_planes(v0, hi[q], lo[q]);
              } else {
                float v[16];
                token_factor(p, tok, sc, j0, v);
                factor_planes(v, hi[q], lo[q]);
              }
            }
            j0 += 16;
            if (j0 >= p.r) {
              j0 = 0;
              ++at;
            }
          }
          ok = mbar_wait_warp(eempty_bar(e), ephase ^ 1u, abort_flag);
          if (!ok) break;
          if (threadIdx.x == 64) {
            if (ahead == 0 && bring(true)) ++ahead;
            while (ahead < ESTAGES && bring(false)) ++ahead;
            --ahead;
          }
          __syncwarp();
          unsigned char* st = ering + (size_t)e * PSTAGE_BYTES;
#pragma unroll
          for (int q = 0; q < CHUNKS; ++q) {
            if (q >= nc) break;
            // 32-byte rows, 32-byte swizzle: the 16-byte halves swap every four rows
            unsigned char* fac = st + FACTORS + (size_t)(2 * q) * EPLANE_BYTES + row * 32;
            const int sw = ((row >> 2) & 1) << 4;
            *reinterpret_cast<uint4*>(fac + sw) = make_uint4(hi[q][0], hi[q][1], hi[q][2], hi[q][3]);
            *reinterpret_cast<uint4*>(fac + (16 ^ sw)) =
                make_uint4(hi[q][4], hi[q][5], hi[q][6], hi[q][7]);
            fac += EPLANE_BYTES;
            *reinterpret_cast<uint4*>(fac + sw) = make_uint4(lo[q][0], lo[q][1], lo[q][2], lo[q][3]);
            *reinterpret_cast<uint4*>(fac + (16 ^ sw)) =
                make_uint4(lo[q][4], lo[q][5], lo[q][6], lo[q][7]);
          }
          ok = mbar_wait_warp(land_bar(e), ephase, abort_flag);
          if (!ok) break;
          for (int q = row; q < nc * (CHUNK_BYTES / 16); q += 128)
            clean_vector(reinterpret_cast<uint4*>(st) + q, poison);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(ready_bar(e), 0));
          if (++e == ESTAGES) {
            e = 0;
            ephase ^= 1u;
          }
        }
      }
      if (!ok) {  // as above: chunks in flight
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue
    const int g = warp & 3, h = (warp - EPI_WARP) >> 2;
    const uint32_t lead_tempty = map_to_cta(tempty_bar(0), 0);
    if (p.early) grid_dependency_wait();
    int q = 0;
    uint32_t tphase = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles; t += npairs) {
      const PairTile tl = pair_tile(p, t);
      ok = ok && mbar_wait_warp(tfull_bar(q), tphase, abort_flag);
      tc_fence_after();
      if (ok) {
        const int n0 = tl.tn * p.nt;
        const int m = tl.tm * PTM + 128 * (int)rank + 32 * g + lane;
        if (ext && tl.tm == 0 && rank == 0) {
          for (int u = n0 + (int)threadIdx.x - 32 * EPI_WARP; u < min(n0 + p.nt, p.N); u += 256)
            if (p.index[u] != -1 && valid_adapter(p, u) < 0)
              atomicCAS(p.status, 0, (int)THANOS_ERR_INVALID_ARG);
        }
        const bool poisoned = ext && *(volatile int*)poison != 0;
        const uint32_t taddr = tmem_base + ((uint32_t)(32 * g) << 16) + (uint32_t)q * 256;
        if constexpr (EPI == PROJ_FINAL) {  // its operands leave room for half as many columns
#pragma unroll 1
          for (int cc = 16 * h; cc < p.nt; cc += 32) {
            float v[16];
            tc_ld16(taddr + cc, v);
            emit<AMN, EPI, 16>(p, tl.z, m, n0 + cc, v, false, false);
            __syncwarp();  // lanes beyond the last row have left emit() early
          }
        } else {
#pragma unroll 1
          for (int cc = 32 * h; cc < p.nt; cc += 64) {
            uint32_t u[32];
            tc_ld32(taddr + cc, u);
            tc_wait_ld();
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
            emit<AMN, EPI, 32>(p, tl.z, m, n0 + cc, v, tl.tm != tl.tn, poisoned);
            __syncwarp();
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(lead_tempty + 8u * q);
      if (++q == 2) {
        q = 0;
        tphase ^= 1u;
      }
    }
  }

  // Neither CTA may leave (or free tensor memory) while its partner can still read its shared
  // memory, signal its barriers or write its tensor memory.
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512)
                 : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(p.status, 0, (int)THANOS_ERR_TIMEOUT);
}

bool make_map3(CUtensorMap* map, const void* base, bool f16, int64_t inner, int64_t rows, int64_t ld,
               int64_t batch, int64_t batch_stride, int box_inner, int box_rows,
               CUtensorMapSwizzle swizzle) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  if (batch_stride <= 0) batch_stride = ld;  // never stepped over when it has one entry
  cuuint64_t gdim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch};
  cuuint64_t gstr[2] = {(cuuint64_t)ld * 2, (cuuint64_t)batch_stride * 2};
  cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
             const_cast<void*>(base), gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool AMN, int EPI>
thanos_status_t launch(const CUtensorMap& mA, const CUtensorMap& mB, const Params& p,
                       cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  THANOS_CUDA(ensure_max_dyn_smem(tile_kernel<AMN, EPI>, 227 * 1024, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.tiles_m * p.tiles_n * p.splits), (unsigned)p.batch_z, 1);
  cfg.blockDim = dim3(TILE_THREADS, 1, 1);
  cfg.dynamicSmemBytes = (size_t)p.ring_bytes + FACTOR_BYTES + 512 /*ids*/ + 256 /*barriers*/ + 1024;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.first ? 1 : 2;   // what runs beside a first launch relies on its plain start
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, tile_kernel<AMN, EPI>, mA, mB, p));
  return THANOS_OK;
}

template <bool AMN, int EPI>
int max_active_pairs() {
  static std::atomic<int> cached_by_dev[64];  // 0 = not asked yet, else pairs + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  const int have = cached_by_dev[dev].load(std::memory_order_relaxed);
  if (have > 0) return have - 1;
  if (cudaFuncSetAttribute(pair_kernel<AMN, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)PSMEM_BYTES) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * sm_count(), 1, 1);
  cfg.blockDim = dim3(pair_threads(EPI), 1, 1);
  cfg.dynamicSmemBytes = PSMEM_BYTES;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, pair_kernel<AMN, EPI>, &cfg) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    n = 0;
  }
  cached_by_dev[dev].store(n + 1, std::memory_order_relaxed);
  return n;
}

template <bool AMN, int EPI>
thanos_status_t launch_pair(const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mP,
                            const Params& p, cudaStream_t stream) {
  const int G = max_active_pairs<AMN, EPI>();
  if (G < 1) return THANOS_ERR_CUDA;
  const int64_t per = p.symmetric ? (int64_t)p.tiles_m * (p.tiles_m + 1) / 2
                                  : (int64_t)p.tiles_m * p.tiles_n;
  const int64_t tiles = per * p.batch_z;
  if (tiles > (1 << 30)) return THANOS_ERR_SHAPE;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * (tiles < G ? tiles : G)), 1, 1);
  cfg.blockDim = dim3(pair_threads(EPI), 1, 1);
  cfg.dynamicSmemBytes = PSMEM_BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, pair_kernel<AMN, EPI>, mA, mB, mP, p, (int)tiles));
  return THANOS_OK;
}

template <bool AMN, int EPI>
thanos_status_t launch_any(bool pairs, const CUtensorMap& mA, const CUtensorMap& mB,
                           const CUtensorMap& mP, const Params& p, cudaStream_t stream) {
  return pairs ? launch_pair<AMN, EPI>(mA, mB, mP, p, stream)
               : launch<AMN, EPI>(mA, mB, p, stream);
}

// Whether a product runs on CTA pairs: once its 256 x 256 tiles occupy at least half of the pairs (512
// tokens, K = 4096: 32 tiles take 37 us on lone CTAs and 41 on pairs, 36 tiles 43 and 41; 64 tiles of
// 1024 tokens 52 and 47).
bool use_pairs(int64_t M, int64_t N, int64_t batch, bool symmetric) {
  const int64_t tm = ceil_div(M, PTM), tn = ceil_div(N, PTM);
  const int64_t tiles = (symmetric ? tm * (tm + 1) / 2 : tm * tn) * batch;
  return M > TM && N > TM && tiles * 4 >= sm_count();
}

}  // namespace

namespace {
// Width and k slices of tile_kernel's tiles, by the clocks that the busiest SM takes, as measured on
// 768 x 768 products and on single tokens.  Elsewhere the choice is up to a fifth off the best (16
// tokens, 2048 x 2048: 12.4 us with 8 slices, 10.3 with 2; 333 tokens, 1001 x 1752: 19.6 and 17.2; 200
// and 500 tokens: the best).  Clusters of 5 and 7 are no worse than their neighbours here (64 tokens,
// 4096 x 11008: 5 slices 30.6 us, 7 30.1, 8 30.0).
//   a k step     what it brings in at 60 bytes per clock, at least 250 (issue and barriers)
//   a CTA        2000 to start, 400 for eight columns of its epilogue (700 with operands to read)
//   a cluster    1500, and 44 a column for the partial sums over distributed shared memory, more with
//                more slices
// Up to 64 tokens of a projection stay in one tile, so that the weights are read once.  A k block takes
// `loads` stages; six of them are three planes, whose products stay with the slice of their block.  The
// tensor cores cut what they add to an accumulator, so an fp32 product's k goes to slices of at most 16
// blocks as far as eight slices go (64 additions of full size; K = 2048 in two slices: 1.0e-6 of the
// result, in four 4.8e-7; the second slice costs 2000 x 2048 x 2048 a tenth of its time).
struct TileShape {
  int nt, splits;
};
TileShape tile_shape(int64_t M, int64_t N, int64_t batch, int64_t blocks, int loads, bool symmetric,
                     int epi) {
  const int64_t sms = sm_count(), tm = ceil_div(M, TM);
  const bool one_tile = (epi == PROJ_OUT || epi == PROJ_OUT32) && N <= 64;
  const double column = epi >= PROJ_POLY && epi <= PROJ_FINAL ? 700.0 : 400.0;
  TileShape best = {128, 1};
  double least = 0.0;
  const int64_t unit = loads >= 3 ? loads : 1, parts = blocks * loads / unit;
  const int64_t most = loads >= 3 ? blocks : parts / 4;   // slices that the work is enough for
  const int64_t need = epi == PROJ_OUT32 ? ceil_div(blocks, 16) : 1;
  for (int nt = 128; nt >= 32; nt /= 2) {
    if (nt > 32 && N <= nt / 2) continue;   // the next narrower one holds all of N
    if (one_tile && N > nt) break;
    int64_t tiles = tm * ceil_div(N, nt) * batch;
    if (symmetric) tiles = (tiles + tm * batch * (TM / nt)) / 2;
    const double step = fmax(250.0, (A_BYTES + nt * BK * 2) / 60.0);
    for (int s = need < 8 ? (int)need : 8; s <= 8 && (s == 1 || s <= most); ++s) {
      const double load = (double)(tiles * s) / (double)sms;
      const double rounds = load <= 1.0 ? 1.0 : two_per_sm(epi) && load <= 2.0 ? load : ceil(load);
      double cta = (double)(ceil_div(parts, s) * unit) * step + 2000.0 + column * (double)ceil_div(nt, 16 * s);
      if (s > 1) cta += 1500.0 + 44.0 * nt * (1.0 + s / 8.0);
      if (least == 0.0 || rounds * cta < least) {
        least = rounds * cta;
        best = {nt, s};
      }
    }
  }
  return best;
}
}  // namespace

// Terms that an entry of S sums in one accumulator for fp32 weights; a longer k goes in pieces, each
// added to what is there.  The tensor cores cut what they add, of the squares on the diagonal always in
// one direction (2048 x 20000, 65536: 1.8e-4, 2.3e-4 of the update, 4096 x 65536: 3.8e-4; in pieces of 4096
// 2e-5, but 4096 x 11008, 4.5e-5 in one, then took 9.1 ms instead of 7.3).
constexpr int64_t LONGEST_GRAM = 16384;

int proj_pair_tile(int64_t N, int64_t M) { return use_pairs(M, N, 1, false) ? PTM : 0; }

thanos_status_t proj_gemm(const ProjArgs& a, cudaStream_t stream) {
  if (a.M <= 0 || a.N <= 0 || a.batch <= 0) return THANOS_OK;
  if (a.lda % 8 || a.ldb % 8 || a.a_batch % 8 || a.b_batch % 8 || !aligned16(a.A) || !aligned16(a.B))
    return THANOS_ERR_ALIGNMENT;
  const bool symmetric = a.epi == PROJ_GRAM || a.epi == PROJ_GRAM_ADD || a.epi == PROJ_POLY;
  Params p = {};
  p.M = a.M;
  p.N = a.N;
  p.K = a.K;
  const bool f32 = a.epi >= PROJ_OUT32;
  const bool pairs = a.epi != PROJ_SHRINK && !f32 && use_pairs(a.M, a.N, a.batch, symmetric);
  const TileShape shape =
      pairs ? TileShape{PTM, 1} : tile_shape(a.M, a.N, a.batch, ceil_div(a.K, BK), f32 ? (a.one_plane ? 3 : 6) : a.fine ? 2 : 1,
                                                 symmetric, a.epi);
  if (a.epi == PROJ_GRAM && a.fine && ceil_div(a.K, shape.splits) > LONGEST_GRAM) {
    const int64_t pieces = ceil_div(ceil_div(a.K, shape.splits), LONGEST_GRAM), blocks = ceil_div(a.K, BK);
    for (int64_t i = 0; i < pieces; ++i) {
      const int64_t k0 = BK * (blocks * i / pieces), k1 = BK * (blocks * (i + 1) / pieces);
      ProjArgs s = a;
      s.A = static_cast<const __half*>(a.A) + k0;
      s.B = static_cast<const __half*>(a.B) + k0;
      s.K = (int)((k1 < a.K ? k1 : a.K) - k0);
      if (i > 0) s.epi = PROJ_GRAM_ADD;
      THANOS_TRY(proj_gemm(s, stream));
    }
    return THANOS_OK;
  }
  p.nt = shape.nt;
  p.splits = shape.splits;
  p.tiles_m = (a.M + (pairs ? PTM : TM) - 1) / (pairs ? PTM : TM);
  p.tiles_n = (a.N + p.nt - 1) / p.nt;
  p.batch_z = a.batch;
  p.products = a.one_plane ? 3 : 6;
  p.symmetric = symmetric;
  p.f16 = a.f16;
  p.early = a.early;
  p.first = a.first;
  p.fine = a.fine;
  p.add = a.add;
  p.status = a.status;
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * a.batch;
  if (tiles > (1 << 27) || a.batch > 65535) return THANOS_ERR_SHAPE;
  const int stage_bytes = A_BYTES + p.nt * BK * 2;
  p.stages = (two_per_sm(a.epi) ? 100 : 200) * 1024 / stage_bytes;
  if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
  p.ring_bytes = p.stages * stage_bytes;
  // the adapter part sits beside the sums; the skinny product has two accumulators
  p.tmem_cols = two_per_sm(a.epi) ? 2 * p.nt : p.nt;
  p.out = a.out;
  p.ldo = a.ldo;
  p.V = a.V;
  p.planes = a.planes;
  p.skinny = static_cast<const __nv_bfloat16*>(a.skinny);
  p.x = static_cast<const __nv_bfloat16*>(a.B);
  p.ld_tok = a.ldb;
  p.index = a.index;
  p.scale = a.scale;
  p.n_adapters = a.n_adapters;
  p.r = a.r;
  p.chunks = (a.r + 15) / 16;
  p.tile_count = a.tile_count;
  p.tile_list = a.tile_list;
  p.P = static_cast<const __nv_bfloat16*>(a.P);
  p.ldp = a.ldp;
  p.p_adapter = a.p_adapter;
  p.alpha = a.alpha;
  p.beta = a.beta;
  p.S = a.S;
  p.lds = a.lds;
  p.s_batch = a.s_batch;
  p.Pm = a.Pm;
  p.s_diag = a.s_diag;
  p.p_diag = a.p_diag;
  p.Xh = a.Xh;
  p.Xl = a.Xl;
  p.Yh = a.Yh;
  p.Yl = a.Yl;
  p.ldx = a.ldx;
  p.x_batch = a.x_batch;
  p.O = a.O;
  p.W_out = a.W_out;
  p.W_in = a.W_in;
  p.mask = a.mask;
  p.w_bf16 = a.w_bf16;
  p.tall = a.tall;
  p.keep = a.keep;
  p.rate = a.rate;

  CUtensorMap mA, mB, mP;
  const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
  const int64_t slabs = f32 ? 3 : a.fine ? 2 * a.batch : a.batch, slabs_a = a.one_plane ? 1 : slabs;
  const bool okA = a.a_mn ? make_map3(&mA, a.A, a.f16, a.M, a.K, a.lda, slabs_a, a.a_batch, 64, BK, sw)
                          : make_map3(&mA, a.A, a.f16, a.K, a.M, a.lda, slabs_a, a.a_batch, BK, TM, sw);
  if (!okA || !make_map3(&mB, a.B, a.f16, a.K, a.N, a.ldb, slabs, a.b_batch, BK,
                         pairs ? p.nt / 2 : p.nt, sw))
    return THANOS_ERR_CUDA;
  mP = mA;
  if (pairs && a.epi == PROJ_OUT && a.n_adapters > 0) {
    if (a.ldp % 8 || a.p_adapter % 8 || !aligned16(a.P)) return THANOS_ERR_ALIGNMENT;
    const bool ok =
        a.a_mn ? make_map3(&mP, a.P, false, a.M, a.r, a.ldp, a.n_adapters, a.p_adapter, 64, 16, sw)
               : make_map3(&mP, a.P, false, a.r, a.M, a.ldp, a.n_adapters, a.p_adapter, 16, TM,
                           CU_TENSOR_MAP_SWIZZLE_32B);
    if (!ok) return THANOS_ERR_CUDA;
  }
  switch (a.epi) {
    case PROJ_OUT:
      return a.a_mn ? launch_any<true, PROJ_OUT>(pairs, mA, mB, mP, p, stream)
                    : launch_any<false, PROJ_OUT>(pairs, mA, mB, mP, p, stream);
    case PROJ_OUT32:
      return a.a_mn ? launch<true, PROJ_OUT32>(mA, mB, p, stream)
                    : launch<false, PROJ_OUT32>(mA, mB, p, stream);
    case PROJ_SHRINK:
      return launch<false, PROJ_SHRINK>(mA, mB, p, stream);
    case PROJ_SHRINK32:
      return launch<false, PROJ_SHRINK32>(mA, mB, p, stream);
    case PROJ_GRAM:
      return launch_any<false, PROJ_GRAM>(pairs, mA, mB, mP, p, stream);
    case PROJ_GRAM_ADD:
      return launch_any<false, PROJ_GRAM_ADD>(pairs, mA, mB, mP, p, stream);
    case PROJ_POLY:
      return launch_any<false, PROJ_POLY>(pairs, mA, mB, mP, p, stream);
    case PROJ_NEXT:
      return launch_any<true, PROJ_NEXT>(pairs, mA, mB, mP, p, stream);
    default:
      return launch_any<true, PROJ_FINAL>(pairs, mA, mB, mP, p, stream);
  }
}

}  // namespace thanos
