// The orthogonalised update: Newton-Schulz iteration X <- a X + (b S + c S S) X, S = X X^T, on the
// shorter side of each matrix, and the optimiser step around it.
//
// Operands of the products are fp16 (11 significant bits: an eighth of bf16's rounding at the same
// rate); powers of two keep the entries of X, S and P = b S + c S S near one, so nothing becomes
// subnormal.  X itself is carried as two fp16 planes hi + lo (22 bits) through the term a X, which
// is the one that amplifies: directions with small singular values grow by a = 3.4 a step, and a
// rounding of X that mixes a strong direction into them grows too (on a low-rank gradient with
// noise 1e-1 of the result with hi alone, 2e-4 with both).  The product P X reads hi only: P acts
// on the strong directions, whose rounding errors are not amplified.
#include "proj_gemm.cuh"
#include "recovery.cuh"

namespace thanos {
namespace {

constexpr int MAX_PARTS = 1024;  // partial sums of squares per matrix

__device__ __forceinline__ float load_any(const void* p, int bf16, int64_t e) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[e])
              : static_cast<const float*>(p)[e];
}

struct StepParams {
  const void* G;
  float* M_out;
  const float* M_in;
  const uint8_t* mask;
  int32_t* status;
  double* part;
  int parts;
  int g_bf16, nesterov, tall;
  float momentum, eps, unit;
  int m, n;
  __half* Xh;
  __half* Xl;
  int64_t ldx, x_batch;
};

__device__ __forceinline__ double block_sum(double v, double* red) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < 8; ++w) s += red[w];
  return s;
}

// The iteration's input at one element; `mo` is the new momentum.
__device__ __forceinline__ float update_of(const StepParams& p, int64_t e, float mo) {
  if (p.mask && p.mask[e] != 0) return 0.f;
  if (!p.M_out) return load_any(p.G, p.g_bf16, e);
  return p.nesterov ? fmaf(p.momentum, mo, load_any(p.G, p.g_bf16, e)) : mo;
}

template <int VEC>
__device__ __forceinline__ void load_vec(const void* p, int bf16, int64_t e, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = load_any(p, bf16, e);
  } else if (bf16) {
    const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + e);
    v[0] = __uint_as_float(q.x << 16);
    v[1] = __uint_as_float(q.x & 0xFFFF0000u);
    v[2] = __uint_as_float(q.y << 16);
    v[3] = __uint_as_float(q.y & 0xFFFF0000u);
  } else {
    const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + e);
    v[0] = q.x;
    v[1] = q.y;
    v[2] = q.z;
    v[3] = q.w;
  }
}

// VEC consecutive elements of the iteration's input; FIRST reads the old momentum and writes the
// new one, else the new one is read.
template <int VEC, bool FIRST>
__device__ __forceinline__ void update_vec(const StepParams& p, int64_t at, float (&v)[VEC]) {
  uint32_t gone = 0;
  if (p.mask) {
    if constexpr (VEC == 4) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(p.mask + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) gone |= ((w >> (8 * e)) & 0xFFu ? 1u : 0u) << e;
    } else {
      gone = p.mask[at] != 0;
    }
  }
  float g[VEC];
  if (FIRST || !p.M_out || p.nesterov) load_vec<VEC>(p.G, p.g_bf16, at, g);
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    if ((gone >> e) & 1u) g[e] = 0.f;
    v[e] = g[e];
  }
  if (!p.M_out) return;
  float mo[VEC];
  if (FIRST) {
    load_vec<VEC>(p.M_in, 0, at, mo);
#pragma unroll
    for (int e = 0; e < VEC; ++e) mo[e] = fmaf(p.momentum, mo[e], g[e]);
    if constexpr (VEC == 4) *reinterpret_cast<float4*>(p.M_out + at) = make_float4(mo[0], mo[1], mo[2], mo[3]);
    else p.M_out[at] = mo[0];
  } else {
    load_vec<VEC>(p.M_out, 0, at, mo);
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    v[e] = (gone >> e) & 1u ? 0.f : p.nesterov ? fmaf(p.momentum, mo[e], g[e]) : mo[e];
}

// New momentum and the sums of squares of the iteration's input (fp32 over a thread's share, fp64
// from there).
template <int VEC>
__global__ void __launch_bounds__(256) norm_kernel(const StepParams p) {
  __shared__ double red[8];
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0;
  const int64_t mn = (int64_t)p.m * p.n, base = (int64_t)blockIdx.y * mn;
  double sum = 0.0;
  const int64_t step = 256ll * VEC * p.parts;
  for (int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC; e0 < mn; e0 += 4 * step) {
    float part = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t e = e0 + u * step;
      if (e >= mn) break;
      float v[VEC];
      update_vec<VEC, true>(p, base + e, v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) part = fmaf(v[i], v[i], part);
    }
    sum += (double)part;
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) p.part[(int64_t)blockIdx.y * p.parts + blockIdx.x] = sum;
}

__device__ __forceinline__ void split_half(float x, uint32_t& hi, uint32_t& lo) {
  const __half h = __float2half_rn(x);
  hi = __half_as_ushort(h);
  lo = __half_as_ushort(__float2half_rn(x - __half2float(h)));
}

// X_0 = unit * update / (norm + eps) as two fp16 planes [s, l], turned when the matrix is tall.
template <int VEC>
__global__ void __launch_bounds__(256) split_kernel(const StepParams p) {
  __shared__ double red[8];
  __shared__ float tile[64][65];
  double sq = 0.0;
  for (int i = threadIdx.x; i < p.parts; i += 256) sq += p.part[(int64_t)blockIdx.y * p.parts + i];
  sq = block_sum(sq, red);
  const float f = p.unit / ((float)sqrt(sq) + p.eps);
  const int64_t base = (int64_t)blockIdx.y * (int64_t)p.m * p.n;
  const int tn = (p.n + 63) / 64;
  const int64_t tiles = (int64_t)((p.m + 63) / 64) * tn;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int r0 = (int)(t / tn) * 64, c0 = (int)(t % tn) * 64;
#pragma unroll 4
    for (int e = threadIdx.x * VEC; e < 4096; e += 256 * VEC) {
      const int r = e >> 6, c = e & 63;
      if (r0 + r >= p.m || c0 + c >= p.n) continue;
      float x[VEC];
      update_vec<VEC, false>(p, base + (int64_t)(r0 + r) * p.n + c0 + c, x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] *= f;
      if (p.tall) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) tile[c + i][r] = x[i];
      } else {
        const int64_t o = (int64_t)blockIdx.y * p.x_batch + (int64_t)(r0 + r) * p.ldx + c0 + c;
        uint32_t hi[VEC], lo[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) split_half(x[i], hi[i], lo[i]);
        if constexpr (VEC == 4) {
          *reinterpret_cast<uint2*>(p.Xh + o) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
          *reinterpret_cast<uint2*>(p.Xl + o) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
        } else {
          p.Xh[o] = __ushort_as_half((unsigned short)hi[0]);
          p.Xl[o] = __ushort_as_half((unsigned short)lo[0]);
        }
      }
    }
    if (p.tall) {
      __syncthreads();
      for (int e = threadIdx.x * 2; e < 4096; e += 512) {
        const int c = e >> 6, r = e & 63;
        if (r0 + r >= p.m || c0 + c >= p.n) continue;
        const int64_t o = (int64_t)blockIdx.y * p.x_batch + (int64_t)(c0 + c) * p.ldx + r0 + r;
        uint32_t hi[2], lo[2];
        split_half(tile[c][r], hi[0], lo[0]);
        split_half(tile[c][r + 1], hi[1], lo[1]);
        // a last row without a partner fills the padding of the leading dimension
        *reinterpret_cast<uint32_t*>(p.Xh + o) = hi[0] | hi[1] << 16;
        *reinterpret_cast<uint32_t*>(p.Xl + o) = lo[0] | lo[1] << 16;
      }
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------ a short side of up to 64
// X_k = Q_k X_0 with Q_k a polynomial in S_0 = X_0 X_0^T, so the matrix is read twice and all steps
// run on s x s matrices: Q' = P Q, S' = P S P with P = a I + b S + c S S.  In fp32 throughout (a
// rounding of S_0 is amplified by a^2 per step; 16-bit operands would not do here).
//   gram_kernel   new momentum, partial Gram matrices over chunks of the long side
//   steps_kernel  one CTA per matrix: sums the partials in order, iterates, Q / (norm + eps)
//   apply_kernel  Q X_0 over chunks of the long side, into O or the new weights
constexpr int SMALL_SIDE = 64;
constexpr int GRAM_COLS = 64;    // long-side columns staged at a time
constexpr int SMALL_LD = SMALL_SIDE + 4;

struct SmallParams {
  StepParams u;
  float* part;       // [batch][chunks][s][s]
  float* Q;          // [batch][s][s]
  int s, l, chunks, chunk_cols, steps;
  float a, b, c;
  __nv_bfloat16* O;
  void* W_out;
  const void* W_in;
  int w_bf16;
  float keep, rate;
};

// stages columns [c0, c0 + GRAM_COLS) as Xs[column][row]; FIRST also writes the momentum
template <bool FIRST>
__device__ __forceinline__ void stage_columns(const SmallParams& p, int64_t base, int c0, int c1,
                                              float (*Xs)[SMALL_LD]) {
  const int s4 = (p.s + 3) & ~3;
  for (int e = threadIdx.x; e < GRAM_COLS * s4; e += 256) {
    // consecutive threads along the contiguous axis of the matrix
    int r, c;
    if (p.u.tall) {
      c = e / s4;
      r = e - c * s4;
    } else {
      r = e / GRAM_COLS;
      c = e - r * GRAM_COLS;
    }
    float v = 0.f;
    if (r < p.s && c0 + c < c1) {
      const int64_t at = base + (p.u.tall ? (int64_t)(c0 + c) * p.s + r : (int64_t)r * p.l + c0 + c);
      float mo = 0.f;
      if (p.u.M_out) {
        if (FIRST) {
          const bool gone = p.u.mask && p.u.mask[at] != 0;
          mo = fmaf(p.u.momentum, p.u.M_in[at], gone ? 0.f : load_any(p.u.G, p.u.g_bf16, at));
          p.u.M_out[at] = mo;
        } else {
          mo = p.u.M_out[at];
        }
      }
      v = update_of(p.u, at, mo);
    }
    Xs[c][r] = v;
  }
}

__global__ void __launch_bounds__(256) gram_kernel(const SmallParams p) {
  __shared__ __align__(16) float Xs[GRAM_COLS][SMALL_LD];
  grid_dependents_launch();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.u.status = 0;
  const int64_t base = (int64_t)blockIdx.y * p.s * p.l;
  const int q = (p.s + 3) / 4, tiles = q * q, groups = 256 / tiles;
  const int g = threadIdx.x / tiles, tile = threadIdx.x - g * tiles;
  const int ti = tile / q, tj = tile - ti * q;
  const int c_lo = blockIdx.x * p.chunk_cols, c_hi = min(p.l, c_lo + p.chunk_cols);
  float acc[4][4] = {};
  for (int c0 = c_lo; c0 < c_hi; c0 += GRAM_COLS) {
    __syncthreads();
    stage_columns<true>(p, base, c0, c_hi, Xs);
    __syncthreads();
    if (g < groups) {
      for (int c = g; c < GRAM_COLS; c += groups) {
        const float4 x = *reinterpret_cast<const float4*>(&Xs[c][4 * ti]);
        const float4 y = *reinterpret_cast<const float4*>(&Xs[c][4 * tj]);
        const float xv[4] = {x.x, x.y, x.z, x.w}, yv[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xv[i], yv[j], acc[i][j]);
      }
    }
  }
  // the groups' sums, in order of the group, through shared memory
  float* red = &Xs[0][0];
  float* out = p.part + ((int64_t)blockIdx.y * p.chunks + blockIdx.x) * p.s * p.s;
  for (int k = 0; k < 16; k += 4) {
    __syncthreads();
    if (g < groups) {
#pragma unroll
      for (int j = 0; j < 4; ++j) red[threadIdx.x * 4 + j] = acc[k / 4][j];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < tiles * 4; e += 256) {
      const int tl = e >> 2, j = e & 3;
      float v = 0.f;
      for (int gg = 0; gg < groups; ++gg) v += red[(gg * tiles + tl) * 4 + j];
      const int r = 4 * (tl / q) + k / 4, c = 4 * (tl % q) + j;
      if (r < p.s && c < p.s) out[r * p.s + c] = v;
    }
  }
}

// D = A^T B for s x s matrices in shared memory (rows padded to SMALL_LD, zeros beyond s); ADD:
// D = a I + b A + c A^T B.  S and P are symmetric up to rounding, S P and Q are not: what is left
// of a rounding in them grows by a = 3.4 per step on one side only, so a transpose of Q in its
// place is wrong by 1e-2 and more on matrices of low rank.
template <bool ADD>
__device__ __forceinline__ void small_product(float (*D)[SMALL_LD], const float (*A)[SMALL_LD],
                                              const float (*B)[SMALL_LD], int s, float a, float b,
                                              float c) {
  const int q = (s + 3) / 4, tiles = q * q;
  if (threadIdx.x < tiles) {
    const int ti = threadIdx.x / q, tj = threadIdx.x - ti * q;
    float acc[4][4] = {};
    for (int k = 0; k < s; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&A[k][4 * ti]);
      const float4 y = *reinterpret_cast<const float4*>(&B[k][4 * tj]);
      const float xv[4] = {x.x, x.y, x.z, x.w}, yv[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xv[i], yv[j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 4 * ti + i, cc = 4 * tj + j;
        float v = acc[i][j];
        if (ADD) v = fmaf(c, v, fmaf(b, A[r][cc], r == cc ? a : 0.f));
        D[r][cc] = v;
      }
  }
  __syncthreads();
}

__global__ void __launch_bounds__(256) steps_kernel(const SmallParams p) {
  extern __shared__ __align__(16) float mats[];
  float(*M[5])[SMALL_LD];
  for (int i = 0; i < 5; ++i)
    M[i] = reinterpret_cast<float(*)[SMALL_LD]>(mats + i * SMALL_SIDE * SMALL_LD);
  __shared__ float norm;
  grid_dependency_wait();
  grid_dependents_launch();
  const int s = p.s, s4 = (s + 3) & ~3;
  const float* part = p.part + (int64_t)blockIdx.x * p.chunks * s * s;
  for (int e = threadIdx.x; e < s4 * s4; e += 256) {
    const int r = e / s4, c = e - r * s4;
    float v = 0.f;
    if (r < s && c < s)
      for (int k = 0; k < p.chunks; ++k) v += part[(int64_t)k * s * s + r * s + c];
    M[0][r][c] = v;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float t = 0.f;
    for (int i = 0; i < s; ++i) t += M[0][i][i];
    norm = sqrtf(t) + p.u.eps;
  }
  __syncthreads();
  const float inv = 1.f / norm;
  for (int e = threadIdx.x; e < s4 * s4; e += 256) {
    const int r = e / s4, c = e - r * s4;
    M[0][r][c] = M[0][r][c] * inv * inv;
  }
  __syncthreads();
  float(*S)[SMALL_LD] = M[0], (*P)[SMALL_LD] = M[1], (*Q)[SMALL_LD] = M[2], (*T)[SMALL_LD] = M[3],
  (*U)[SMALL_LD] = M[4];
  for (int it = 0; it < p.steps; ++it) {
    small_product<true>(P, S, S, s, p.a, p.b, p.c);
    if (it == 0) {
      for (int e = threadIdx.x; e < s4 * s4; e += 256) Q[e / s4][e % s4] = P[e / s4][e % s4];
      __syncthreads();
    } else {
      small_product<false>(U, P, Q, s, 0.f, 0.f, 0.f);
      float(*t)[SMALL_LD] = Q;
      Q = U;
      U = t;
    }
    if (it + 1 < p.steps) {
      small_product<false>(T, S, P, s, 0.f, 0.f, 0.f);   // S P
      small_product<false>(S, T, P, s, 0.f, 0.f, 0.f);   // (S P)^T P = P S P
    }
  }
  float* out = p.Q + (int64_t)blockIdx.x * s * s;
  for (int e = threadIdx.x; e < s * s; e += 256) out[e] = Q[e / s][e % s] * inv;
}

__global__ void __launch_bounds__(256) apply_kernel(const SmallParams p) {
  __shared__ __align__(16) float Xs[GRAM_COLS][SMALL_LD];
  __shared__ __align__(16) float Qs[SMALL_SIDE][SMALL_LD];
  grid_dependency_wait();
  const int64_t base = (int64_t)blockIdx.y * p.s * p.l;
  const float* Q = p.Q + (int64_t)blockIdx.y * p.s * p.s;
  const int s4 = (p.s + 3) & ~3;
  for (int e = threadIdx.x; e < s4 * s4; e += 256) {
    const int r = e / s4, c = e - r * s4;
    Qs[c][r] = r < p.s && c < p.s ? Q[r * p.s + c] : 0.f;
  }
  for (int64_t t = blockIdx.x; t * GRAM_COLS < p.l; t += gridDim.x) {
    const int c0 = (int)t * GRAM_COLS;
    __syncthreads();
    stage_columns<false>(p, base, c0, p.l, Xs);
    __syncthreads();
    // four rows of one column a thread
    const int q = s4 / 4;
    for (int e = threadIdx.x; e < q * GRAM_COLS; e += 256) {
      int rq, c;
      if (p.u.tall) {
        c = e / q;
        rq = e - c * q;
      } else {
        rq = e / GRAM_COLS;
        c = e - rq * GRAM_COLS;
      }
      float o[4] = {};
      for (int k = 0; k < p.s; ++k) {
        const float4 y = *reinterpret_cast<const float4*>(&Qs[k][4 * rq]);
        const float x = Xs[c][k];
        o[0] = fmaf(y.x, x, o[0]);
        o[1] = fmaf(y.y, x, o[1]);
        o[2] = fmaf(y.z, x, o[2]);
        o[3] = fmaf(y.w, x, o[3]);
      }
      if (c0 + c >= p.l) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * rq + i;
        if (r >= p.s) break;
        const int64_t at =
            base + (p.u.tall ? (int64_t)(c0 + c) * p.s + r : (int64_t)r * p.l + c0 + c);
        if (p.O) {
          p.O[at] = __float2bfloat16_rn(o[i]);
        } else {
          float w = fmaf(-p.rate, o[i], p.keep * load_any(p.W_in, p.w_bf16, at));
          if (p.u.mask && p.u.mask[at] != 0) w = 0.f;
          if (p.w_bf16) static_cast<__nv_bfloat16*>(p.W_out)[at] = __float2bfloat16_rn(w);
          else static_cast<float*>(p.W_out)[at] = w;
        }
      }
    }
  }
}

// chunks of the long side per matrix: enough CTAs for the device, at most 64 partial matrices
int small_chunks(int64_t batch, int64_t l) {
  int64_t want = ceil_div(2 * NUM_SMS, batch);
  const int64_t most = ceil_div(l, GRAM_COLS);
  if (want > most) want = most;
  if (want > 64) want = 64;
  return (int)want;
}

template <typename K>
thanos_status_t launch_after(K kernel, dim3 grid, size_t smem, const SmallParams& p,
                             cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(256, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  return THANOS_OK;
}

thanos_status_t small_side(const OrthogonalArgs& a, StepParams u, int s, int l, float* part,
                           float* Q, int chunks, cudaStream_t stream) {
  SmallParams p = {};
  p.u = u;
  p.part = part;
  p.Q = Q;
  p.s = s;
  p.l = l;
  p.chunk_cols = (int)round_up((size_t)ceil_div(l, chunks), GRAM_COLS);
  p.chunks = (int)ceil_div(l, p.chunk_cols);
  p.steps = a.steps;
  p.a = a.coef[0];
  p.b = a.coef[1];
  p.c = a.coef[2];
  p.O = a.O;
  p.W_out = a.W_out;
  p.W_in = a.W_in;
  p.w_bf16 = a.wdtype == THANOS_BF16;
  p.keep = a.keep;
  p.rate = a.rate;
  gram_kernel<<<dim3((unsigned)p.chunks, (unsigned)a.batch), 256, 0, stream>>>(p);
  THANOS_CHECK_LAUNCH();
  constexpr int kSmem = 5 * SMALL_SIDE * SMALL_LD * 4;
  static std::atomic<unsigned long long> done{0};
  THANOS_CUDA(ensure_max_dyn_smem(steps_kernel, kSmem, done));
  THANOS_TRY(launch_after(steps_kernel, dim3((unsigned)a.batch), kSmem, p, stream));
  int64_t blocks = ceil_div(l, GRAM_COLS);
  if (blocks * a.batch > 4 * NUM_SMS) blocks = ceil_div(4 * NUM_SMS, a.batch);
  return launch_after(apply_kernel, dim3((unsigned)blocks, (unsigned)a.batch), 0, p, stream);
}

float pow2_at_most(double x, int most) {
  int e = 0;
  while (e < most && (double)(1 << (e + 1)) <= x) ++e;
  return (float)(1 << e);
}

int norm_parts(int64_t mn) {
  const int64_t want = ceil_div(mn, 8192);
  return (int)(want < MAX_PARTS ? want : MAX_PARTS);
}

}  // namespace

size_t orthogonal_workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  const size_t s = (size_t)(m < n ? m : n), l = (size_t)(m < n ? n : m), k = (size_t)batch;
  if (s <= SMALL_SIDE)
    return 256 + round_up(k * small_chunks(batch > 0 ? batch : 1, l) * s * s * 4, 256) +
           round_up(k * s * s * 4, 256);
  return 256 + round_up(k * MAX_PARTS * 8, 256) + 4 * round_up(k * s * round_up(l, 8) * 2, 256) +
         2 * round_up(k * s * round_up(s, 8) * 2, 256);
}

thanos_status_t orthogonal_impl(const OrthogonalArgs& a, void* workspace, size_t ws_bytes,
                                cudaStream_t stream) {
  const int s = (int)(a.m < a.n ? a.m : a.n), l = (int)(a.m < a.n ? a.n : a.m);
  const int64_t lds = (int64_t)round_up(s, 8), ldx = (int64_t)round_up(l, 8);
  const size_t k = (size_t)a.batch;
  Arena ar(workspace, ws_bytes);
  int32_t* status = ar.take<int32_t>(64);
  StepParams sp = {};
  sp.G = a.G;
  sp.M_out = a.M_out;
  sp.M_in = a.M_in;
  sp.mask = a.mask;
  sp.status = status;
  sp.g_bf16 = a.gdtype == THANOS_BF16;
  sp.nesterov = a.nesterov;
  sp.tall = a.m > a.n;
  sp.momentum = a.momentum;
  sp.eps = a.eps;
  sp.m = (int)a.m;
  sp.n = (int)a.n;
  if (s <= SMALL_SIDE) {
    const int chunks = small_chunks(a.batch, l);
    float* parts = ar.take<float>(k * chunks * s * s);
    float* Q = ar.take<float>(k * s * s);
    if (!ar.ok()) return THANOS_ERR_WORKSPACE;
    return small_side(a, sp, s, l, parts, Q, chunks, stream);
  }
  double* part = ar.take<double>(k * MAX_PARTS);
  __half* X[2][2];
  for (auto& x : X)
    for (auto& plane : x) plane = ar.take<__half>(k * s * ldx);
  __half* S = ar.take<__half>(k * s * lds);
  __half* P = ar.take<__half>(k * s * lds);
  if (!ar.ok()) return THANOS_ERR_WORKSPACE;
  // Entries of X are at most the spectral norm (about 1.2), on average (s l)^-1/2 at the start;
  // entries of S at most its square, on average 1 / s; P is up to some ten times S.
  const float ux = pow2_at_most(sqrt((double)s * l), 14), us = pow2_at_most(s, 13),
              up = pow2_at_most(s, 11);
  sp.part = part;
  sp.parts = norm_parts(a.m * a.n);
  sp.unit = ux;
  sp.Xh = X[0][0];
  sp.Xl = X[0][1];
  sp.ldx = ldx;
  sp.x_batch = s * ldx;
  const int64_t tiles = ceil_div(a.m, 64) * ceil_div(a.n, 64);
  const dim3 norm_grid((unsigned)sp.parts, (unsigned)k);
  const dim3 split_grid((unsigned)(tiles < 8 * NUM_SMS ? tiles : 8 * NUM_SMS), (unsigned)k);
  if (a.n % 4 == 0) {
    norm_kernel<4><<<norm_grid, 256, 0, stream>>>(sp);
    THANOS_CHECK_LAUNCH();
    split_kernel<4><<<split_grid, 256, 0, stream>>>(sp);
  } else {
    norm_kernel<1><<<norm_grid, 256, 0, stream>>>(sp);
    THANOS_CHECK_LAUNCH();
    split_kernel<1><<<split_grid, 256, 0, stream>>>(sp);
  }
  THANOS_CHECK_LAUNCH();
  ProjArgs g;
  g.batch = (int)k;
  g.f16 = 1;
  g.status = status;
  g.S = S;
  g.Pm = P;
  g.lds = lds;
  g.s_batch = s * lds;
  g.ldx = ldx;
  g.x_batch = s * ldx;
  for (int it = 0; it < a.steps; ++it) {
    __half** x = X[it & 1];
    ProjArgs q = g;                 // S = X X^T
    q.epi = PROJ_GRAM;
    q.M = q.N = s;
    q.K = l;
    q.A = q.B = x[0];
    q.lda = q.ldb = ldx;
    q.a_batch = q.b_batch = s * ldx;
    q.alpha = us / (ux * ux);
    THANOS_TRY(proj_gemm(q, stream));
    q.epi = PROJ_POLY;              // P = b S + c S S
    q.K = s;
    q.A = q.B = S;
    q.lda = q.ldb = lds;
    q.a_batch = q.b_batch = s * lds;
    q.alpha = a.coef[2] * (up / (us * us));
    q.beta = a.coef[1] * (up / us);
    THANOS_TRY(proj_gemm(q, stream));
    q = g;                          // X' = a X + P X
    const bool last = it + 1 == a.steps;
    q.epi = last ? PROJ_FINAL : PROJ_NEXT;
    q.M = l;
    q.N = s;
    q.K = s;
    q.A = x[0];
    q.a_mn = 1;
    q.lda = ldx;
    q.a_batch = s * ldx;
    q.B = P;
    q.ldb = lds;
    q.b_batch = s * lds;
    q.Xh = x[0];
    q.Xl = x[1];
    q.Yh = X[(it + 1) & 1][0];
    q.Yl = X[(it + 1) & 1][1];
    q.alpha = (last ? 1.f / ux : 1.f) / up;
    q.beta = last ? a.coef[0] / ux : a.coef[0];
    q.O = a.O;
    q.W_out = a.W_out;
    q.W_in = a.W_in;
    q.mask = a.mask;
    q.w_bf16 = a.wdtype == THANOS_BF16;
    q.tall = sp.tall;
    q.keep = a.keep;
    q.rate = a.rate;
    THANOS_TRY(proj_gemm(q, stream));
  }
  return THANOS_OK;
}

}  // namespace thanos
