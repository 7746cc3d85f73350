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
//
// That is 1 to 2e-3 of the result, as much as the bf16 rounding of O or of bf16 weights.  A step on
// fp32 weights carries S and P as two planes too and takes three products of planes for each (fine):
// 2e-5 to 1e-4 of the update, mostly the cut sums on the diagonal of S.  It costs three times the tensor
// work and twice the operand traffic: 768 x 768 in 168 us instead of 107, 4096 x 4096 in 3.4 ms
// instead of 1.34.
#include <type_traits>

#include "proj_gemm.cuh"
#include "recovery.cuh"

namespace thanos {
namespace {

// Sides up to which the diagonals of S and P are kept apart in fp32.  The rows of a long matrix are
// nearly orthogonal, S nearly its diagonal, and a rounding of a diagonal entry is a factor of a whole
// row that a + b s + c s^2 = 3.4 - 4.8 + 2.0 makes four times as large (8000 x 128: error 1.8e-3 of
// the result beside the rounding of O, 0.9e-3 with them apart).  With larger sides the rest of S
// outweighs its diagonal (4096 x 4096: no difference, and 60 of 1330 us for reading it).
constexpr int DIAG_SIDE = 512;
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

template <int VEC>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = *p;
  } else {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x;
    v[1] = q.y;
    v[2] = q.z;
    v[3] = q.w;
  }
}

// N vectors of the iteration's input, the first at `at`, the others `step` elements apart; those from
// `count` on are zero.  FIRST reads the old momentum and writes the new one, else the new one is
// read.  Every operand is loaded for all N vectors before any is used: which operands there are is
// asked once, since a branch between two loads keeps them from being in flight together.
template <int VEC, int N, bool FIRST>
__device__ __forceinline__ void update_batch(const StepParams& p, int64_t at, int64_t step, int count,
                                             float (&v)[N][VEC]) {
  uint32_t gone[N] = {};
  float mo[N][VEC] = {};
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[u][e] = 0.f;
  if (FIRST || !p.M_out || p.nesterov) {
    if (p.g_bf16) {
      const __nv_bfloat16* G = static_cast<const __nv_bfloat16*>(p.G) + at;
      uint2 q[N] = {};
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (u < count) {
          if constexpr (VEC == 1) q[u].x = *reinterpret_cast<const unsigned short*>(G + u * step);
          else q[u] = *reinterpret_cast<const uint2*>(G + u * step);
        }
#pragma unroll
      for (int u = 0; u < N; ++u) {
        v[u][0] = __uint_as_float(q[u].x << 16);
        if constexpr (VEC == 4) {
          v[u][1] = __uint_as_float(q[u].x & 0xFFFF0000u);
          v[u][2] = __uint_as_float(q[u].y << 16);
          v[u][3] = __uint_as_float(q[u].y & 0xFFFF0000u);
        }
      }
    } else {
      const float* G = static_cast<const float*>(p.G) + at;
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (u < count) load_f32<VEC>(G + u * step, v[u]);
    }
  }
  if (p.M_out) {
    const float* M = (FIRST ? p.M_in : p.M_out) + at;
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (u < count) load_f32<VEC>(M + u * step, mo[u]);
  }
  if (p.mask) {
    const uint8_t* k = p.mask + at;
    uint32_t w[N] = {};
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (u < count) {
        if constexpr (VEC == 1) w[u] = k[u * step];
        else w[u] = *reinterpret_cast<const uint32_t*>(k + u * step);
      }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) gone[u] |= ((w[u] >> (8 * e)) & 0xFFu ? 1u : 0u) << e;
  }
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if ((gone[u] >> e) & 1u) v[u][e] = 0.f;
  if (!p.M_out) return;
  if (FIRST) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) mo[u][e] = fmaf(p.momentum, mo[u][e], v[u][e]);
      if (u < count) {
        float* M = p.M_out + at + u * step;
        if constexpr (VEC == 4)
          *reinterpret_cast<float4*>(M) = make_float4(mo[u][0], mo[u][1], mo[u][2], mo[u][3]);
        else *M = mo[u][0];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      v[u][e] = (gone[u] >> e) & 1u ? 0.f
                : p.nesterov       ? fmaf(p.momentum, mo[u][e], v[u][e])
                                   : mo[u][e];
}

// Whether fp32 squares that add up to this may have left fp32's range: beyond it, or below it where
// eps does not hide that.
__device__ __forceinline__ bool squares_out_of_range(float sum, float eps) {
  return !(sum < 1e36f) || (sum < 1e-28f && eps < 1e-8f);
}

// A block's sum of squares once more, in fp64.
template <int VEC>
__device__ __noinline__ double squares_again(const StepParams& p, int64_t base, int64_t step,
                                             int64_t mn) {
  double sum = 0.0;
  for (int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC; e0 < mn; e0 += step) {
    float v[1][VEC];
    update_batch<VEC, 1, false>(p, base + e0, step, 1, v);
    for (int i = 0; i < VEC; ++i) sum = fma((double)v[0][i], (double)v[0][i], sum);
  }
  return sum;
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
    float v[4][VEC];
    const int count = e0 + 3 * step < mn ? 4 : (int)((mn - e0 + step - 1) / step);
    update_batch<VEC, 4, true>(p, base + e0, step, count, v);
    float part = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) part = fmaf(v[u][i], v[u][i], part);
    sum += (double)part;
  }
  sum = block_sum(sum, red);
  if (squares_out_of_range((float)sum, p.eps)) {
    __syncthreads();
    sum = block_sum(squares_again<VEC>(p, base, step, mn), red);
  }
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
  const double norm = sqrt(sq);
  float f = p.unit / ((float)norm + p.eps);
  if (norm > 1e38) f = (float)((double)p.unit / (norm + (double)p.eps));  // beyond fp32, or nearly
  const int64_t base = (int64_t)blockIdx.y * (int64_t)p.m * p.n;
  const int tn = (p.n + 63) / 64;
  const int64_t tiles = (int64_t)((p.m + 63) / 64) * tn;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int r0 = (int)(t / tn) * 64, c0 = (int)(t % tn) * 64;
    // a thread's column, and the rows it takes, 4 VEC apart
    const int c = (threadIdx.x * VEC) & 63;
    constexpr int HOP = 4 * VEC;
#pragma unroll 1
    for (int r = (threadIdx.x * VEC) >> 6; r < 64; r += 4 * HOP) {
      const int left = p.m - r0 - r;   // rows from here on
      const int count = c0 + c >= p.n || left <= 0 ? 0 : min(4, (left + HOP - 1) / HOP);
      float x[4][VEC];
      update_batch<VEC, 4, false>(p, base + (int64_t)(r0 + r) * p.n + c0 + c, (int64_t)HOP * p.n,
                                  count, x);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (u >= count) break;
        const int rr = r + u * HOP;
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[u][i] *= f;
        if (p.tall) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) tile[c + i][rr] = x[u][i];
        } else {
          const int64_t o = (int64_t)blockIdx.y * p.x_batch + (int64_t)(r0 + rr) * p.ldx + c0 + c;
          uint32_t hi[VEC], lo[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) split_half(x[u][i], hi[i], lo[i]);
          if constexpr (VEC == 4) {
            *reinterpret_cast<uint2*>(p.Xh + o) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
            *reinterpret_cast<uint2*>(p.Xl + o) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
          } else {
            p.Xh[o] = __ushort_as_half((unsigned short)hi[0]);
            p.Xl[o] = __ushort_as_half((unsigned short)lo[0]);
          }
        }
      }
    }
    if (p.tall) {
      __syncthreads();
      const int r = (threadIdx.x * 4) & 63;
#pragma unroll 2
      for (int c = threadIdx.x >> 4; c < 64; c += 16) {
        if (r0 + r >= p.m || c0 + c >= p.n) continue;
        const int64_t o = (int64_t)blockIdx.y * p.x_batch + (int64_t)(c0 + c) * p.ldx + r0 + r;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) split_half(tile[c][r + i], hi[i], lo[i]);
        // rows beyond the last fill the padding of the leading dimension (a multiple of 8)
        *reinterpret_cast<uint2*>(p.Xh + o) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
        *reinterpret_cast<uint2*>(p.Xl + o) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
      }
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------ a short side of up to 64
// X_k = Q_k X_0 with Q_k a polynomial in S_0 = X_0 X_0^T, so the matrix is read twice and all steps
// run on s x s matrices: Q' = P Q, S' = P S P with P = a I + b S + c S S.  In fp32 (a rounding of S_0
// is amplified by a^2 per step; 16-bit operands would not do here).  The s x s
// products are a chain on one CTA: 64 x 64 takes 60 us alone, of which the wide products take twice
// the time whatever the size (4096 x 64: 90 against 123 us, 3 x 7697 x 40: 70 against 178), but a side
// of 128 would take eight times as much.  What fp32 loses of directions 20 times weaker than the
// strongest is 5e-4 of the result, which bf16 does not show.  For fp32 weights the Gram matrix and its
// powers are fp64 (below 6e-5; 32 steps of 16 x 4096: 37 us instead of 33), and a side above 32 goes by
// the wide products and two planes (2 to 6e-5).
//   gram_kernel   new momentum, partial Gram matrices over chunks of the long side
//   steps_kernel  one CTA per matrix: sums the partials in order, iterates, Q / (norm + eps)
//   apply_kernel  Q X_0 over chunks of the long side, into O or the new weights
// Many matrices are bound by the loads of the two elementwise passes, whose phases (load, turn, multiply)
// follow one another in a CTA: 57 steps of 18 x 9804, 141 MB, take 130 us, 1.1 TB/s.
constexpr int SMALL_SIDE = 64, SMALL_SIDE_FINE = 32;  // FINE: fp32 weights
// TS x TS entries of a product a thread on 16 x 16 threads: TS = 1 and 2 share a layout
__host__ __device__ constexpr int small_ld(int ts) { return (ts <= 2 ? 32 : 64) + 4; }
__host__ __device__ constexpr int small_size(int ts) {  // and a row of zeros
  return (small_ld(ts) - 3) * small_ld(ts);
}
constexpr int STAGE_FLOATS = 10240;  // a tile of the long side, padded rows: 512 columns of 16 rows

template <typename Real, int N>
struct alignas(sizeof(Real) * N < 16 ? sizeof(Real) * N : 16) Vec {
  Real v[N];
};
template <typename Real>
__device__ __forceinline__ void add4(Vec<Real, 4>& a, const Vec<Real, 4>& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a.v[i] += b.v[i];
}

struct SmallParams {
  StepParams u;
  void* part;        // [batch][chunks][4 x 4 tiles of the Gram matrix], fp32, fp64 for fp32 weights
  float* Q;          // [batch][s][s]
  int s, l, chunks, chunk_cols, tile_cols, steps;
  uint32_t inv_q;    // ceil(2^32 / q) for q = ceil(s / 4) > 1: e / q is the high word of e inv_q
  float a, b, c;
  __nv_bfloat16* O;
  void* W_out;
  const void* W_in;
  int w_bf16;
  float keep, rate;
};

// Stages columns [c0, c0 + cols) of the long side as Xs[column * ld + row], rows up to the next
// multiple of four (zeros beyond s); FIRST also writes the momentum.  A thread takes blocks of four
// rows x VEC columns, turns them in registers and writes whole 16-byte rows; neighbours take the
// row blocks of a column first, which keeps both the loads and the shared-memory stores wide.
template <int VEC, bool FIRST>
__device__ __forceinline__ void stage_columns(const SmallParams& p, int64_t base, int c0, int cols,
                                              float* Xs, int ld) {
  const int q = (p.s + 3) / 4;
  const int blocks = q * (p.u.tall ? cols : (cols + VEC - 1) / VEC);
#pragma unroll 1
  for (int it = threadIdx.x; it < blocks; it += 256) {
    const int cb = q == 1 ? it : (int)__umulhi((uint32_t)it, p.inv_q), r = 4 * (it - cb * q);
    if (p.u.tall) {     // [l, s]: the four rows of a column are neighbours
      const int64_t at = base + (int64_t)(c0 + cb) * p.s + r;
      float4 x;
      if constexpr (VEC == 4) {
        float v[1][4];
        update_batch<4, 1, FIRST>(p.u, at, 0, 1, v);
        x = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
      } else {
        float v[4][1];
        update_batch<1, 4, FIRST>(p.u, at, 1, min(4, p.s - r), v);
        x = make_float4(v[0][0], v[1][0], v[2][0], v[3][0]);
      }
      *reinterpret_cast<float4*>(Xs + cb * ld + r) = x;
    } else {
      const int c = cb * VEC;
      float v[4][VEC];
      update_batch<VEC, 4, FIRST>(p.u, base + (int64_t)r * p.l + c0 + c, p.l, min(4, p.s - r), v);
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        *reinterpret_cast<float4*>(Xs + (c + i) * ld + r) =
            make_float4(v[0][i], v[1][i], v[2][i], v[3][i]);
    }
  }
}

// FINE (fp32 weights): a thread's products are added in fp64, sixteen at a time.
template <int VEC, bool FINE>
__global__ void __launch_bounds__(256) gram_kernel(const SmallParams p) {
  using Real = std::conditional_t<FINE, double, float>;
  constexpr int RUN = 16;
  extern __shared__ __align__(16) float Xs[];
  grid_dependents_launch();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.u.status = 0;
  const int64_t base = (int64_t)blockIdx.y * p.s * p.l;
  const int q = (p.s + 3) / 4, tiles = q * q, groups = 256 / tiles, ld = 4 * q + 4;
  const int g = threadIdx.x / tiles, tile = threadIdx.x - g * tiles;
  const int ti = tile / q, tj = tile - ti * q;
  const int c_lo = blockIdx.x * p.chunk_cols, c_hi = min(p.l, c_lo + p.chunk_cols);
  Real acc[4][4] = {};
  // acc += the products of columns c, c + groups, .. below `end`
  auto columns = [&](int c, int end, auto& sums) {
#pragma unroll 4
    for (; c < end; c += groups) {
      const float4 x = *reinterpret_cast<const float4*>(Xs + c * ld + 4 * ti);
      const float4 y = *reinterpret_cast<const float4*>(Xs + c * ld + 4 * tj);
      const float xv[4] = {x.x, x.y, x.z, x.w}, yv[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[i][j] = fmaf(xv[i], yv[j], sums[i][j]);
    }
  };
  for (int c0 = c_lo; c0 < c_hi; c0 += p.tile_cols) {
    const int cols = min(p.tile_cols, c_hi - c0);
    __syncthreads();
    stage_columns<VEC, true>(p, base, c0, cols, Xs, ld);
    __syncthreads();
    if (g < groups) {
      if constexpr (FINE) {
        for (int c = g; c < cols; c += RUN * groups) {
          float run[4][4] = {};
          columns(c, min(cols, c + RUN * groups), run);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] += (double)run[i][j];
        }
      } else {
        columns(g, cols, acc);
      }
    }
  }
  // the groups' sums, in order of the group
  __syncthreads();
  using Four = Vec<Real, 4>;
  Four* sums = reinterpret_cast<Four*>(Xs);
  if (g < groups) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sums[(g * tiles + tile) * 4 + i] = Four{acc[i][0], acc[i][1], acc[i][2], acc[i][3]};
  }
  __syncthreads();
  Four* out = static_cast<Four*>(p.part) + ((int64_t)blockIdx.y * p.chunks + blockIdx.x) * (tiles * 4);
  for (int e = threadIdx.x; e < tiles * 4; e += 256) {
    Four v = sums[e];
#pragma unroll 4
    for (int k = 1; k < groups; ++k) add4(v, sums[k * tiles * 4 + e]);
    out[e] = v;
  }
}

// D = A^T B for s x s matrices in shared memory (rows padded to LD, zeros beyond s); with
// `add`, D = a I + b A + c A^T B.  S and P are symmetric up to rounding, S P and Q are not: what is
// left of a rounding in them grows by a = 3.4 per step on one side only, so a transpose of Q in its
// place is wrong by 1e-2 and more on matrices of low rank.  TS x TS outputs a thread; one copy of the
// code for all the products of a step, which run one after another on one CTA.
template <int TS, typename Real>
__device__ __noinline__ void small_product(int D_at, int A_at, int B_at, int s, bool add, Real a, Real b,
                                           Real c) {
  extern __shared__ __align__(16) unsigned char small_smem[];
  Real* mats = reinterpret_cast<Real*>(small_smem);
  constexpr int LD = small_ld(TS);
  const int q = (s + TS - 1) / TS;
  const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;  // 16 x 16 threads
  if (ti < q && tj < q) {
    const Real* x = mats + A_at + TS * ti;
    const Real* y = mats + B_at + TS * tj;
    Real acc[2][TS][TS] = {};   // even and odd k apart: half the chain of dependent additions
#pragma unroll 4
    for (int k = 0; k < s; k += 2) {   // row s is zero
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Vec<Real, TS> xv = *reinterpret_cast<const Vec<Real, TS>*>(x + (k + h) * LD);
        const Vec<Real, TS> yv = *reinterpret_cast<const Vec<Real, TS>*>(y + (k + h) * LD);
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
          for (int j = 0; j < TS; ++j) acc[h][i][j] = fma(xv.v[i], yv.v[j], acc[h][i][j]);
      }
    }
#pragma unroll
    for (int i = 0; i < TS; ++i)
#pragma unroll
      for (int j = 0; j < TS; ++j) {
        const int r = TS * ti + i, cc = TS * tj + j;
        Real v = acc[0][i][j] + acc[1][i][j];
        if (add) v = fma(c, v, fma(b, mats[A_at + r * LD + cc], r == cc ? a : (Real)0));
        if (r < s && cc < s) mats[D_at + r * LD + cc] = v;
      }
  }
  __syncthreads();
}

constexpr int STEP_THREADS = 256;

// Every hop-th of the chunks' partial matrices from the first-th on.
template <typename Real>
__device__ __forceinline__ Vec<Real, 4> sum_parts(const Vec<Real, 4>* part, int first, int hop,
                                                  int chunks, int vecs) {
  Vec<Real, 4> sum = {};
#pragma unroll 8
  for (int k = first; k < chunks; k += hop) add4(sum, part[(int64_t)k * vecs]);
  return sum;
}

// The Gram matrix of a matrix whose squares leave fp32's range, once more by this one CTA: X scaled by
// the power of two that brings its largest value to between one and two.  Returns that exponent (the
// product is 2^(-2 e) of what it stands for); with infinities or NaN everything stays as it is.
// The matrices behind the first are used for staging and left zero.
template <int TS, typename Real>
__device__ __noinline__ int gram_again(const SmallParams& p) {
  extern __shared__ __align__(16) unsigned char small_smem[];
  Real* mats = reinterpret_cast<Real*>(small_smem);
  __shared__ uint32_t tops[STEP_THREADS / 32];
  constexpr int LD = small_ld(TS), SZ = small_size(TS);
  float* Xs = reinterpret_cast<float*>(mats + SZ);
  const int64_t base = (int64_t)blockIdx.x * p.s * p.l;
  const int q = (p.s + 3) / 4, ld = 4 * q + 4, ti = threadIdx.x / q, tj = threadIdx.x - ti * q;
  uint32_t top = 0;  // largest magnitude, as bits
  for (int c0 = 0; c0 < p.l; c0 += p.tile_cols) {
    const int cols = min(p.tile_cols, p.l - c0);
    __syncthreads();
    stage_columns<1, false>(p, base, c0, cols, Xs, ld);
    __syncthreads();
    for (int e = threadIdx.x; e < cols * 4 * q; e += STEP_THREADS)
      top = max(top, __float_as_uint(Xs[e / (4 * q) * ld + e % (4 * q)]) & 0x7FFFFFFFu);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  for (int w = 0; w < STEP_THREADS / 32; ++w) top = max(top, tops[w]);
  int e = 0;
  if (top > 0 && top < 0x7F800000u) {
    e = max((int)(top >> 23) - 127, -120);
    const float scale = ldexpf(1.f, -e);
    Real acc[4][4] = {};
    for (int c0 = 0; c0 < p.l; c0 += p.tile_cols) {
      const int cols = min(p.tile_cols, p.l - c0);
      __syncthreads();
      stage_columns<1, false>(p, base, c0, cols, Xs, ld);
      __syncthreads();
      if (ti >= q) continue;
      for (int c = 0; c < cols; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = fma((Real)(scale * Xs[c * ld + 4 * ti + i]),
                            (Real)(scale * Xs[c * ld + 4 * tj + j]), acc[i][j]);
      }
    }
    if (ti < q) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mats[(4 * ti + i) * LD + 4 * tj + j] = acc[i][j];
    }
  }
  __syncthreads();
  for (int k = SZ + threadIdx.x; k < 5 * SZ; k += STEP_THREADS) mats[k] = (Real)0;
  __syncthreads();
  return e;
}

template <int TS, typename Real>
__global__ void __launch_bounds__(STEP_THREADS) steps_kernel(const SmallParams p) {
  extern __shared__ __align__(16) unsigned char small_smem[];
  Real* mats = reinterpret_cast<Real*>(small_smem);
  using Four = Vec<Real, 4>;
  // S, P, Q, T, U: a row more than they need, which stays zero
  constexpr int LD = small_ld(TS), SZ = small_size(TS);
  Real *S = mats, *T = mats + 3 * SZ;
  int Q = 2 * SZ, U = 4 * SZ;
  __shared__ Real square;
  const int s = p.s, ss = s * s;
  for (int e = threadIdx.x; e < 5 * SZ; e += STEP_THREADS) mats[e] = (Real)0;
  __syncthreads();
  grid_dependency_wait();
  grid_dependents_launch();
  // the partial matrices, four entries a thread; threads to spare take every groups-th of them
  const int q = (s + 3) / 4, vecs = q * q * 4;
  const Four* part = static_cast<const Four*>(p.part) + (int64_t)blockIdx.x * p.chunks * vecs;
  if constexpr (TS <= 2) {
    const int groups = STEP_THREADS / vecs;
    const int g = threadIdx.x / vecs, e = threadIdx.x - g * vecs;
    Four sum = {};
    if (g < groups) {
      sum = sum_parts(part + e, g, groups, p.chunks, vecs);
      reinterpret_cast<Four*>(T)[threadIdx.x] = sum;  // T holds 297 of them
    }
    __syncthreads();
    if (threadIdx.x < vecs) {
      for (int k = 1; k < groups; ++k) add4(sum, reinterpret_cast<const Four*>(T)[k * vecs + e]);
      const int tl = e >> 2, tr = tl / q;
      *reinterpret_cast<Four*>(S + (4 * tr + (e & 3)) * LD + 4 * (tl - tr * q)) = sum;
    }
  } else {
    for (int e = threadIdx.x; e < vecs; e += STEP_THREADS) {
      const int tl = e >> 2, tr = tl / q;
      *reinterpret_cast<Four*>(S + (4 * tr + (e & 3)) * LD + 4 * (tl - tr * q)) =
          sum_parts(part + e, 0, 1, p.chunks, vecs);
    }
  }
  __syncthreads();
  auto trace = [&]() {
    if (threadIdx.x < 32) {
      Real t = 0;
      for (int i = threadIdx.x; i < s; i += 32) t += S[i * LD + i];
      for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
      if (threadIdx.x == 0) square = t;
    }
    __syncthreads();
  };
  trace();
  int exponent = 0;
  Real eps = p.u.eps;
  if (squares_out_of_range((float)square, p.u.eps)) {
    exponent = gram_again<TS, Real>(p);
    eps = ldexpf(p.u.eps, -exponent);
    trace();
  }
  const Real inv = (Real)1 / (sqrt(square) + eps);
  for (int i = threadIdx.x; i < s * LD; i += STEP_THREADS) S[i] = S[i] * inv * inv;
  __syncthreads();
  // T held partial sums: its row s has to be zero again
  for (int i = threadIdx.x; i < SZ; i += STEP_THREADS) T[i] = (Real)0;
  __syncthreads();
#pragma unroll 1
  for (int it = 0; it < p.steps; ++it) {
    const int P = it == 0 ? Q : SZ;                         // Q_1 = P_0
    small_product<TS, Real>(P, 0, 0, s, true, p.a, p.b, p.c);
    if (it > 0) {
      small_product<TS, Real>(U, P, Q, s, false, 0.f, 0.f, 0.f);
      const int t = Q;
      Q = U;
      U = t;
    }
    if (it + 1 < p.steps) {
      small_product<TS, Real>(3 * SZ, 0, P, s, false, 0.f, 0.f, 0.f);       // S P
      small_product<TS, Real>(0, 3 * SZ, P, s, false, 0.f, 0.f, 0.f);       // (S P)^T P = P S P
    }
  }
  float* out = p.Q + (int64_t)blockIdx.x * ss;
  const float inv_out = exponent == 0 ? (float)inv : ldexpf((float)inv, -exponent);
  for (int r = threadIdx.x >> 5; r < s; r += STEP_THREADS / 32)
    if constexpr (TS <= 2) {
      if ((threadIdx.x & 31) < s)
        out[r * s + (threadIdx.x & 31)] = (float)mats[Q + r * LD + (threadIdx.x & 31)] * inv_out;
    } else {
      for (int c = threadIdx.x & 31; c < s; c += 32) out[r * s + c] = (float)mats[Q + r * LD + c] * inv_out;
    }
}

template <int VEC, int TS>
__global__ void __launch_bounds__(256) apply_kernel(const SmallParams p) {
  extern __shared__ __align__(16) float Xs[];
  constexpr int LD = small_ld(TS);
  float* Qs = Xs + STAGE_FLOATS;                            // Qs[k][row], zeros beyond s
  const int64_t base = (int64_t)blockIdx.y * p.s * p.l;
  const int q = (p.s + 3) / 4, ld = 4 * q + 4;
  for (int e = threadIdx.x; e < (LD - 4) * LD; e += 256) Qs[e] = 0.f;
  __syncthreads();
  grid_dependency_wait();   // the momentum, too, is an earlier launch's
  const float* Q = p.Q + (int64_t)blockIdx.y * p.s * p.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int r = warp; r < p.s; r += 8)
    if constexpr (TS <= 2) {
      if (lane < p.s) Qs[lane * LD + r] = Q[r * p.s + lane];
    } else {
      for (int k = lane; k < p.s; k += 32) Qs[k * LD + r] = Q[r * p.s + k];
    }
  for (int c0 = blockIdx.x * p.tile_cols; c0 < p.l; c0 += gridDim.x * p.tile_cols) {
    const int cols = min(p.tile_cols, p.l - c0);
    __syncthreads();
    stage_columns<VEC, false>(p, base, c0, cols, Xs, ld);
    __syncthreads();
    // a warp takes four rows of 64 columns, a lane two of the columns
    const int items = q * ((cols + 63) >> 6);
#pragma unroll 1
    for (int it = warp; it < items; it += 8) {
      const int cb = q == 1 ? it : (int)__umulhi((uint32_t)it, p.inv_q), r = 4 * (it - cb * q);
      const int c = 64 * cb + lane;
      float o[2][4] = {};
#pragma unroll 2
      for (int k = 0; k < 4 * q; k += 4) {
        float4 x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          x[u] = *reinterpret_cast<const float4*>(Xs + min(c + 32 * u, cols - 1) * ld + k);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const float4 w = *reinterpret_cast<const float4*>(Qs + (k + kk) * LD + r);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float xv = kk == 0 ? x[u].x : kk == 1 ? x[u].y : kk == 2 ? x[u].z : x[u].w;
            o[u][0] = fmaf(w.x, xv, o[u][0]);
            o[u][1] = fmaf(w.y, xv, o[u][1]);
            o[u][2] = fmaf(w.z, xv, o[u][2]);
            o[u][3] = fmaf(w.w, xv, o[u][3]);
          }
        }
      }
      const int64_t step = p.u.tall ? 1 : p.l;
      const int nr = min(4, p.s - r);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int cc = c + 32 * u;
        if (cc >= cols) break;
        const int64_t at =
            base + (p.u.tall ? (int64_t)(c0 + cc) * p.s + r : (int64_t)r * p.l + c0 + cc);
        if (p.O) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < nr) p.O[at + i * step] = __float2bfloat16_rn(o[u][i]);
          continue;
        }
        float w[4] = {};
        uint32_t gone = 0;
        if (p.w_bf16) {
          const __nv_bfloat16* W = static_cast<const __nv_bfloat16*>(p.W_in) + at;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < nr) w[i] = __bfloat162float(W[i * step]);
        } else {
          const float* W = static_cast<const float*>(p.W_in) + at;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < nr) w[i] = W[i * step];
        }
        if (p.u.mask) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < nr && p.u.mask[at + i * step] != 0) gone |= 1u << i;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= nr) break;
          const float v = (gone >> i) & 1u ? 0.f : fmaf(-p.rate, o[u][i], p.keep * w[i]);
          if (p.w_bf16) static_cast<__nv_bfloat16*>(p.W_out)[at + i * step] = __float2bfloat16_rn(v);
          else static_cast<float*>(p.W_out)[at + i * step] = v;
        }
      }
    }
  }
}

// long-side columns staged at a time
int small_tile(int64_t s) {
  const int ld = (int)round_up((size_t)s, 4) + 4;
  return STAGE_FLOATS / ld / 4 * 4;
}

// Chunks of the long side per matrix, at most 32 partial matrices: two CTAs per SM, and where that
// leaves a CTA several stages, one after another, up to eight (steps of 57 x 18 x 9804: 130 us, with two
// 161).
int small_chunks(int64_t batch, int64_t s, int64_t l) {
  int64_t want = ceil_div(2 * NUM_SMS, batch);
  const int64_t stages = l / small_tile(s), more = ceil_div(8 * NUM_SMS, batch);
  if (want < stages) want = stages < more ? stages : more;
  const int64_t most = ceil_div(l, 64);
  if (want > most) want = most;
  if (want > 32) want = 32;
  return (int)want;
}

template <typename K>
thanos_status_t launch_after(K kernel, dim3 grid, int threads, size_t smem, const SmallParams& p,
                             cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
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

template <int VEC, int TS>
thanos_status_t launch_apply(const SmallParams& p, dim3 grid, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  const size_t smem = STAGE_FLOATS * 4 + (small_ld(TS) - 4) * small_ld(TS) * 4;
  THANOS_CUDA(ensure_max_dyn_smem(apply_kernel<VEC, TS>, (int)smem, done));
  return launch_after(apply_kernel<VEC, TS>, grid, 256, smem, p, stream);
}

thanos_status_t small_side(const OrthogonalArgs& a, StepParams u, int s, int l, bool fine, void* part,
                           float* Q, int chunks, cudaStream_t stream) {
  SmallParams p = {};
  p.u = u;
  p.part = part;
  p.Q = Q;
  p.s = s;
  p.l = l;
  p.chunk_cols = (int)round_up((size_t)ceil_div(l, chunks), 4);
  p.chunks = (int)ceil_div(l, p.chunk_cols);
  p.tile_cols = small_tile(s);
  const int q = (s + 3) / 4;
  p.inv_q = (uint32_t)(((1ull << 32) + q - 1) / q);
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
  const bool wide = a.n % 4 == 0;
  // The steps are a chain on one CTA per matrix: CTAs that share an SM slow one another down, so they
  // ask for more shared memory than half of an SM's, and spread out.
  const size_t stage = STAGE_FLOATS * 4, squares = 116 * 1024;
  static_assert(5 * small_size(4) * 4 <= 116 * 1024, "five matrices");
  const dim3 chunks_grid((unsigned)p.chunks, (unsigned)a.batch), one((unsigned)a.batch);
  if (fine) {
    if (wide) gram_kernel<4, true><<<chunks_grid, 256, stage, stream>>>(p);
    else gram_kernel<1, true><<<chunks_grid, 256, stage, stream>>>(p);
  } else {
    if (wide) gram_kernel<4, false><<<chunks_grid, 256, stage, stream>>>(p);
    else gram_kernel<1, false><<<chunks_grid, 256, stage, stream>>>(p);
  }
  THANOS_CHECK_LAUNCH();
  static_assert(5 * small_size(2) * 8 <= 116 * 1024, "five matrices in fp64");
  static std::atomic<unsigned long long> done1{0}, done2{0}, done4{0}, fine1{0}, fine2{0};
  const auto steps = [&](auto kernel, std::atomic<unsigned long long>& done) -> thanos_status_t {
    THANOS_CUDA(ensure_max_dyn_smem(kernel, (int)squares, done));
    return launch_after(kernel, one, STEP_THREADS, squares, p, stream);
  };
  // one entry of a product a thread, four or sixteen
  if (s <= 16) {
    THANOS_TRY(fine ? steps(steps_kernel<1, double>, fine1) : steps(steps_kernel<1, float>, done1));
  } else if (s <= 32) {
    THANOS_TRY(fine ? steps(steps_kernel<2, double>, fine2) : steps(steps_kernel<2, float>, done2));
  } else {
    THANOS_TRY(steps(steps_kernel<4, float>, done4));
  }
  // tiles of the apply pass: enough for the device, four to a thread at least
  int tile = p.tile_cols;
  while (tile > 128 && ceil_div(l, tile) * a.batch < 2 * NUM_SMS) tile = tile / 2 / 4 * 4;
  p.tile_cols = tile;
  int64_t blocks = ceil_div(l, tile);
  if (blocks * a.batch > 16 * NUM_SMS) blocks = ceil_div(16 * NUM_SMS, a.batch);
  const dim3 grid((unsigned)blocks, (unsigned)a.batch);
  if (wide) return s <= 32 ? launch_apply<4, 2>(p, grid, stream) : launch_apply<4, 4>(p, grid, stream);
  return s <= 32 ? launch_apply<1, 2>(p, grid, stream) : launch_apply<1, 4>(p, grid, stream);
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
  size_t small = 0, wide = 0;
  if (s <= SMALL_SIDE)
    small = 256 +
            round_up(k * small_chunks(batch > 0 ? batch : 1, s, l) * round_up(s, 4) * round_up(s, 4) *
                         (s <= SMALL_SIDE_FINE ? 8 : 4),
                     256) +
            round_up(k * s * s * 4, 256);
  if (s > SMALL_SIDE_FINE)
    wide = 256 + round_up(k * MAX_PARTS * 8, 256) + 2 * round_up(k * round_up(s, 8) * 4, 256) +
           2 * round_up(2 * k * s * round_up(l, 8) * 2, 256) +
           2 * round_up(2 * k * s * round_up(s, 8) * 2, 256);
  return small > wide ? small : wide;
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
  const bool fine = a.W_out && a.wdtype == THANOS_F32;
  if (s <= (fine ? SMALL_SIDE_FINE : SMALL_SIDE)) {
    const int chunks = small_chunks(a.batch, s, l);
    const size_t s4 = round_up((size_t)s, 4);
    char* parts = ar.take<char>(k * chunks * s4 * s4 * (fine ? 8 : 4));
    float* Q = ar.take<float>(k * s * s);
    if (!ar.ok()) return THANOS_ERR_WORKSPACE;
    return small_side(a, sp, s, l, fine, parts, Q, chunks, stream);
  }
  double* part = ar.take<double>(k * MAX_PARTS);
  __half* X[2][2];
  for (auto& x : X) {
    x[0] = ar.take<__half>(2 * k * s * ldx);
    x[1] = x[0] + k * s * ldx;
  }
  __half* S = ar.take<__half>(2 * k * s * lds);
  __half* P = ar.take<__half>(2 * k * s * lds);
  float* s_diag = ar.take<float>(k * lds);
  float* p_diag = ar.take<float>(k * lds);
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
  g.fine = fine;
  g.status = status;
  g.S = S;
  g.Pm = P;
  if (s <= DIAG_SIDE) {
    g.s_diag = s_diag;
    g.p_diag = p_diag;
  }
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
