// The orthogonalised update: Newton-Schulz iteration X <- a X + (b S + c S S) X, S = X X^T, on the
// shorter side of each matrix, and the optimiser step around it.
#include "recovery.cuh"
#include "simt_gemm.cuh"

namespace thanos {
namespace {

constexpr int NORM_BLOCKS = 64;

__device__ __forceinline__ float load_any(const void* p, int bf16, int64_t e) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[e])
              : static_cast<const float*>(p)[e];
}

struct StepParams {
  const void* G;
  float* M_out;
  const float* M_in;
  const uint8_t* mask;
  int g_bf16, nesterov, tall;
  float momentum;
  int m, n;
};

// One element's input to the iteration; writes the new momentum.
__device__ __forceinline__ float update_of(const StepParams& p, int64_t e) {
  const bool gone = p.mask && p.mask[e] != 0;
  float g = gone ? 0.f : load_any(p.G, p.g_bf16, e);
  if (p.M_out) {
    const float mo = fmaf(p.momentum, p.M_in[e], g);
    p.M_out[e] = mo;
    g = gone ? 0.f : (p.nesterov ? fmaf(p.momentum, mo, g) : mo);
  }
  return g;
}

// X [s, l] (transposed when the matrix is tall) and the sum of squares by block.
__global__ void __launch_bounds__(256)
load_kernel(const StepParams p, float* __restrict__ X, double* __restrict__ part) {
  const int64_t mn = (int64_t)p.m * p.n, base = (int64_t)blockIdx.y * mn;
  double sum = 0.0;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < mn; e += 256ll * NORM_BLOCKS) {
    const float v = update_of(p, base + e);
    const int64_t row = e / p.n, col = e - row * p.n;
    X[base + (p.tall ? col * p.m + row : e)] = v;
    sum += (double)v * (double)v;
  }
  __shared__ double red[256];
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * NORM_BLOCKS + blockIdx.x] = red[0];
}

__global__ void __launch_bounds__(256)
scale_kernel(float* __restrict__ X, const double* __restrict__ part, int64_t mn, float eps) {
  double s = 0.0;
  for (int i = 0; i < NORM_BLOCKS; ++i) s += part[(int64_t)blockIdx.y * NORM_BLOCKS + i];
  const float d = (float)sqrt(s) + eps;
  float* x = X + (int64_t)blockIdx.y * mn;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < mn; e += 256ll * gridDim.x) x[e] /= d;
}

// D = alpha A op(B) + beta C
template <bool TB>
__global__ void __launch_bounds__(256)
gemm_kernel(float* __restrict__ D, const float* __restrict__ A, const float* __restrict__ B,
            const float* __restrict__ C, int M, int N, int K, float alpha, float beta, int64_t sd,
            int64_t sa, int64_t sb) {
  using Tile = SimtGemm<64, 64, 16, 4, 4, false, TB, float, float>;
  __shared__ float smem[Tile::SMEM_FLOATS];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  float acc[4][4] = {};
  Tile::run(A + blockIdx.z * sa, K, B + blockIdx.z * sb, TB ? K : N, M, N, m0, n0, 0, K, acc, smem);
  const int tx = threadIdx.x % Tile::TX, ty = threadIdx.x / Tile::TX;
  for (int a = 0; a < 4; ++a)
    for (int e = 0; e < 4; ++e) {
      const int r = m0 + Tile::row_of(ty, a), f = n0 + Tile::col_of(tx, e);
      if (r >= M || f >= N) continue;
      const int64_t at = blockIdx.z * sd + (int64_t)r * N + f;
      D[at] = alpha * acc[a][e] + (beta != 0.f ? beta * C[at] : 0.f);
    }
}

struct StoreParams {
  __nv_bfloat16* O;
  void* W_out;
  const void* W_in;
  const uint8_t* mask;
  int w_bf16, tall, m, n;
  float keep, rate;
};

__global__ void __launch_bounds__(256) store_kernel(const StoreParams p, const float* __restrict__ X) {
  const int64_t mn = (int64_t)p.m * p.n, base = (int64_t)blockIdx.y * mn;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < mn; e += 256ll * gridDim.x) {
    const int64_t row = e / p.n, col = e - row * p.n;
    const float o = X[base + (p.tall ? col * p.m + row : e)];
    if (p.O) {
      p.O[base + e] = __float2bfloat16_rn(o);
    } else {
      float w = fmaf(-p.rate, o, p.keep * load_any(p.W_in, p.w_bf16, base + e));
      if (p.mask && p.mask[base + e] != 0) w = 0.f;
      if (p.w_bf16) static_cast<__nv_bfloat16*>(p.W_out)[base + e] = __float2bfloat16_rn(w);
      else static_cast<float*>(p.W_out)[base + e] = w;
    }
  }
}

}  // namespace

size_t orthogonal_workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  const size_t s = (size_t)(m < n ? m : n), k = (size_t)batch;
  return 256 + round_up(k * NORM_BLOCKS * 8, 256) + 2 * round_up(k * (size_t)m * (size_t)n * 4, 256) +
         2 * round_up(k * s * s * 4, 256);
}

thanos_status_t orthogonal_impl(const OrthogonalArgs& a, void* workspace, size_t ws_bytes,
                                cudaStream_t stream) {
  const int s = (int)(a.m < a.n ? a.m : a.n), l = (int)(a.m < a.n ? a.n : a.m);
  const size_t mn = (size_t)a.m * a.n, ss = (size_t)s * s, k = (size_t)a.batch;
  Arena ar(workspace, ws_bytes);
  int32_t* status = ar.take<int32_t>(64);
  double* part = ar.take<double>(k * NORM_BLOCKS);
  float* X = ar.take<float>(k * mn);
  float* X2 = ar.take<float>(k * mn);
  float* S = ar.take<float>(k * ss);
  float* P = ar.take<float>(k * ss);
  if (!ar.ok()) return THANOS_ERR_WORKSPACE;
  THANOS_CUDA(cudaMemsetAsync(status, 0, 16, stream));
  StepParams sp = {a.G, a.M_out, a.M_in, a.mask, a.gdtype == THANOS_BF16, a.nesterov,
                   a.m > a.n, a.momentum, (int)a.m, (int)a.n};
  load_kernel<<<dim3(NORM_BLOCKS, (unsigned)k), 256, 0, stream>>>(sp, X, part);
  THANOS_CHECK_LAUNCH();
  scale_kernel<<<dim3(256, (unsigned)k), 256, 0, stream>>>(X, part, (int64_t)mn, a.eps);
  THANOS_CHECK_LAUNCH();
  const unsigned gs = (unsigned)ceil_div(s, 64), gl = (unsigned)ceil_div(l, 64);
  for (int it = 0; it < a.steps; ++it) {
    gemm_kernel<true><<<dim3(gs, gs, (unsigned)k), 256, 0, stream>>>(
        S, X, X, nullptr, s, s, l, 1.f, 0.f, (int64_t)ss, (int64_t)mn, (int64_t)mn);
    THANOS_CHECK_LAUNCH();
    gemm_kernel<true><<<dim3(gs, gs, (unsigned)k), 256, 0, stream>>>(
        P, S, S, S, s, s, s, a.coef[2], a.coef[1], (int64_t)ss, (int64_t)ss, (int64_t)ss);
    THANOS_CHECK_LAUNCH();
    gemm_kernel<false><<<dim3(gl, gs, (unsigned)k), 256, 0, stream>>>(
        X2, P, X, X, s, l, s, 1.f, a.coef[0], (int64_t)mn, (int64_t)ss, (int64_t)mn);
    THANOS_CHECK_LAUNCH();
    float* t = X;
    X = X2;
    X2 = t;
  }
  StoreParams st = {a.O, a.W_out, a.W_in, a.mask, a.wdtype == THANOS_BF16, a.m > a.n, (int)a.m,
                    (int)a.n, a.keep, a.rate};
  store_kernel<<<dim3(256, (unsigned)k), 256, 0, stream>>>(st, X);
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

}  // namespace thanos
