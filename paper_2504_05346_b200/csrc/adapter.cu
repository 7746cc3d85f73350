// The projection with low-rank adapters, forward and backward:
//   V[t] = X[t] A_i^T,  Y[t] = X[t] W^T + s_i V[t] B_i^T
//   U[t] = s_i dY[t] B_i,  dX[t] = dY[t] W + U[t] A_i,  dA_i = sum_t U[t]^T X[t],
//   dB_i = s_i sum_t dY[t]^T V[t]
#include "recovery.cuh"
#include "simt_gemm.cuh"

namespace thanos {
namespace {

template <typename E>
__device__ __forceinline__ E from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

// The token's adapter, or -1 for none and for values that name no adapter.
__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ index, int64_t t, int n) {
  const int i = n > 0 ? index[t] : -1;
  return i >= 0 && i < n ? i : -1;
}

// out[t, j] = f sum_k in[t, k] P_i(j, k): forward P = A_i [r, K], f = 1; backward P(j, k) = B_i[k, j],
// f = s_i.  One warp per (t, j); lanes stride over k and meet in a fixed shuffle order.
template <typename E, bool BACK>
__global__ void __launch_bounds__(256)
shrink_kernel(float* __restrict__ out, const E* __restrict__ in, int64_t ldi,
              const E* __restrict__ P, const int32_t* __restrict__ index,
              const float* __restrict__ scale, int64_t T, int K, int n, int r,
              int32_t* __restrict__ status) {
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (w >= T * r) return;
  const int64_t t = w / r;
  const int j = (int)(w - t * r);
  const int i = adapter_of(index, t, n);
  if (lane == 0 && j == 0 && index[t] != -1 && i < 0)
    atomicCAS(status, 0, (int)THANOS_ERR_INVALID_ARG);
  float s = 0.f;
  if (i >= 0) {
    const E* x = in + t * ldi;
    const E* p = P + (int64_t)i * r * K + (BACK ? (int64_t)j : (int64_t)j * K);
    const int64_t step = BACK ? r : 1;
    for (int k = lane; k < K; k += 32) s = fmaf(to_float(x[k]), to_float(p[k * step]), s);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (BACK) s *= scale[i];
  }
  if (lane == 0) out[w] = s;
}

// forward: out[t, f] = sum_k in[t, k] W[f, k] + s_i sum_j R[t, j] B_i[f, j]
// backward: out[t, f] = sum_k in[t, k] W[k, f] + sum_j R[t, j] A_i[j, f]
template <typename E, bool BACK>
__global__ void __launch_bounds__(256)
project_kernel(E* __restrict__ out, int64_t ldo, const E* __restrict__ in, int64_t ldi,
               const E* __restrict__ W, int64_t ldw, const float* __restrict__ R,
               const E* __restrict__ P, const int32_t* __restrict__ index,
               const float* __restrict__ scale, int T, int F, int K, int n, int r) {
  using Tile = SimtGemm<64, 64, 16, 4, 4, false, !BACK, E, E>;
  __shared__ float smem[Tile::SMEM_FLOATS];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  float acc[4][4] = {};
  Tile::run(in, ldi, W, ldw, T, F, m0, n0, 0, K, acc, smem);
  const int tx = threadIdx.x % Tile::TX, ty = threadIdx.x / Tile::TX;
  for (int a = 0; a < 4; ++a) {
    const int t = m0 + Tile::row_of(ty, a);
    if (t >= T) continue;
    const int i = adapter_of(index, t, n);
    for (int e = 0; e < 4; ++e) {
      const int f = n0 + Tile::col_of(tx, e);
      if (f >= F) continue;
      float v = acc[a][e];
      if (i >= 0) {
        float s = 0.f;
        for (int j = 0; j < r; ++j) {
          const E p = BACK ? P[((int64_t)i * r + j) * F + f] : P[((int64_t)i * F + f) * r + j];
          s = fmaf(R[(int64_t)t * r + j], to_float(p), s);
        }
        v += BACK ? s : scale[i] * s;
      }
      out[(int64_t)t * ldo + f] = from_float<E>(v);
    }
  }
}

// grad_i(j, f) = g sum over the adapter's tokens, ascending, of R[t, j] Z[t, f]
//   dA: g = 1, R = U, Z = X, stored [n, r, F];   dB: g = s_i, R = V, Z = dY, stored [n, F, r]
template <typename E, bool IS_B>
__global__ void __launch_bounds__(256)
grad_kernel(float* __restrict__ out, const float* __restrict__ R, const E* __restrict__ Z,
            int64_t ldz, const int32_t* __restrict__ index, const float* __restrict__ scale,
            int64_t T, int F, int n, int r, int accumulate) {
  const int f = blockIdx.x * 256 + threadIdx.x;
  const int64_t ij = blockIdx.y + (int64_t)blockIdx.z * 65535;
  if (f >= F || ij >= (int64_t)n * r) return;
  const int i = (int)(ij / r), j = (int)(ij - (int64_t)i * r);
  float s = 0.f;
  for (int64_t t = 0; t < T; ++t)
    if (index[t] == i) s = fmaf(R[t * r + j], to_float(Z[t * ldz + f]), s);
  float* o = out + (IS_B ? ((int64_t)i * F + f) * r + j : ij * F + f);
  if (IS_B) s *= scale[i];
  *o = accumulate ? *o + s : s;
}

template <typename E, bool BACK>
thanos_status_t project(const AdapterArgs& a, const float* R, cudaStream_t stream) {
  const int F = (int)(BACK ? a.b : a.c), K = (int)(BACK ? a.c : a.b);
  for (int64_t t0 = 0; t0 < a.T; t0 += 65535 * 64) {
    const int64_t nt = a.T - t0 < 65535 * 64 ? a.T - t0 : 65535 * 64;
    dim3 grid((unsigned)ceil_div(F, 64), (unsigned)ceil_div(nt, 64));
    project_kernel<E, BACK><<<grid, 256, 0, stream>>>(
        static_cast<E*>(a.out) + t0 * a.ldo, a.ldo, static_cast<const E*>(a.in) + t0 * a.ldi, a.ldi,
        static_cast<const E*>(a.W), a.ldw, R + t0 * a.r,
        static_cast<const E*>(BACK ? a.A : a.B), a.index + t0, a.scale, (int)nt, F, K, (int)a.n,
        a.r);
    THANOS_CHECK_LAUNCH();
  }
  return THANOS_OK;
}

template <typename E>
thanos_status_t forward(const AdapterArgs& a, int32_t* status, float* V, cudaStream_t stream) {
  if (a.n > 0) {
    const int64_t warps = a.T * a.r;
    shrink_kernel<E, false><<<(unsigned)ceil_div(warps, 8), 256, 0, stream>>>(
        V, static_cast<const E*>(a.in), a.ldi, static_cast<const E*>(a.A), a.index, a.scale, a.T,
        (int)a.b, (int)a.n, a.r, status);
    THANOS_CHECK_LAUNCH();
  }
  return project<E, false>(a, V, stream);
}

template <typename E>
thanos_status_t backward(const AdapterArgs& a, int32_t* status, float* U, cudaStream_t stream) {
  if (a.n > 0) {
    const int64_t warps = a.T * a.r;
    shrink_kernel<E, true><<<(unsigned)ceil_div(warps, 8), 256, 0, stream>>>(
        U, static_cast<const E*>(a.in), a.ldi, static_cast<const E*>(a.B), a.index, a.scale, a.T,
        (int)a.c, (int)a.n, a.r, status);
    THANOS_CHECK_LAUNCH();
  }
  if (a.out) THANOS_TRY((project<E, true>(a, U, stream)));
  if (a.dA) {
    const int64_t nr = a.n * a.r;
    const unsigned gy = (unsigned)(nr < 65535 ? nr : 65535), gz = (unsigned)ceil_div(nr, 65535);
    grad_kernel<E, false><<<dim3((unsigned)ceil_div(a.b, 256), gy, gz), 256, 0, stream>>>(
        a.dA, U, static_cast<const E*>(a.X), a.ldx, a.index, a.scale, a.T, (int)a.b, (int)a.n, a.r,
        a.accumulate);
    THANOS_CHECK_LAUNCH();
    grad_kernel<E, true><<<dim3((unsigned)ceil_div(a.c, 256), gy, gz), 256, 0, stream>>>(
        a.dB, a.Vin, static_cast<const E*>(a.in), a.ldi, a.index, a.scale, a.T, (int)a.c, (int)a.n,
        a.r, a.accumulate);
    THANOS_CHECK_LAUNCH();
  }
  return THANOS_OK;
}

}  // namespace

size_t adapter_workspace_bytes(bool, int64_t T, int64_t, int64_t, int64_t, int r, thanos_dtype_t) {
  return 256 + round_up((size_t)T * (size_t)r * 4, 256);
}

thanos_status_t adapter_forward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                     cudaStream_t stream) {
  Arena ar(workspace, ws_bytes);
  int32_t* status = ar.take<int32_t>(64);
  float* V = ar.take<float>((size_t)a.T * a.r);
  if (!ar.ok()) return THANOS_ERR_WORKSPACE;
  if (a.V) V = a.V;
  THANOS_CUDA(cudaMemsetAsync(status, 0, 16, stream));
  return a.dtype == THANOS_F32 ? forward<float>(a, status, V, stream)
                               : forward<__nv_bfloat16>(a, status, V, stream);
}

thanos_status_t adapter_backward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                      cudaStream_t stream) {
  Arena ar(workspace, ws_bytes);
  int32_t* status = ar.take<int32_t>(64);
  float* U = ar.take<float>((size_t)a.T * a.r);
  if (!ar.ok()) return THANOS_ERR_WORKSPACE;
  THANOS_CUDA(cudaMemsetAsync(status, 0, 16, stream));
  return a.dtype == THANOS_F32 ? backward<float>(a, status, U, stream)
                               : backward<__nv_bfloat16>(a, status, U, stream);
}

}  // namespace thanos
