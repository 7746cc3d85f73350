// The adapted projection on fp32 operands.
//
// The wide product runs on the tensor cores with fp32 accuracy: three bf16 planes per operand, six
// products of planes (proj_gemm.cu, whose epilogue adds the adapter's part in fp32 as well).  The
// planes are made here, in the same launch that computes the skinny product V (or U) in fp32.  The
// adapters' gradients are plain fp32 sums, bound by reading their operands.
//
//   front_f32_kernel    planes of the activations and of W; V or U, a warp per token and eight ranks, or
//                       the planes that PROJ_SHRINK32 computes it from
//   proj_gemm           out = in W^T (or in W) + the adapter's part
//   grad_f32_kernel     both gradients: 32 features and up to 8 ranks of one adapter per CTA, eight
//                       warps share the adapter's tokens, in the order of sort_tokens
#include "adapter_grad.cuh"
#include "packed.cuh"
#include "proj_gemm.cuh"
#include "recovery.cuh"

namespace thanos {
namespace {

__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ index, int64_t t, int n) {
  const int i = n > 0 ? index[t] : -1;
  return i >= 0 && i < n ? i : -1;
}

struct SplitJob {
  const float* src = nullptr;
  int64_t ld = 0;
  int64_t rows = 0;
  int cols = 0;
  __nv_bfloat16* planes = nullptr;  // [3][rows, ldp]
  int64_t ldp = 0;
  int blocks = 0;
};

struct Front32Params {
  SplitJob in, w, p;     // p: the narrow factor A, where the skinny product runs on the tensor cores
  int n_turn;            // or B_i^T, turned on the way: blocks
  __nv_bfloat16* turned; // [3][n r, turn_ld]
  int64_t turn_ld;
  int32_t* status;       // cleared here
  float* R;              // [T, r]
  const float* P;        // forward: A [n, r, K]; backward: B [n, K, r]
  const int32_t* index;
  const float* scale;    // backward: s_i
  int64_t T;
  int K, n, r, back;
};

// What bf16 cannot hold by rounding alone.  Infinities and NaN: the planes are +-1, 0 and the value
// itself, because the last plane meets only the first one of the other operand (the products are mm,
// hl, lh, hm, mh and hh), so the value is multiplied by the other operand once, and never by a zero
// that is only one of its planes: infinity times 2 is infinity and infinity times 0 is NaN, as in
// fp32.  (Factors below 2^-133 count as zeros here.)  Finite values that would round to infinity:
// the first plane is bf16's largest, the others hold the rest.
constexpr float BF16_LARGEST = 0x1.FEp127f;
__device__ __forceinline__ bool fits_bf16(float x) { return fabsf(x) <= BF16_LARGEST; }
__device__ __forceinline__ void store_split_odd(__nv_bfloat16* p, int64_t plane, float x) {
  if (isfinite(x)) {
    const float h = fits_bf16(x) ? __bfloat162float(__float2bfloat16_rn(x)) : copysignf(BF16_LARGEST, x);
    const __nv_bfloat16 m = __float2bfloat16_rn(x - h);
    p[0] = __float2bfloat16_rn(h);
    p[plane] = m;
    p[2 * plane] = __float2bfloat16_rn(x - h - __bfloat162float(m));
  } else {
    p[0] = __float2bfloat16_rn(copysignf(1.f, x));
    p[plane] = __float2bfloat16_rn(0.f);
    p[2 * plane] = __float2bfloat16_rn(x);
  }
}
__device__ __forceinline__ void store_split(__nv_bfloat16* p, int64_t plane, float x) {
  if (fits_bf16(x)) store_split3(p, plane, x);
  else store_split_odd(p, plane, x);
}

// A warp per row in turn, so that no index has to be divided.
__device__ void split_job(const SplitJob& s, int blk) {
  const int64_t plane = s.rows * s.ldp;
  const int lane = threadIdx.x & 31;
  const bool wide = s.cols % 4 == 0 && s.ld % 4 == 0;
  for (int64_t row = (int64_t)blk * 8 + (threadIdx.x >> 5); row < s.rows; row += 8ll * s.blocks) {
    const float* src = s.src + row * s.ld;
    __nv_bfloat16* dst = s.planes + row * s.ldp;
    if (wide) {
#pragma unroll 2
      for (int c = 4 * lane; c < s.cols; c += 128) {
        const float4 x = *reinterpret_cast<const float4*>(src + c);
        float o[4] = {x.x, x.y, x.z, x.w};
        if (!(fits_bf16(x.x) && fits_bf16(x.y) && fits_bf16(x.z) && fits_bf16(x.w))) {
#pragma unroll 1
          for (int k = 0; k < 4; ++k) store_split_odd(dst + c + k, plane, src[c + k]);
          continue;
        }
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) {
          uint32_t h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const __nv_bfloat16 b = __float2bfloat16_rn(o[k]);
            h[k] = __bfloat16_as_ushort(b);
            o[k] -= __bfloat162float(b);
          }
          *reinterpret_cast<uint2*>(dst + pl * plane + c) =
              make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        }
      }
    } else {
      for (int c = lane; c < s.cols; c += 32) store_split(dst + c, plane, src[c]);
    }
  }
}

// Planes of every B_i [K, r] turned round, 64 rows at a time through shared memory.
__device__ void turn_job(const Front32Params& p, int blk) {
  __shared__ float sh[32][65];
  const int tiles = (p.K + 63) / 64;
  const int64_t units = (int64_t)p.n * tiles, plane = (int64_t)p.n * p.r * p.turn_ld;
  for (int64_t u = blk; u < units; u += p.n_turn) {
    const int64_t i = u / tiles;
    const int k0 = (int)(u - i * tiles) * 64;
    for (int j0 = 0; j0 < p.r; j0 += 32) {
      const int nj = min(32, p.r - j0);
      __syncthreads();
      for (int e = threadIdx.x; e < 64 * nj; e += 256) {
        const int row = e / nj, j = e - row * nj;
        if (k0 + row < p.K) sh[j][row] = p.P[(i * p.K + k0 + row) * p.r + j0 + j];
      }
      __syncthreads();
      for (int e = threadIdx.x; e < 64 * nj; e += 256) {
        const int j = e >> 6, row = e & 63;
        if (k0 + row < p.K)
          store_split(p.turned + (i * p.r + j0 + j) * p.turn_ld + k0 + row, plane, sh[j][row]);
      }
    }
  }
}

constexpr int RANKS = 8;

__global__ void __launch_bounds__(256) front_f32_kernel(const Front32Params p) {
  grid_dependents_launch();
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
  int blk = blockIdx.x;
  if (blk < p.in.blocks) {
    split_job(p.in, blk);
    return;
  }
  blk -= p.in.blocks;
  if (blk < p.w.blocks) {
    split_job(p.w, blk);
    return;
  }
  blk -= p.w.blocks;
  if (blk < p.p.blocks) {
    split_job(p.p, blk);
    return;
  }
  blk -= p.p.blocks;
  if (blk < p.n_turn) {
    turn_job(p, blk);
    return;
  }
  blk -= p.n_turn;
  const int lane = threadIdx.x & 31;
  const int groups = (p.r + RANKS - 1) / RANKS;
  const int64_t w = (int64_t)blk * 8 + (threadIdx.x >> 5);
  if (w >= p.T * groups) return;
  const int64_t t = w / groups;
  const int j0 = (int)(w - t * groups) * RANKS, nj = min(RANKS, p.r - j0);
  const int i = adapter_of(p.index, t, p.n);
  float s[RANKS] = {};
  if (i >= 0) {
    const float* x = p.in.src + t * p.in.ld;
    const float* a = p.P + (int64_t)i * p.r * p.K + (p.back ? (int64_t)j0 : (int64_t)j0 * p.K);
    // ranks beyond the last read the last one again: a load under a condition is not issued ahead
    int at[RANKS];
    if (p.back && p.r % 4 == 0) {
      const int second = nj > 4 ? 4 : 0;
#pragma unroll 4
      for (int k = lane; k < p.K; k += 32) {
        const float xv = x[k];
        const float* ak = a + (int64_t)k * p.r;
        const float4 u = *reinterpret_cast<const float4*>(ak);
        const float4 w = *reinterpret_cast<const float4*>(ak + second);
        s[0] = fmaf(xv, u.x, s[0]);
        s[1] = fmaf(xv, u.y, s[1]);
        s[2] = fmaf(xv, u.z, s[2]);
        s[3] = fmaf(xv, u.w, s[3]);
        s[4] = fmaf(xv, w.x, s[4]);
        s[5] = fmaf(xv, w.y, s[5]);
        s[6] = fmaf(xv, w.z, s[6]);
        s[7] = fmaf(xv, w.w, s[7]);
      }
    } else if (p.back) {
#pragma unroll
      for (int j = 0; j < RANKS; ++j) at[j] = min(j, nj - 1);
#pragma unroll 4
      for (int k = lane; k < p.K; k += 32) {
        const float xv = x[k];
        const float* ak = a + (int64_t)k * p.r;
#pragma unroll
        for (int j = 0; j < RANKS; ++j) s[j] = fmaf(xv, ak[at[j]], s[j]);
      }
    } else {  // K is a multiple of 8
#pragma unroll
      for (int j = 0; j < RANKS; ++j) at[j] = min(j, nj - 1) * p.K;
#pragma unroll 2
      for (int k = 4 * lane; k < p.K; k += 128) {
        const float4 xv = *reinterpret_cast<const float4*>(x + k);
#pragma unroll
        for (int j = 0; j < RANKS; ++j) {
          const float4 av = *reinterpret_cast<const float4*>(a + at[j] + k);
          s[j] = fmaf(xv.x, av.x, s[j]);
          s[j] = fmaf(xv.y, av.y, s[j]);
          s[j] = fmaf(xv.z, av.z, s[j]);
          s[j] = fmaf(xv.w, av.w, s[j]);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < RANKS; ++j) {
    for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    if (lane == 0 && j < nj) p.R[t * p.r + j0 + j] = p.back && i >= 0 ? p.scale[i] * s[j] : s[j];
  }
}

constexpr int GRAD_TOKENS = 512;

struct Grad32Side {
  const float* Z;
  int64_t ldz;
  const float* R;
  const float* scale;
  float* out;
  int F, by_feature;
  const int8_t* Z8;     // packed activations in the place of Z (ldz: of the codes)
  const uint8_t* exps;
  int64_t lde;
};
struct Grad32Params {
  Grad32Side side[2];
  int tiles0;
  const int32_t* order;
  const int32_t* off;
  int n, r, accumulate;
};

__global__ void __launch_bounds__(256) grad_f32_kernel(const Grad32Params p) {
  __shared__ float red[8][RANKS][33];
  __shared__ int tok[GRAD_TOKENS];
  __shared__ __align__(16) float fac[GRAD_TOKENS * RANKS];
  __shared__ float step[GRAD_TOKENS];   // packed activations: 2^e of the token and these 32 features
  const Grad32Side& sd = blockIdx.x < p.tiles0 ? p.side[0] : p.side[1];
  const int f = ((int)blockIdx.x - (blockIdx.x < p.tiles0 ? 0 : p.tiles0)) * 32 + (threadIdx.x & 31);
  const int g = threadIdx.x >> 5;
  const int j0 = blockIdx.z * RANKS, nj = min(RANKS, p.r - j0);
  for (int64_t i = blockIdx.y; i < p.n; i += gridDim.y) {
    const int lo = p.off[i], hi = p.off[i + 1];
    const int64_t at = sd.by_feature ? (i * sd.F + f) * p.r + j0 + g
                                     : (i * p.r + j0 + g) * (int64_t)sd.F + f;
    if (hi == lo) {  // no tokens: zero, whatever the scale
      if (g < nj && f < sd.F && !p.accumulate) sd.out[at] = 0.f;
      continue;
    }
    // sums of a round, and of rounds: with many tokens one chain of additions would round away more
    // than it may (2^24 tokens: 3.5e-5 of the result)
    float s[RANKS] = {}, total[RANKS] = {};
    for (int q0 = lo; q0 < hi; q0 += GRAD_TOKENS) {
      // the tokens of this round and their factors once through shared memory
      const int nq = min(GRAD_TOKENS, hi - q0);
      __syncthreads();
      for (int e = threadIdx.x; e < nq; e += 256) tok[e] = p.order[q0 + e];
      __syncthreads();
      // eight loads in flight (one at a time: 34 us for 1000 tokens, 768 + 768 features, three adapters)
      const int rank = threadIdx.x & (RANKS - 1);   // 256 is a multiple of RANKS
      for (int e0 = threadIdx.x; e0 < nq * RANKS; e0 += 256 * 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int e = e0 + 256 * u;
          v[u] = e < nq * RANKS && rank < nj ? sd.R[(int64_t)tok[e / RANKS] * p.r + j0 + rank] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (e0 + 256 * u < nq * RANKS) fac[e0 + 256 * u] = v[u];
      }
      if (sd.Z8) {
        const int group = blockIdx.x;   // side 0: a CTA's 32 features are one group
        for (int e = threadIdx.x; e < nq; e += 256)
          step[e] = __uint_as_float((uint32_t)sd.exps[(int64_t)tok[e] * sd.lde + group] << 23);
      }
      __syncthreads();
      if (f < sd.F) {
        // sixteen tokens of a warp in flight, added in their order
        constexpr int FLIGHT = 16;
        for (int first = g; first < nq; first += 8 * FLIGHT) {
          float z[FLIGHT];
          if (sd.Z8) {
            // a byte with its sign turned is code + 128, as the low bits of 2^23 a float; a conversion
            // instruction takes as long as the eight products
            uint32_t u[FLIGHT];
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
              u[k] = first + 8 * k < nq ? (uint8_t)sd.Z8[(int64_t)tok[first + 8 * k] * sd.ldz + f] : 0x80u;
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
              z[k] = (__uint_as_float((u[k] ^ 0x80u) | 0x4B000000u) - 8388736.f) *
                     (first + 8 * k < nq ? step[first + 8 * k] : 0.f);
          } else {
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
              z[k] = first + 8 * k < nq ? sd.Z[(int64_t)tok[first + 8 * k] * sd.ldz + f] : 0.f;
          }
#pragma unroll
          for (int k = 0; k < FLIGHT; ++k) {
            if (first + 8 * k < nq) {
#pragma unroll
              for (int j = 0; j < RANKS; ++j)
                s[j] = fmaf(fac[(first + 8 * k) * RANKS + j], z[k], s[j]);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < RANKS; ++j) {
        total[j] += s[j];
        s[j] = 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < RANKS; ++j) red[g][j][threadIdx.x & 31] = total[j];
    __syncthreads();
    // thread (g, lane) adds rank g of its feature over the eight groups, in their order
    if (g < nj && f < sd.F) {
      float v = 0.f;
      for (int k = 0; k < 8; ++k) v += red[k][g][threadIdx.x & 31];
      if (sd.scale) v *= sd.scale[i];
      float* o = sd.out + at;
      *o = p.accumulate ? *o + v : v;
    }
    __syncthreads();
  }
}

struct Layout32 {
  int32_t* status;
  float* R;
  __nv_bfloat16* in;
  __nv_bfloat16* w;
  __nv_bfloat16* p;
  int32_t* order;
  int32_t* spare;
  int32_t* off;
  int64_t k8, w8;
};

// Where the skinny product is computed.  On the ALUs every token reads its adapter's narrow factor
// anew, whole lines of A_i forward, pieces of rows of B_i backward; on the tensor cores
// (PROJ_SHRINK32) the factors are split into planes first and the product is a launch of its own.
// 2000 tokens, K = 2048, one adapter, launch with the planes (25 us) and the product:
//   rank          16    32    64
//   forward   ALUs 41    54    75 us     tensor cores 32 to 35 us, but a launch that the wide product
//   backward  ALUs 62   157   282 us     waits for (16 adapters of rank 16, forward: 74 against 58 us)
// Adapters in excess of the tokens that use them are not worth their planes.
bool shrink_on_tensor_cores(bool back, int64_t T, int64_t n, int r) {
  return T * r >= (back ? 16384 : 65536) && n * r <= 2 * T;
}

template <typename Take>
void layout32(Layout32& L, bool back, int64_t T, int64_t c, int64_t b, int64_t n, int r, bool packed,
              Take take) {
  const int64_t K = back ? c : b;
  // Rows of whole 128-byte lines: TMA fetches a tile's row that straddles two lines twice (c = b =
  // 1000, 2000 tokens: the wide product takes 46 us instead of 78).
  L.k8 = (int64_t)round_up((size_t)K, 64);
  L.w8 = back ? (int64_t)round_up((size_t)b, 64) : L.k8;  // W's planes keep W's own rows
  L.status = static_cast<int32_t*>(take(256));
  L.R = static_cast<float*>(take((size_t)T * r * 4));
  L.in = static_cast<__nv_bfloat16*>(take((size_t)3 * T * L.k8 * 2));
  // packed weights are bf16 numbers: one plane
  L.w = static_cast<__nv_bfloat16*>(take((size_t)(packed ? 1 : 3) * c * L.w8 * 2));
  L.p = nullptr;
  if (shrink_on_tensor_cores(back, T, n, r))
    L.p = static_cast<__nv_bfloat16*>(take((size_t)3 * n * r * L.k8 * 2));
  L.order = L.spare = L.off = nullptr;
  if (back) {
    L.order = static_cast<int32_t*>(take((size_t)T * 4));
    L.spare = static_cast<int32_t*>(take((size_t)T * 4));
    L.off = static_cast<int32_t*>(take(((size_t)n + 1) * 4));
  }
}

// Terms of a sum of one launch (K = 8192: 1.0e-6 of the result; in one launch 65536: 9.1e-6, 262144:
// 3.8e-5).
constexpr int64_t LONGEST_SUM = 8192;

int split_blocks(int64_t rows) {
  const int64_t want = ceil_div(rows, 8);
  return (int)(want < 8 * NUM_SMS ? want : 8 * NUM_SMS);
}

}  // namespace

size_t adapter_f32_workspace_bytes(bool back, int64_t T, int64_t c, int64_t b, int64_t n, int r,
                                   bool packed) {
  size_t total = 0;
  Layout32 L;
  layout32(L, back, T, c, b, n, r, packed, [&](size_t bytes) -> void* {
    total += round_up(bytes, 256);
    return nullptr;
  });
  return total;
}

// forward: in = X, out = Y; backward: in = dY, out = dX (may be null)
thanos_status_t adapter_f32(bool back, const AdapterArgs& a, void* workspace, size_t ws_bytes,
                            cudaStream_t stream) {
  const bool packed = a.packed != nullptr;
  if (ws_bytes < adapter_f32_workspace_bytes(back, a.T, a.c, a.b, a.n, a.r, packed))
    return THANOS_ERR_WORKSPACE;
  char* at = static_cast<char*>(workspace);
  Layout32 L;
  layout32(L, back, a.T, a.c, a.b, a.n, a.r, packed, [&](size_t bytes) -> void* {
    void* q = at;
    at += round_up(bytes, 256);
    return q;
  });
  const int K = (int)(back ? a.c : a.b), F = (int)(back ? a.b : a.c);
  float* R = !back && a.V ? a.V : L.R;
  Front32Params f = {};
  f.status = L.status;
  f.in.src = static_cast<const float*>(a.in);
  f.in.ld = a.ldi;
  const bool tc = a.n > 0 && shrink_on_tensor_cores(back, a.T, a.n, a.r);
  if (a.out || tc) {
    f.in.rows = a.T;
    f.in.cols = K;
    f.in.planes = L.in;
    f.in.ldp = L.k8;
    f.in.blocks = split_blocks(a.T);
  }
  if (a.out && !packed) {
    f.w.src = static_cast<const float*>(a.W);
    f.w.ld = a.ldw;
    f.w.rows = a.c;
    f.w.cols = (int)a.b;
    f.w.planes = L.w;
    f.w.ldp = L.w8;
    f.w.blocks = split_blocks(a.c);
  }
  int64_t skinny = 0;
  if (a.n > 0) {
    f.R = R;
    f.P = static_cast<const float*>(back ? a.B : a.A);
    f.index = a.index;
    f.scale = a.scale;
    f.T = a.T;
    f.K = K;
    f.n = (int)a.n;
    f.r = a.r;
    f.back = back;
    if (!tc) {
      skinny = ceil_div(a.T * ceil_div(a.r, RANKS), 8);
    } else if (back) {
      const int64_t units = a.n * ceil_div(K, 64);
      f.n_turn = (int)(units < 4 * NUM_SMS ? units : 4 * NUM_SMS);
      f.turned = L.p;
      f.turn_ld = L.k8;
    } else {
      f.p.src = f.P;
      f.p.ld = K;
      f.p.rows = a.n * a.r;
      f.p.cols = K;
      f.p.planes = L.p;
      f.p.ldp = L.k8;
      f.p.blocks = split_blocks(f.p.rows);
    }
  }
  const int64_t blocks = f.in.blocks + f.w.blocks + f.p.blocks + f.n_turn + skinny;
  if (blocks > 0) {
    front_f32_kernel<<<(unsigned)blocks, 256, 0, stream>>>(f);
    THANOS_CHECK_LAUNCH();
    if (a.out && packed)
      THANOS_TRY(unpack_weights(L.w, L.w8, THANOS_BF16, *a.packed, a.c, a.b, stream, true));
    if (tc) {
      ProjArgs s;
      s.epi = PROJ_SHRINK32;
      s.M = (int)(a.n * a.r);
      s.N = (int)a.T;
      s.K = K;
      s.A = L.p;
      s.lda = L.k8;
      s.a_batch = a.n * a.r * L.k8;
      s.B = L.in;
      s.ldb = L.k8;
      s.b_batch = a.T * L.k8;
      s.status = L.status;
      s.V = R;
      s.index = a.index;
      s.scale = back ? a.scale : nullptr;
      s.n_adapters = (int)a.n;
      s.r = a.r;
      THANOS_TRY(proj_gemm(s, stream));
    }
    if (a.dA) THANOS_TRY(sort_tokens(a.index, a.T, a.n, L.order, L.spare, L.off, L.status, stream));
  } else {
    THANOS_CUDA(cudaMemsetAsync(L.status, 0, 16, stream));
  }
  if (a.out) {
    ProjArgs g;
    g.epi = PROJ_OUT32;
    g.M = F;
    g.N = (int)a.T;
    g.K = K;
    g.A = L.w;
    g.lda = L.w8;
    g.a_batch = a.c * L.w8;
    g.one_plane = packed ? 1 : 0;
    g.a_mn = back ? 1 : 0;
    g.B = L.in;
    g.ldb = L.k8;
    g.b_batch = a.T * L.k8;
    g.status = L.status;
    g.out = a.out;
    g.ldo = a.ldo;
    // A long k in pieces that are added in fp32, rounded to nearest: the tensor cores cut what they add to
    // an accumulator, and beyond 8192 there are no more slices to keep the chains of additions short.
    const int64_t pieces = ceil_div(K, LONGEST_SUM), blocks64 = ceil_div(K, 64);
    for (int64_t i = 0; i + 1 < pieces; ++i) {
      const int64_t k0 = 64 * (blocks64 * i / pieces), k1 = 64 * (blocks64 * (i + 1) / pieces);
      ProjArgs s = g;
      s.A = L.w + (back ? k0 * L.w8 : k0);
      s.B = L.in + k0;
      s.K = (int)(k1 - k0);
      s.add = i > 0;
      THANOS_TRY(proj_gemm(s, stream));
    }
    if (pieces > 1) {
      const int64_t k0 = 64 * (blocks64 * (pieces - 1) / pieces);
      g.A = L.w + (back ? k0 * L.w8 : k0);
      g.B = L.in + k0;
      g.K = (int)(K - k0);
      g.add = 1;
    }
    if (a.n > 0) {
      g.V = R;
      g.index = a.index;
      g.scale = back ? nullptr : a.scale;
      g.n_adapters = (int)a.n;
      g.r = a.r;
      g.P = back ? a.A : a.B;
      g.ldp = back ? a.b : a.r;
      g.p_adapter = back ? a.r * a.b : a.c * a.r;
    }
    THANOS_TRY(proj_gemm(g, stream));
  }
  if (a.dA) {
    Grad32Params g = {};
    g.side[0] = {static_cast<const float*>(a.X), a.X8 ? a.ldx8 : a.ldx, L.R, nullptr, a.dA, (int)a.b, 0,
                 a.X8, a.exps, a.lde};
    g.side[1] = {static_cast<const float*>(a.in), a.ldi, a.Vin, a.scale, a.dB, (int)a.c, 1,
                 nullptr, nullptr, 0};
    g.tiles0 = (int)ceil_div(a.b, 32);
    g.order = L.order;
    g.off = L.off;
    g.n = (int)a.n;
    g.r = a.r;
    g.accumulate = a.accumulate;
    const dim3 grid((unsigned)(g.tiles0 + ceil_div(a.c, 32)), (unsigned)(a.n < 65535 ? a.n : 65535),
                    (unsigned)ceil_div(a.r, RANKS));
    grad_f32_kernel<<<grid, 256, 0, stream>>>(g);
    THANOS_CHECK_LAUNCH();
  }
  return THANOS_OK;
}

}  // namespace thanos
