// The adapted projection of up to 16 tokens (fp32: 64) on 4-bit weights:
//   Y[t] = X[t] w^T + s_i V[t] B_i^T,   V[t] = X[t] A_i^T,   w^ = code scale
//
// Floor: reading the weights, half a byte each.  A warp takes 16 MT rows and 8 NT tokens, and of k a run
// of 64-column blocks; the warps of a CTA split k and add up in a fixed order (same inputs, same bits).
// In a block a lane reads eight bytes of each of its rows, which are 16 consecutive columns: which k a
// lane holds at which place of the operand does not matter, as long as both operands agree, so the
// activations are read the same way, straight from memory, once per warp.
//   code   (nibble | 0x3E80) is the bf16 number 2^-2 + 2^-9 nibble; less 2^-2 + 2^-6 it is 2^-9 code
//   scale  the block's products are summed apart and multiplied by the row's scale in fp32: four
//          multiplications per 16 x 8 tile and block instead of one per weight.  64 products of up to 8 x
//          are 2^9 x, which is what the codes' 2^-9 is for: a sum does not leave fp32's range where w^
//          would not, and the results take it back, exactly (those below 2^-117 had fewer bits to be
//          held in)
// fp32 activations go as three bf16 planes (cut, not rounded: 24 bits in all), three products.
//
// mma.sync and not tcgen05: at this width the tensor cores are a fifth busy, and codes that go to tensor
// memory need a permutation and a multiplication per pair more (packed_tc.cu).  One token: 4096 x 4096 4.7
// us, 11008 x 4096 9.6, 28672 x 8192 38 us (3.2 TB/s); 16 tokens: 6.8, 11.7 and 45 us.  The last of each comes
// from memory, the others, replayed, from L2; over a set of layers larger than L2 they take up to 0.5 us
// more.
// What bounds it: loads and decoding, neither full, that overlap in part only.  28672 x 8192 takes 24 us
// without the arithmetic and 35 with all loads from L1.  Of some 89 instructions for 16 x 64 weights half are
// integer and a third bf16 ones, at half rate both; the issue slots are 56 % used, and of a warp's time 38 %
// is waiting for loads: registers hold what is in flight, and 64 to 128 of them leave 16 to 32 warps on an
// SM.  16 tokens with adapters: 30 % of the slots, 55 % of the time; latency.
#include "packed_few.cuh"

namespace thanos {
namespace {

constexpr int SHRINK_RANKS = 4;

__device__ __forceinline__ int adapter_of(const int32_t* index, int t, int n) {
  const int i = index[t];
  return i >= 0 && i < n ? i : -1;
}

// ------------------------------------------------------------------------------ V[t] = X[t] A_i^T
// A CTA per token and four ranks, as many threads as a row has pieces of 16 bytes (1024 at most): one
// round of loads in flight, two at 11008 columns (256 threads, six rounds: 15 us there, beside products of
// 14).  Clears the status word of the call.
template <typename T>
__global__ void __launch_bounds__(1024) shrink_kernel(const FewParams p) {
  __shared__ float sh[SHRINK_RANKS][32];
  grid_dependents_launch();
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && tid == 0) *p.status = 0;
  const int groups = (p.r + SHRINK_RANKS - 1) / SHRINK_RANKS;
  const int t = blockIdx.x / groups, j0 = (blockIdx.x - t * groups) * SHRINK_RANKS;
  const int i = adapter_of(p.index, t, p.n);
  float s[SHRINK_RANKS] = {};
  if (i >= 0) {
    constexpr int VEC = 16 / sizeof(T);
    const T* x = static_cast<const T*>(p.X) + (int64_t)t * p.ldx;
    const T* a = static_cast<const T*>(p.A) + ((int64_t)i * p.r + j0) * p.b;
    for (int k = tid * VEC; k < p.b; k += (int)blockDim.x * VEC) {
      const uint4 xv = *reinterpret_cast<const uint4*>(x + k);
      const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
      for (int j = 0; j < SHRINK_RANKS; ++j) {
        if (j0 + j < p.r) {
          const uint4 av = *reinterpret_cast<const uint4*>(a + (int64_t)j * p.b + k);
          const uint32_t aw[4] = {av.x, av.y, av.z, av.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (VEC == 8) {
              s[j] = fmaf(__uint_as_float(xw[e] << 16), __uint_as_float(aw[e] << 16), s[j]);
              s[j] = fmaf(__uint_as_float(xw[e] & 0xFFFF0000u),
                          __uint_as_float(aw[e] & 0xFFFF0000u), s[j]);
            } else {
              s[j] = fmaf(__uint_as_float(xw[e]), __uint_as_float(aw[e]), s[j]);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < SHRINK_RANKS; ++j) {
    for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    if ((tid & 31) == 0) sh[j][tid >> 5] = s[j];
  }
  __syncthreads();
  if (tid < SHRINK_RANKS && j0 + tid < p.r) {
    float v = 0.f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) v += sh[tid][w];
    p.V[(int64_t)t * p.r + j0 + tid] = v;
  }
}

// --------------------------------------------------------------------------------------- products
// Codes j and j + 4 of a word of eight, times 2^-9, as a pair of bf16.
constexpr uint32_t CODE_BASE = 0x3E803E80u, CODE_ZERO = 0x3E883E88u;
constexpr float CODE_UNIT = 512.f;
__device__ __forceinline__ uint32_t codes_of(const Nibbles& nib, uint32_t w, int j) {
  const uint32_t v = nib(w, j), zero = CODE_ZERO;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                                   *reinterpret_cast<const __nv_bfloat162*>(&zero));
  return *reinterpret_cast<const uint32_t*>(&d);
}
// Eight activations, and as four pairs (x_j, x_j+4) in one plane or in three.
template <typename T>
struct Vec8;
template <>
struct Vec8<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* x, bool in) {
    v = in ? *reinterpret_cast<const uint4*>(x) : make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void pairs(uint32_t (&o)[1][4]) const {
    o[0][0] = __byte_perm(v.x, v.z, 0x5410);
    o[0][1] = __byte_perm(v.x, v.z, 0x7632);
    o[0][2] = __byte_perm(v.y, v.w, 0x5410);
    o[0][3] = __byte_perm(v.y, v.w, 0x7632);
  }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* x, bool in) {
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    a = in ? reinterpret_cast<const float4*>(x)[0] : zero;
    b = in ? reinterpret_cast<const float4*>(x)[1] : zero;
  }
  // The first plane keeps an infinity or NaN and the others are zero beside it: the codes are finite.
  __device__ __forceinline__ void pairs(uint32_t (&o)[3][4]) const {
    float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int pl = 0; pl < 3; ++pl) {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool odd = pl == 0 && !isfinite(v[e]);
        // cut to bf16; a NaN stays one
        h[e] = odd && isnan(v[e]) ? 0x7FFF0000u : __float_as_uint(v[e]) & 0xFFFF0000u;
        v[e] = odd ? 0.f : v[e] - __uint_as_float(h[e]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) o[pl][j] = __byte_perm(h[j], h[j + 4], 0x7632);
    }
  }
};

__device__ __forceinline__ uint2 load_codes(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];"
               : "=r"(v.x), "=r"(v.y)
               : "l"(p));
  return v;
}

// Two blocks of 64 columns at a time (one group of 128, or two of 64).  What a lane reads of them lies at
// fixed distances from pointers that move on, and nothing is tested: rows and tokens beyond the last are
// the last one's, and only their results are left out.  The columns from the last whole pair of blocks on
// are read with tests, by the last warp.  (16 rows at a time, every load with its own address and tests:
// 131 instructions for 16 x 64 weights instead of 89.)
template <typename T, int MT, int NT>
__device__ __forceinline__ void block_products(const Nibbles& nib, const uint2 (&w)[MT][2],
                                               const uint32_t (&s)[MT][2],
                                               const Vec8<T> (&x)[NT][2], float (&acc)[MT][NT][4]) {
  constexpr int PL = sizeof(T) == 2 ? 1 : 3;
  float sum[MT][NT][4];
#pragma unroll
  for (int half = 0; half < 2; ++half) {  // the lane's eight columns of the first, the second word
    uint32_t xb[NT][PL][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) x[j][half].pairs(xb[j]);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t lo = half ? w[i][0].y : w[i][0].x, hi = half ? w[i][1].y : w[i][1].x;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const uint32_t a[4] = {codes_of(nib, lo, 2 * v), codes_of(nib, hi, 2 * v),
                               codes_of(nib, lo, 2 * v + 1), codes_of(nib, hi, 2 * v + 1)};
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int pl = PL - 1; pl >= 0; --pl)
            mma_16816(sum[i][j], a, xb[j][pl][2 * v], xb[j][pl][2 * v + 1],
                      half == 0 && v == 0 && pl == PL - 1);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[i][j][e] = fmaf(__uint_as_float((s[i][e >> 1] & SCALE_BITS) << 16), sum[i][j][e],
                            acc[i][j][e]);
}

template <typename T, int MT, int NT, int GW>
__global__ void __launch_bounds__(32 * GW, (MT * NT == 1 ? 4 : MT * NT == 2 ? 3 : 2) * 8 / GW)
few_kernel(const FewParams p) {
  constexpr int ROWS = 16 * MT, TOKS = 8 * NT, GT = 32 * GW;
  __shared__ float part[GW][TOKS][ROWS + 4];
  if (p.n == 0 && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t4 = lane & 3;
  const int m0 = blockIdx.x * ROWS, t0 = blockIdx.y * TOKS;
  const int pairs = p.b >> 7;  // whole ones
  const int k0 = pairs * warp / GW, k1 = pairs * (warp + 1) / GW;

  const uint8_t* q[MT][2];
  const unsigned short* sc[MT][2];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = min(m0 + 16 * i + 8 * h + g, p.c - 1);
      q[i][h] = p.codes + (int64_t)row * p.ldq + 8 * t4 + (int64_t)k0 * 64;
      sc[i][h] = reinterpret_cast<const unsigned short*>(p.scales) + row +
                 (int64_t)((k0 << 7) >> p.shift) * p.c;
    }
  }
  const T* x[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
    x[j] = static_cast<const T*>(p.X) + (int64_t)min(t0 + 8 * j + g, p.T - 1) * p.ldx + 16 * t4 +
           (int64_t)k0 * 128;
  const int64_t second = p.shift == 6 ? p.c : 0, step = p.shift == 6 ? 2 * (int64_t)p.c : p.c;
  const Nibbles nib(CODE_BASE);
  float acc[MT][NT][4] = {};
#pragma unroll 1
  for (int k = k0; k < k1; ++k) {
    uint2 w[2][MT][2];
    uint32_t s[2][MT][2];
    Vec8<T> xr[2][NT][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          w[u][i][h] = load_codes(q[i][h] + 32 * u);
          s[u][i][h] = sc[i][h][u ? second : 0];
        }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int half = 0; half < 2; ++half) xr[u][j][half].load(x[j] + 64 * u + 8 * half, true);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        q[i][h] += 64;
        sc[i][h] += step;
      }
#pragma unroll
    for (int j = 0; j < NT; ++j) x[j] += 128;
    block_products<T, MT, NT>(nib, w[0], s[0], xr[0], acc);
    block_products<T, MT, NT>(nib, w[1], s[1], xr[1], acc);
  }
  if (warp == GW - 1) {  // k1 is the end of the whole pairs here
#pragma unroll 1
    for (int col = pairs * 128; col < p.b; col += 64) {
      uint2 w[MT][2];
      uint32_t s[MT][2];
      Vec8<T> xr[NT][2];
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          w[i][h] = load_codes(q[i][h]);
          s[i][h] = sc[i][h][0];
          q[i][h] += 32;
          sc[i][h] += second;
        }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
          xr[j][half].load(x[j] + 8 * half, col + 16 * t4 + 8 * half < p.b);
        x[j] += 64;
      }
      block_products<T, MT, NT>(nib, w, s, xr, acc);
    }
  }
  // ---- sums over the warps
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[warp][8 * j + 2 * t4 + (e & 1)][16 * i + g + 8 * (e >> 1)] = acc[i][j][e];
  __syncthreads();
  if (p.n > 0) grid_dependency_wait();
  for (int e = threadIdx.x; e < TOKS * ROWS; e += GT) {
    const int t = e / ROWS, m = e % ROWS;
    float v[1] = {};
#pragma unroll
    for (int u = 0; u < GW; ++u) v[0] += part[u][t][m];
    v[0] *= CODE_UNIT;
    const int row[1] = {m0 + m}, at[1] = {t0 + t};
    if (row[0] < p.c && at[0] < p.T) finish<T>(p, row, at, v);
  }
}

template <typename T, int MT, int NT, int GW = 8>
thanos_status_t launch(const FewParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ceil_div(p.c, 16 * MT), (unsigned)ceil_div(p.T, 8 * NT), 1);
  cfg.blockDim = dim3(32 * GW, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.n > 0 ? 1 : 0;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, few_kernel<T, MT, NT, GW>, p));
  return THANOS_OK;
}

template <typename T>
thanos_status_t forward_few(const FewParams& p, cudaStream_t stream) {
  if (p.n > 0) {
    const size_t pieces = round_up((size_t)p.b * sizeof(T) / 16, 32);
    shrink_kernel<T><<<(unsigned)(p.T * ceil_div(p.r, SHRINK_RANKS)),
                       (unsigned)(pieces < 1024 ? pieces : 1024), 0, stream>>>(p);
    THANOS_CHECK_LAUNCH();
  }
  // Two tiles of rows share a warp's activations, where there are rows enough for every SM.  With 16 tokens
  // these are then four warps to a CTA, more and smaller pieces for two CTAs' worth of registers: 11008 x
  // 4096 11.7 and 12.9 us, 28672 x 8192 45.4 and 48.8; below, eight: 4096 x 4096 6.8 and 7.1, 4096 x 11008
  // 13.7 and 15.2.  fp32 keeps eight: 9 tokens, 11008 x 4096, 4 adapters 33.3 us, with four 42.2 (without
  // adapters 30.7 and 31.0).
  const bool wide = p.c >= 32 * NUM_SMS;
  if (p.T <= 8) return wide ? launch<T, 2, 1>(p, stream) : launch<T, 1, 1>(p, stream);
  if constexpr (sizeof(T) == 4) {
    return launch<T, 2, 2>(p, stream);
  } else {
    if (p.T <= 16) return wide ? launch<T, 2, 2, 4>(p, stream) : launch<T, 1, 2>(p, stream);
    return packed_tiles(p, stream);
  }
}

}  // namespace

// Up to here the codes are turned into weights where they meet the activations; with more tokens they are
// unpacked once and multiplied as they would be from memory.  Replayed, both ways:
//   4096 x 4096     128 tokens   12.7 and 20.8 us    256 tokens   17.4 and 24.8 us
//   4096 x 11008    128 tokens   21.6 and 54.9       256 tokens   34.1 and 63.7
//   11008 x 4096    128 tokens   25.1 and 51.5       256 tokens   49.7 and 63.0    384 tokens  49.7 and 81.6
//   1024 x 4096                                      256 tokens   18.5 and 14.4
//   with adapters, 256 tokens    16 of rank 16    4 of rank 64    8 of rank 12
//     1024 x 4096                 29 and  23       66 and  46      31 and  22
//     4096 x 4096                 32 and  34       49 and  74      36 and  31
//     4096 x 11008                57 and  70       97 and 126      58 and  66
//     8192 x 8192                 72 and 102      102 and 199      77 and  99
//     11008 x 4096                81 and  79      111 and  83      95 and  73
//     28672 x 8192               271 and 274      316 and 280     294 and 263
//     12288 x 2048, three of rank 20: 88 and 44
//   320 tokens:     4096 x 4096, 8 of rank 16, 44 and 39;  4096 x 11008, 16 of rank 16, 102 and 78
//   fp32            2048 x 2048, 64 tokens   15.8 and 31.7;  768 x 768, 64 tokens   4.9 and 15.2;  11008 x
//     4096, 16 tokens 32, 64 tokens 97, 65 (unpacked) 77
// The number of tokens is all it looks at.  Over 288 sizes with adapters and 136 to 256 tokens 256 is the
// better limit in the mean (6 % above the faster way for each size; 128: 19 %), but not for each: few rows,
// ranks that are no multiple of 8, and tiles that fill little more than half of the SMs twice (11008 rows)
// lose to unpacking, up to the half of their time.  Rules on rows, tokens and rank that fit one half of the
// sizes did not fit the other: what decides is the shape of both launches.
bool packed_few_tokens(const AdapterArgs& a) { return a.T <= (a.dtype == THANOS_F32 ? 64 : 256); }

size_t packed_few_workspace_bytes(int64_t T, int r) { return 256 + round_up((size_t)T * r * 4, 256); }

thanos_status_t packed_forward_few(const AdapterArgs& a, const PackedWeights& w, void* workspace,
                                   cudaStream_t stream) {
  FewParams p = {};
  p.Y = a.out;
  p.ldy = a.ldo;
  p.X = a.in;
  p.ldx = a.ldi;
  p.codes = w.codes;
  p.ldq = w.ldq;
  p.scales = w.scales;
  p.A = a.A;
  p.B = a.B;
  p.index = a.index;
  p.scale = a.scale;
  p.status = static_cast<int32_t*>(workspace);
  p.V = a.V ? a.V : reinterpret_cast<float*>(static_cast<char*>(workspace) + 256);
  p.c = (int)a.c;
  p.b = (int)a.b;
  p.T = (int)a.T;
  p.n = (int)a.n;
  p.r = a.r;
  p.shift = w.group == 64 ? 6 : 7;
  return a.dtype == THANOS_BF16 ? forward_few<bf16>(p, stream) : forward_few<float>(p, stream);
}

}  // namespace thanos
