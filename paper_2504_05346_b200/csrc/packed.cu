// Weights in 4 bits with group scales and activations in 8 bits with group exponents: packing and
// reading back.
//
// Weights, groups of 64 or 128 columns of a row:   w^ = code scale,   code in -8 .. 7
//   scale = max |w| / 7, rounded to five significant bits;  code = w / scale, rounded, in -7 .. 7.
//   A code of three bits (or 8) times a scale of five is a number of eight: bf16 holds w^ exactly, and
//   the tensor cores multiply what the definition says.  Zeros stay zeros: a pruned weight stays pruned.
// Activations, groups of 32 columns of a row:   x^ = code 2^(e - 127),   code in -127 .. 127
//   the smallest power of two for which no code leaves that range.  bf16 holds x^ exactly, too.
//
// Floor: every value is read and written once.  A thread takes eight columns of four rows, whose loads are
// in flight together; the lanes of a group share its largest value by shuffles; numbers become codes and
// codes numbers by additions to 2^23 and byte permutations (a value at a time, with conversion instructions
// and divisions, weights took 132 us both ways).  11008 x 4096 in bf16: weights packed in 26.5 us (4.3
// TB/s) and unpacked in 26.2, activations in 26.4 (5.1 TB/s) and 24.6.  Packing weights issues in 82 % of
// the cycles; unpacking them in 54 %, and half of its warps' time is waiting for loads.
#include "packed.cuh"
#include "proj_gemm.cuh"

namespace thanos {
namespace {

using bf16 = __nv_bfloat16;
constexpr int PT = 256;
constexpr int RB = 4;  // rows of a thread, whose loads are in flight together

// Eight values as they are in memory.
template <typename T>
struct Raw {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void expand(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          x[2 * e] = __uint_as_float(w[e] << 16);
          x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        } else {
          x[4 * i + e] = __uint_as_float(w[e]);
        }
      }
    }
  }
};
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// The largest magnitude of LANES neighbouring lanes' values, as the bits of a float (they are ordered
// like the magnitudes, infinity and NaN above all).
template <int LANES, typename T>
__device__ __forceinline__ uint32_t group_top(const Raw<T>& raw) {
  uint32_t top = 0;
  if constexpr (sizeof(T) == 2) {  // two to a register, and the upper half of a float at the end
    const uint32_t w[4] = {raw.v[0].x, raw.v[0].y, raw.v[0].z, raw.v[0].w};
    uint32_t two = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) two = __vmaxu2(two, w[e] & 0x7FFF7FFFu);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, o));
    top = max(two << 16, two & 0xFFFF0000u);
  } else {
    float x[8];
    raw.expand(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  return top;
}

// A float of this size has whole numbers next to it: what is added to it is rounded to one, ties to even,
// which then stands in its low bits.
constexpr float WHOLE = 0x1.8p23f;

// A thread's place: eight columns from `col`, and RB rows from `row`, then again `rows` further on.
// blockDim.x vectors of a row, RB blockDim.y rows; all threads of a warp stay together.  Rows that follow
// one another share the 32 bytes that the weights' scales are fetched and written in.
struct Place {
  int64_t row, rows;
  int col;
  __device__ Place()
      : row(((int64_t)blockIdx.y * blockDim.y + threadIdx.y) * RB),
        rows((int64_t)gridDim.y * blockDim.y * RB),
        col((blockIdx.x * blockDim.x + threadIdx.x) * 8) {}
};

template <typename T>
__global__ void __launch_bounds__(PT) pack_act_kernel(int8_t* __restrict__ codes, int64_t ldc,
                                                      uint8_t* __restrict__ exps, int64_t lde,
                                                      const T* __restrict__ X, int64_t ldx, int64_t n,
                                                      int b) {
  const Place at;
  const bool in = at.col < b;
  const int64_t turns = (n + at.rows - 1) / at.rows;
  Raw<T> raw[RB];
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row0 = at.row + i * at.rows;
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (in && row < n) raw[u].load(X + row * ldx + at.col);
      else raw[u].clear();
    }
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      const uint32_t top = group_top<4>(raw[u]);
      if (!in || row >= n) continue;
      float x[8];
      raw[u].expand(x);
      // 64 to 128 steps of 2^e; one power of two more where 127.5 and above would round to 128 (where
      // that is no float, the code stays at 127)
      int e = max((int)(top >> 23) - 133, -126);
      const float high = __uint_as_float(top) * __uint_as_float((uint32_t)(127 - e) << 23);
      if (high >= 127.5f && e < 121) ++e;
      const bool odd = top >= 0x7F800000u;
      uint32_t q[8];
      if (!odd && e < 121) {
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = __float_as_uint(fmaf(x[k], inv, WHOLE));
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (odd)  // infinities keep their sign, what is beside them reads back as NaN
            q[k] = isinf(x[k]) ? (x[k] > 0.f ? 1u : 255u) : 0u;
          else
            q[k] = (uint32_t)max(-127, min(127, __float2int_rn(x[k] * 0x1p-121f)));
        }
      }
      uint32_t w[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        w[k] = __byte_perm(__byte_perm(q[4 * k], q[4 * k + 1], 0x0040),
                           __byte_perm(q[4 * k + 2], q[4 * k + 3], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(codes + row * ldc + at.col) = make_uint2(w[0], w[1]);
      if (at.col % ACT_GROUP == 0)
        exps[row * lde + at.col / ACT_GROUP] = odd ? 255 : top == 0 ? 0 : (uint8_t)(e + 127);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(PT) unpack_act_kernel(T* __restrict__ X, int64_t ldx,
                                                        const int8_t* __restrict__ codes, int64_t ldc,
                                                        const uint8_t* __restrict__ exps, int64_t lde,
                                                        int64_t n, int b) {
  const Place at;
  if (at.col >= b) return;
  for (int64_t row0 = at.row; row0 < n; row0 += at.rows) {
    uint2 w[RB];
    uint32_t e[RB];
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (row >= n) break;
      w[u] = *reinterpret_cast<const uint2*>(codes + row * ldc + at.col);
      e[u] = exps[row * lde + at.col / ACT_GROUP];
    }
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (row >= n) break;
      const float step = __uint_as_float(e[u] << 23);
      float x[8];
      // a byte with its sign turned is code + 128; as the low bits of 2^23 it is a float (the product and
      // the difference are exact)
      const uint32_t h[2] = {w[u].x ^ 0x80808080u, w[u].y ^ 0x80808080u};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        x[k] = (__uint_as_float(__byte_perm(h[k / 4], 0x4B000000u, 0x7440 + (k & 3))) - 8388736.f) *
               step;
      store8(X + row * ldx + at.col, x);
    }
  }
}

__device__ __forceinline__ float reciprocal(float x) {  // to 2^-23 of it
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// x / scale, rounded to the nearest whole number, ties to even, plus 8: in the low four bits.  The
// product with the reciprocal is off by 2^-19 at most, which matters next to a half only:
//   bf16   eight bits over five: a quotient is a half or 2^-10 and more from one, so what is within 2^-15
//          of a multiple of 2^-14 is taken for it;
//   fp32   the quotient itself is computed there (one value in thousands).
// A scale is 2^-126 at least and below 2^126: its reciprocal is a normal number.  It is at most 1/33 below
// a seventh of the largest value: no code leaves -7 .. 7.
template <typename T>
__device__ __forceinline__ uint32_t code_of(float x, float scale, float inv) {
  float q;
  if constexpr (sizeof(T) == 2) {
    constexpr float SNAP = 0x1.8p9f;  // numbers next to it are 2^-14 apart
    q = __fsub_rn(fmaf(x, inv, SNAP), SNAP);
  } else {
    q = x * inv;
    const float off = q - __fsub_rn(__fadd_rn(q, WHOLE), WHOLE);
    if (fabsf(fabsf(off) - 0.5f) < 0x1p-12f) q = __fdiv_rn(x, scale);
  }
  return __float_as_uint(__fadd_rn(q, WHOLE + 8.f));
}

// A seventh of a group's largest value with five significant bits, ties to even.
template <typename T>
__device__ __forceinline__ uint32_t scale_of(uint32_t top) {
  uint32_t bits;
  if constexpr (sizeof(T) == 2) {
    // a seventh of eight bits is a tie or 2^-10 and more from one: twelve bits say which
    bits = (__float_as_uint(__uint_as_float(top) * 0x1.24924ap-3f) + 0x400u) & 0xFFFFF800u;
  } else {
    bits = __float_as_uint(__fdiv_rn(__uint_as_float(top), 7.f));
  }
  const uint32_t s = (bits + 0x3FFFFu + ((bits >> 19) & 1u)) & 0xFFF80000u;
  return s < 0x00800000u ? 0u : s;  // below the normal numbers: zero
}

template <typename T, int GROUP>
__global__ void __launch_bounds__(PT) pack_w_kernel(uint8_t* __restrict__ codes, int64_t ldq,
                                                    bf16* __restrict__ scales,
                                                    const T* __restrict__ W, int64_t ldw, int64_t c,
                                                    int b, int wide) {
  const Place at;
  const bool in = at.col < b;
  const int64_t turns = (c + at.rows - 1) / at.rows;
  Raw<T> raw[RB];
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row0 = at.row + i * at.rows;
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (in && row < c) raw[u].load(W + row * ldw + at.col);
      else raw[u].clear();
    }
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      const uint32_t top = group_top<GROUP / 8>(raw[u]);
      if (at.col >= wide || row >= c) continue;
      float x[8];
      raw[u].expand(x);
      uint32_t s = scale_of<T>(top);
      const bool odd = top >= 0x7F800000u;
      if (odd) s = 0x7FC00000u;  // a group that is not finite reads back as NaN
      uint32_t w = 0x88888888u;
      if (s != 0u && !odd) {
        const float scale = __uint_as_float(s), inv = reciprocal(scale);
        w = 0;
#pragma unroll
        for (int k = 7; k >= 0; --k) w = (w << 4) + (code_of<T>(x[k], scale, inv) - __float_as_uint(WHOLE));
      }
      *reinterpret_cast<uint32_t*>(codes + row * ldq + at.col / 2) = w;
      if (in && at.col % GROUP == 0)
        scales[(int64_t)(at.col / GROUP) * c + row] = __ushort_as_bfloat16((unsigned short)(s >> 16));
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(PT) unpack_w_kernel(T* __restrict__ W, int64_t ldw,
                                                      const uint8_t* __restrict__ codes, int64_t ldq,
                                                      const bf16* __restrict__ scales, int64_t c,
                                                      int b, int group) {
  const Place at;
  grid_dependents_launch();
  const Nibbles nib;
  for (int64_t row0 = at.row; at.col < b && row0 < c; row0 += at.rows) {
    uint32_t w[RB], s[RB];
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (row >= c) break;
      w[u] = *reinterpret_cast<const uint32_t*>(codes + row * ldq + at.col / 2);
      s[u] = __bfloat16_as_ushort(scales[(int64_t)(at.col / group) * c + row]) & SCALE_BITS;
    }
#pragma unroll
    for (int u = 0; u < RB; ++u) {
      const int64_t row = row0 + u;
      if (row >= c) break;
      if constexpr (sizeof(T) == 2) {
        // codes j and j + 4 as a pair of bf16, 128 + nibble less 136; the product is exact
        const uint32_t off = 0x43084308u, two = s[u] | s[u] << 16;
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = nib(w[u], j);
          const __nv_bfloat162 d =
              __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                              *reinterpret_cast<const __nv_bfloat162*>(&off)),
                      *reinterpret_cast<const __nv_bfloat162*>(&two));
          h[j] = *reinterpret_cast<const uint32_t*>(&d);
        }
        *reinterpret_cast<uint4*>(W + row * ldw + at.col) =
            make_uint4(__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410),
                       __byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x7632));
      } else {
        const float scale = __uint_as_float(s[u] << 16);
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          x[k] = (__uint_as_float(((w[u] >> (4 * k)) & 15u) | 0x4B000000u) - 8388616.f) * scale;
        store8(W + row * ldw + at.col, x);
      }
    }
  }
  // whoever waits for this launch finds the one before it finished too
  if (blockIdx.x == 0 && blockIdx.y == 0) grid_dependency_wait();
}

// Vectors of a row beside one another (a power of two of at least a group's lanes), rows above.
void shape_of(int64_t rows, int64_t cols, dim3& grid, dim3& block) {
  const int64_t vecs = ceil_div(cols, 8);
  int x = 16;
  while (x < PT && x < vecs) x *= 2;
  block = dim3((unsigned)x, (unsigned)(PT / x), 1);
  const int64_t gy = ceil_div(rows, RB * (PT / x));
  grid = dim3((unsigned)ceil_div(vecs, x), (unsigned)(gy < 65535 ? gy : 65535), 1);
}

}  // namespace

thanos_status_t pack_weights(uint8_t* codes, int64_t ldq, bf16* scales, const void* W, int64_t ldw,
                             thanos_dtype_t dtype, int64_t c, int64_t b, int group,
                             cudaStream_t stream) {
  const int wide = (int)round_up((size_t)b, 64);
  dim3 grid, block;
  shape_of(c, wide, grid, block);
  auto run = [&](auto* kernel, auto* src) {
    kernel<<<grid, block, 0, stream>>>(codes, ldq, scales, src, ldw, c, (int)b, wide);
  };
  if (dtype == THANOS_BF16) {
    const bf16* src = static_cast<const bf16*>(W);
    if (group == 64) run(pack_w_kernel<bf16, 64>, src);
    else run(pack_w_kernel<bf16, 128>, src);
  } else {
    const float* src = static_cast<const float*>(W);
    if (group == 64) run(pack_w_kernel<float, 64>, src);
    else run(pack_w_kernel<float, 128>, src);
  }
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

thanos_status_t unpack_weights(void* W, int64_t ldw, thanos_dtype_t dtype, const PackedWeights& w,
                               int64_t c, int64_t b, cudaStream_t stream, bool beside) {
  cudaLaunchConfig_t cfg = {};
  shape_of(c, b, cfg.gridDim, cfg.blockDim);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = beside ? 1 : 0;
  count_launch();
  if (dtype == THANOS_BF16)
    THANOS_CUDA(cudaLaunchKernelEx(&cfg, unpack_w_kernel<bf16>, static_cast<bf16*>(W), ldw, w.codes,
                                   w.ldq, w.scales, c, (int)b, w.group));
  else
    THANOS_CUDA(cudaLaunchKernelEx(&cfg, unpack_w_kernel<float>, static_cast<float*>(W), ldw, w.codes,
                                   w.ldq, w.scales, c, (int)b, w.group));
  return THANOS_OK;
}

thanos_status_t pack_activations(int8_t* codes, int64_t ldc, uint8_t* exps, int64_t lde,
                                 const void* X, int64_t ldx, thanos_dtype_t dtype, int64_t T,
                                 int64_t b, cudaStream_t stream) {
  dim3 grid, block;
  shape_of(T, b, grid, block);
  if (dtype == THANOS_BF16)
    pack_act_kernel<bf16><<<grid, block, 0, stream>>>(codes, ldc, exps, lde,
                                                      static_cast<const bf16*>(X), ldx, T, (int)b);
  else
    pack_act_kernel<float><<<grid, block, 0, stream>>>(codes, ldc, exps, lde,
                                                       static_cast<const float*>(X), ldx, T, (int)b);
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

thanos_status_t unpack_activations(void* X, int64_t ldx, thanos_dtype_t dtype, const int8_t* codes,
                                   int64_t ldc, const uint8_t* exps, int64_t lde, int64_t T,
                                   int64_t b, cudaStream_t stream) {
  dim3 grid, block;
  shape_of(T, b, grid, block);
  if (dtype == THANOS_BF16)
    unpack_act_kernel<bf16><<<grid, block, 0, stream>>>(static_cast<bf16*>(X), ldx, codes, ldc, exps,
                                                        lde, T, (int)b);
  else
    unpack_act_kernel<float><<<grid, block, 0, stream>>>(static_cast<float*>(X), ldx, codes, ldc,
                                                         exps, lde, T, (int)b);
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

}  // namespace thanos
