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
// Bound by memory: every value is read and written once.  A thread takes eight columns; the lanes of a
// group share its largest value by shuffles.
#include "packed.cuh"

namespace thanos {
namespace {

using bf16 = __nv_bfloat16;
constexpr int PT = 256;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
}
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

// The largest magnitude of `lanes` neighbouring lanes, as the bits of a float (they are ordered like the
// magnitudes, infinity and NaN above all).
__device__ __forceinline__ uint32_t group_top(const float (&x)[8], int lanes) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  for (int o = 1; o < lanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  return top;
}

// A thread's place: eight columns from `col`, rows from `row` in steps of `rows`.  blockDim.x vectors of
// a row, blockDim.y rows; all threads of a warp stay together.
struct Place {
  int64_t row, rows;
  int col;
  __device__ Place()
      : row((int64_t)blockIdx.y * blockDim.y + threadIdx.y), rows((int64_t)gridDim.y * blockDim.y),
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
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row = at.row + i * at.rows;
    float x[8] = {};
    if (in && row < n) load8(X + row * ldx + at.col, x);
    const uint32_t top = group_top(x, 4);
    if (!in || row >= n) continue;
    // 64 to 128 steps of 2^e; one power of two more where 127.5 and above would round to 128 (where
    // that is no float, the code stays at 127)
    int e = max((int)(top >> 23) - 133, -126);
    const float high = __uint_as_float(top) * __uint_as_float((uint32_t)(127 - e) << 23);
    if (rintf(high) > 127.f && e < 121) ++e;
    const bool odd = top >= 0x7F800000u;
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      int q;
      if (odd)  // infinities keep their sign, what is beside them reads back as NaN
        q = isinf(x[k]) ? (x[k] > 0.f ? 1 : -1) : 0;
      else
        q = max(-127, min(127, __float2int_rn(x[k] * inv)));
      w[k >> 2] |= (uint32_t)(q & 255) << (8 * (k & 3));
    }
    *reinterpret_cast<uint2*>(codes + row * ldc + at.col) = make_uint2(w[0], w[1]);
    if (at.col % ACT_GROUP == 0)
      exps[row * lde + at.col / ACT_GROUP] = odd ? 255 : top == 0 ? 0 : (uint8_t)(e + 127);
  }
}

template <typename T>
__global__ void __launch_bounds__(PT) unpack_act_kernel(T* __restrict__ X, int64_t ldx,
                                                        const int8_t* __restrict__ codes, int64_t ldc,
                                                        const uint8_t* __restrict__ exps, int64_t lde,
                                                        int64_t n, int b) {
  const Place at;
  if (at.col >= b) return;
  for (int64_t row = at.row; row < n; row += at.rows) {
    const uint2 w = *reinterpret_cast<const uint2*>(codes + row * ldc + at.col);
    const float step = __uint_as_float((uint32_t)exps[row * lde + at.col / ACT_GROUP] << 23);
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      x[k] = (float)(int8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3))) * step;
    store8(X + row * ldx + at.col, x);
  }
}

template <typename T>
__global__ void __launch_bounds__(PT) pack_w_kernel(uint8_t* __restrict__ codes, int64_t ldq,
                                                    bf16* __restrict__ scales,
                                                    const T* __restrict__ W, int64_t ldw, int64_t c,
                                                    int b, int wide, int group) {
  const Place at;
  const bool in = at.col < b;
  const int64_t turns = (c + at.rows - 1) / at.rows;
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row = at.row + i * at.rows;
    float x[8] = {};
    if (in && row < c) load8(W + row * ldw + at.col, x);
    const uint32_t top = group_top(x, group / 8);
    if (at.col >= wide || row >= c) continue;
    // five significant bits, ties to even; below the normal numbers: zero
    const uint32_t bits = __float_as_uint(__fdiv_rn(__uint_as_float(top), 7.f));
    uint32_t s = (bits + 0x3FFFFu + ((bits >> 19) & 1u)) & 0xFFF80000u;
    if (s < 0x00800000u) s = 0u;
    const bool odd = top >= 0x7F800000u;
    if (odd) s = 0x7FC00000u;  // a group that is not finite reads back as NaN
    const float scale = __uint_as_float(s);
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      int q = 0;
      if (s != 0u && !odd) q = max(-7, min(7, __float2int_rn(__fdiv_rn(x[k], scale))));
      w |= (uint32_t)(q + 8) << (4 * k);
    }
    *reinterpret_cast<uint32_t*>(codes + row * ldq + at.col / 2) = w;
    if (in && at.col % group == 0)
      scales[(int64_t)(at.col / group) * c + row] = __ushort_as_bfloat16((unsigned short)(s >> 16));
  }
}

template <typename T>
__global__ void __launch_bounds__(PT) unpack_w_kernel(T* __restrict__ W, int64_t ldw,
                                                      const uint8_t* __restrict__ codes, int64_t ldq,
                                                      const bf16* __restrict__ scales, int64_t c,
                                                      int b, int group) {
  const Place at;
  if (at.col >= b) return;
  for (int64_t row = at.row; row < c; row += at.rows) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * ldq + at.col / 2);
    const uint32_t s = __bfloat16_as_ushort(scales[(int64_t)(at.col / group) * c + row]) & SCALE_BITS;
    const float scale = __uint_as_float(s << 16);
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (float)((int)((w >> (4 * k)) & 15u) - 8) * scale;
    store8(W + row * ldw + at.col, x);
  }
}

// Vectors of a row beside one another (a power of two of at least a group's lanes), rows above, and as
// many CTAs as fill the device twice over.
void shape_of(int64_t rows, int64_t cols, dim3& grid, dim3& block) {
  const int64_t vecs = ceil_div(cols, 8);
  int x = 16;
  while (x < PT && x < vecs) x *= 2;
  block = dim3((unsigned)x, (unsigned)(PT / x), 1);
  const int64_t gx = ceil_div(vecs, x), want = ceil_div(rows, PT / x);
  int64_t gy = ceil_div(NUM_SMS * 16, gx);
  if (gy > want) gy = want;
  if (gy > 65535) gy = 65535;
  grid = dim3((unsigned)gx, (unsigned)gy, 1);
}

}  // namespace

thanos_status_t pack_weights(uint8_t* codes, int64_t ldq, bf16* scales, const void* W, int64_t ldw,
                             thanos_dtype_t dtype, int64_t c, int64_t b, int group,
                             cudaStream_t stream) {
  const int wide = (int)round_up((size_t)b, 64);
  dim3 grid, block;
  shape_of(c, wide, grid, block);
  if (dtype == THANOS_BF16)
    pack_w_kernel<bf16><<<grid, block, 0, stream>>>(codes, ldq, scales, static_cast<const bf16*>(W),
                                                    ldw, c, (int)b, wide, group);
  else
    pack_w_kernel<float><<<grid, block, 0, stream>>>(codes, ldq, scales, static_cast<const float*>(W),
                                                     ldw, c, (int)b, wide, group);
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

thanos_status_t unpack_weights(void* W, int64_t ldw, thanos_dtype_t dtype, const PackedWeights& w,
                               int64_t c, int64_t b, cudaStream_t stream) {
  dim3 grid, block;
  shape_of(c, b, grid, block);
  if (dtype == THANOS_BF16)
    unpack_w_kernel<bf16><<<grid, block, 0, stream>>>(static_cast<bf16*>(W), ldw, w.codes, w.ldq,
                                                      w.scales, c, (int)b, w.group);
  else
    unpack_w_kernel<float><<<grid, block, 0, stream>>>(static_cast<float*>(W), ldw, w.codes, w.ldq,
                                                       w.scales, c, (int)b, w.group);
  THANOS_CHECK_LAUNCH();
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
