// The adapted projection of a few hundred tokens on 4-bit weights, bf16 activations, on tcgen05:
//   D[m, t] = sum_k w^(m, k) x(t, k)      128 rows and up to 128 tokens a CTA
//
// The weights are the operand in tensor memory: what a lane of it holds is a row's k, so a thread turns
// the codes of its own row into bf16 (exactly: see packed.cu), with its own row's scale, and nothing is
// exchanged between threads.
//   last but one TMA: per stage 256 columns of the codes (128 rows x 128 bytes) and of the activations
//                (four boxes of 64 columns), both with the 128-byte swizzle
//   warps 0..7   codes -> bf16 -> tensor memory, 64 columns at a time into one of two buffers of the warp
//                group, which takes every other block; 0..15 and every fourth block where a CTA has the SM
//                to itself (these warps are what a block waits for)
//   next warp    tcgen05.mma, 128 x N x 16, A from tensor memory, B from shared memory
// A cluster splits k; the partial sums are added over distributed shared memory in rank order (same
// inputs, same bits).
//
// What bounds it is turning codes into bf16: 19 instructions for eight weights (shift, mask, subtract,
// multiply, and a permutation, because a word gives the columns j and j + 4 at once and an activation's
// columns come as they are), most of them at half rate; 128 x 64 weights take an SM some 480 clocks, and
// the tensor cores are a quarter busy.  The issue slots are 56 % used: with four warps to a scheduler, each
// waiting for its own last result, a pipe or a load in turn, there is not always one that can go on.  64
// tokens: 4096 x 4096 10.5 us, 11008 x 4096 17.6, 28672 x 8192 60 us.
#include <type_traits>

#include "packed_few.cuh"

namespace thanos {
namespace {

constexpr int QM = 128;                  // rows
constexpr int QBLOCK = 64;               // columns that are turned into bf16 at a time
constexpr int QSTAGE = 256;              // columns of a stage
constexpr int QCODES = QM * QSTAGE / 2;  // bytes of a stage's codes
constexpr int QMAX_BUFS = 8;             // buffers of weights in tensor memory, 32 columns each
constexpr int threads_of(int groups) { return 128 * groups + 64; }
constexpr int QMAX_STAGES = 6;
constexpr int OUT = 4;                   // results that a thread finishes at a time

struct TilesParams {
  FewParams f;
  int N, stages, split, blocks, ring_bytes, tmem_cols;
};

__device__ __forceinline__ uint64_t sw128_desc(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x,
                                            int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
// A from tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
      "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
      "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
      "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
      "r"(v[30]), "r"(v[31])
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
        "=r"(v[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(addr));
  return v;
}

// Eight weights of a word, in the order of their columns.
__device__ __forceinline__ void decode8(const Nibbles& nib, uint32_t w, uint32_t scale2,
                                        uint32_t* out) {
  const uint32_t off = 0x43084308u;  // 136
  uint32_t h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t v = nib(w, j);
    const __nv_bfloat162 d = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                                             *reinterpret_cast<const __nv_bfloat162*>(&off)),
                                     *reinterpret_cast<const __nv_bfloat162*>(&scale2));
    h[j] = *reinterpret_cast<const uint32_t*>(&d);
  }
  out[0] = __byte_perm(h[0], h[1], 0x5410);
  out[1] = __byte_perm(h[2], h[3], 0x5410);
  out[2] = __byte_perm(h[0], h[1], 0x7632);
  out[3] = __byte_perm(h[2], h[3], 0x7632);
}

// Sums over a cluster of a row's tokens first, first + step, ..., O at a time (with few to a thread the
// larger O is slower: 4096 x 4096, 32 tokens, two to a thread, 10.2 and 10.8 us; 11008 x 4096, 64 tokens,
// eleven to a thread, 20.7 and 18.6; with rows of adapters to wait for it pays from four on: 32 tokens, 16
// adapters, five to a thread, 24.3 and 22.3).
template <int O, bool ADAPTERS>
__device__ __forceinline__ void sum_and_finish(const FewParams& f, uint32_t smem_base, int first,
                                               int step, int toks, int t0, int m0, int row, int S) {
  if (m0 + row >= f.c) return;
#pragma unroll 1
  for (int t = first; t < toks; t += O * step) {
    float v[O] = {};
    int rows[O], at[O];
    uint32_t from[O];
#pragma unroll
    for (int o = 0; o < O; ++o) {
      const int mine = t + o * step, there = mine < toks ? mine : t;
      at[o] = t0 + there;
      rows[o] = mine < toks ? m0 + row : -1;
      from[o] = smem_base + 4u * (uint32_t)(there * QM + row);
    }
#pragma unroll 4
    for (int u = 0; u < S; ++u) {
      float z[O];
#pragma unroll
      for (int o = 0; o < O; ++o)
        asm volatile("ld.shared::cluster.f32 %0, [%1];"
                     : "=f"(z[o])
                     : "r"(map_to_cta(from[o], u))
                     : "memory");
#pragma unroll
      for (int o = 0; o < O; ++o) v[o] += z[o];
    }
    finish<bf16, O, ADAPTERS>(f, rows, at, v);
  }
}

// Eight fp32 values as pairs of bf16 in three planes (cut, not rounded: 24 bits in all).  The first plane
// keeps an infinity or NaN and the others are zero beside it.
__device__ __forceinline__ void planes_of(const float4& a, const float4& b, uint32_t (&o)[3][4]) {
  float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int pl = 0; pl < 3; ++pl) {
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool odd = pl == 0 && !isfinite(v[e]);
      h[e] = odd && isnan(v[e]) ? 0x7FFF0000u : __float_as_uint(v[e]) & 0xFFFF0000u;
      v[e] = odd ? 0.f : v[e] - __uint_as_float(h[e]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) o[pl][j] = __byte_perm(h[2 * j], h[2 * j + 1], 0x7632);
  }
}

// The adapter's part of one result as a sum of plain products.  In planes, an infinite weight would meet a
// zero that is only a plane of its factor.
__device__ __noinline__ float adapter_sum(const FewParams& f, int i, int t, int row) {
  const bf16* b = static_cast<const bf16*>(f.B) + ((int64_t)i * f.c + row) * f.r;
  const float* v = f.V + (int64_t)t * f.r;
  float d = 0.f;
#pragma unroll 1
  for (int j = 0; j < f.r; ++j) d = fmaf(v[j], to_float(b[j]), d);
  return d;
}

// The same for adapters of more ranks: a warp's 32 rows and its tokens, up to eight of one adapter at a
// time, as products on the tensor cores.  Which rank a lane holds at which place does not matter: a lane
// reads eight consecutive ones of each of its rows of B and of its token of V.  (A row of B to a lane, token
// by token, is 32 lines to a load of B and four passes to each of V: 128 tokens of 11008 x 4096 with four
// adapters of rank 64 took 133 us; here 50.)
__device__ __forceinline__ void finish_by_adapter(const FewParams& f, uint32_t smem_base, int first,
                                                  int step, int toks, int t0, int m0, int row,
                                                  int S) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3, r0 = row & ~31;
  // at most 32: 128 tokens and sixteen warps, or, where the rings of two CTAs fit, 64 and eight
  const int count = first < toks ? (toks - first + step - 1) / step : 0;
  int own = lane < count ? f.index[t0 + first + lane * step] : -1;
  if (own < -1 || own >= f.n) {
    if (m0 + r0 == 0) atomicCAS(f.status, 0, (int)THANOS_ERR_INVALID_ARG);
    own = -1;
  }
  unsigned left = __ballot_sync(0xffffffffu, lane < count);
  while (left) {
    // the next token's adapter, and up to eight of its tokens: the g-th is this lane's of the operand, the
    // 2 t4-th and the one after it are its results'
    const int i = __shfl_sync(0xffffffffu, own, __ffs(left) - 1);
    unsigned same = __ballot_sync(0xffffffffu, own == i) & left;
    int in = -1, out[2] = {-1, -1};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int k = __ffs(same) - 1;  // -1: no more
      if (e == g) in = k;
      if (e == 2 * t4) out[0] = k;
      if (e == 2 * t4 + 1) out[1] = k;
      if (k >= 0) left &= ~(1u << k);
      same &= same - 1;
    }
    float d[2][4] = {};
    if (i >= 0) {
      const float* vt = f.V + (int64_t)(t0 + first + (in < 0 ? 0 : in) * step) * f.r + 8 * t4;
      const bf16* bw[2][2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          bw[m][h] = static_cast<const bf16*>(f.B) +
                     ((int64_t)i * f.c + min(m0 + r0 + 16 * m + 8 * h + g, f.c - 1)) * f.r + 8 * t4;
#pragma unroll 2
      for (int j = 0; j < f.r; j += 32) {
        const bool there = j + 8 * t4 < f.r;
        uint4 w[2][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            w[m][h] = there ? *reinterpret_cast<const uint4*>(bw[m][h] + j) : make_uint4(0u, 0u, 0u, 0u);
        const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 va = there && in >= 0 ? *reinterpret_cast<const float4*>(vt + j) : none;
        const float4 vb = there && in >= 0 ? *reinterpret_cast<const float4*>(vt + j + 4) : none;
        uint32_t x[3][4];
        planes_of(va, vb, x);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const uint32_t lo[4] = {w[m][0].x, w[m][1].x, w[m][0].y, w[m][1].y};
          const uint32_t hi[4] = {w[m][0].z, w[m][1].z, w[m][0].w, w[m][1].w};
#pragma unroll
          for (int pl = 2; pl >= 0; --pl) {
            mma_16816(d[m], lo, x[pl][0], x[pl][1], false);
            mma_16816(d[m], hi, x[pl][2], x[pl][3], false);
          }
        }
      }
    }
    float zero = 0.f;  // or NaN
#pragma unroll
    for (int e = 0; e < 8; ++e) zero = fmaf(d[e >> 2][e & 3], 0.f, zero);
    if (zero != 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float& add = d[e >> 2][e & 3];
        const int at = m0 + r0 + 8 * (e >> 1) + g, k = out[e & 1];
        if (!isfinite(add) && k >= 0 && at < f.c) add = adapter_sum(f, i, t0 + first + k * step, at);
      }
    }
    const float scale = i >= 0 ? f.scale[i] : 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int t = first + (out[e] < 0 ? 0 : out[e]) * step;
      float v[4] = {};
#pragma unroll 2
      for (int u = 0; u < S; ++u) {
        float z[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          asm volatile("ld.shared::cluster.f32 %0, [%1];"
                       : "=f"(z[q])
                       : "r"(map_to_cta(smem_base + 4u * (uint32_t)(t * QM + r0 + 8 * q + g), u))
                       : "memory");
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += z[q];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = m0 + r0 + 8 * q + g;
        if (out[e] >= 0 && at < f.c)
          static_cast<bf16*>(f.Y)[(int64_t)(t0 + t) * f.ldy + at] =
              __float2bfloat16_rn(i >= 0 ? fmaf(scale, d[q >> 1][2 * (q & 1) + e], v[q]) : v[q]);
      }
    }
  }
}

// What is added to the products.
enum { NO_ADAPTERS, BY_TOKEN, BY_ADAPTER };

// GROUPS of four warps that turn codes into weights, with two buffers each.
template <int GROUPS, int ADD>
__global__ void __launch_bounds__(threads_of(GROUPS), GROUPS == 2 ? 2 : 1)
tiles_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
             const __grid_constant__ TilesParams p) {
  constexpr int QBUFS = 2 * GROUPS, PER = 4 / GROUPS;  // blocks of a stage that a group takes
  constexpr int PRODUCER = 4 * GROUPS, ISSUER = PRODUCER + 1;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.ring_bytes);
  // full, empty (QMAX_STAGES each), weights full, weights empty (QMAX_BUFS each), done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * QMAX_STAGES + 2 * QMAX_BUFS + 1);
  volatile int* abort_flag =
      reinterpret_cast<volatile int*>(bars + 2 * QMAX_STAGES + 2 * QMAX_BUFS + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (QMAX_STAGES + s); };
  auto wfull_bar = [&](int q) { return bar_base + 8u * (2 * QMAX_STAGES + q); };
  auto wempty_bar = [&](int q) { return bar_base + 8u * (2 * QMAX_STAGES + QMAX_BUFS + q); };
  const uint32_t done_bar = bar_base + 8u * (2 * QMAX_STAGES + 2 * QMAX_BUFS);

  const FewParams& f = p.f;
  const int S = p.split, rank = S > 1 ? (int)cluster_ctarank() : 0;
  const int m0 = (int)(blockIdx.x / S) * QM, t0 = blockIdx.y * p.N, N = p.N;
  const int stages_all = (p.blocks + 3) / 4;
  const int st0 = (int)((int64_t)stages_all * rank / S), st1 = (int)((int64_t)stages_all * (rank + 1) / S);
  const int nblk = min(4 * st1, p.blocks) - 4 * st0;  // of this CTA, at least one
  const int stage_bytes = QCODES + N * QSTAGE * 2;

  if (ADD == NO_ADAPTERS && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *f.status = 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 4 * GROUPS + 1);
    }
    for (int q = 0; q < QBUFS; ++q) {
      mbar_init(wfull_bar(q), 4);
      mbar_init(wempty_bar(q), 1);
    }
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(p.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot, weights = tmem_base + (uint32_t)(p.tmem_cols - QBUFS * 32);
  bool ok = true;

  if (warp == PRODUCER) {
    // ------------------------------------------------------------ TMA producer
    if (elect_one()) {
      int s = 0;
      uint32_t phase = 0;
      for (int st = st0; st < st1 && ok; ++st) {
        ok = mbar_wait(empty_bar(s), phase ^ 1u, abort_flag);
        if (ok) {
          const uint32_t dst = smem_base + (uint32_t)(s * stage_bytes);
          mbar_expect_tx(full_bar(s), stage_bytes);
          tma_load_2d(dst, &map_w, full_bar(s), st * (QSTAGE / 2), m0);
#pragma unroll
          for (int u = 0; u < QSTAGE / QBLOCK; ++u)
            tma_load_2d(dst + QCODES + u * N * 128, &map_x, full_bar(s), st * QSTAGE + u * QBLOCK, t0);
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
  } else if (warp == ISSUER) {
    // ------------------------------------------------------------ MMA issuer
    if (elect_one()) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t)(N >> 3) << 17 |
                             (uint32_t)(QM >> 4) << 24;
      int s = 0;
      uint32_t phase = 0;
      for (int i = 0; i < nblk && ok; ++i) {
        const int u = i & 3, q = i % QBUFS;
        if (u == 0) ok = mbar_wait(full_bar(s), phase, abort_flag);
        ok = ok && mbar_wait(wfull_bar(q), (uint32_t)(i / QBUFS) & 1u, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint64_t bd = sw128_desc(smem_base + (uint32_t)(s * stage_bytes) + QCODES + u * N * 128);
#pragma unroll
        for (int k4 = 0; k4 < QBLOCK / 16; ++k4)
          mma_ts(tmem_base, weights + q * 32 + k4 * 8, bd + (uint64_t)(k4 * 32 >> 4), idesc,
                 i > 0 || k4 > 0 ? 1u : 0u);
        tc_commit(wempty_bar(q));
        if (u == 3 || i + 1 == nblk) {
          tc_commit(empty_bar(s));
          if (++s == p.stages) {
            s = 0;
            phase ^= 1u;
          }
        }
      }
      if (ok) tc_commit(done_bar);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ codes into tensor memory
    const int group = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const unsigned short* scales =
        reinterpret_cast<const unsigned short*>(f.scales) + min(m0 + row, f.c - 1);
    auto scale_of = [&](int i) {  // of block i of this CTA, as it is in memory
      const int kb = min(4 * st0 + i, p.blocks - 1);
      return (uint32_t)scales[(int64_t)((kb * QBLOCK) >> f.shift) * f.c];
    };
    const Nibbles nib;
    int s = 0, q = group;         // stage; buffer of the next block: this group's two in turn
    uint32_t phase = 0, turn = 1; // parity of the buffer's barrier
    // a stage's scales are fetched a stage ahead, and not looked at until then
    uint32_t next[PER];
#pragma unroll
    for (int h = 0; h < PER; ++h) next[h] = scale_of(group + GROUPS * h);
    for (int i0 = 0; i0 < nblk; i0 += 4) {
      uint32_t raw[PER];
#pragma unroll
      for (int h = 0; h < PER; ++h) {
        raw[h] = next[h];
        next[h] = scale_of(i0 + 4 + group + GROUPS * h);
      }
      ok = mbar_wait_warp(full_bar(s), phase, abort_flag);
      if (!ok) break;
      const uint32_t codes = smem_base + (uint32_t)(s * stage_bytes) + row * 128;
      uint4 c[PER][2];
#pragma unroll
      for (int h = 0; h < PER; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          c[h][e] = ld_shared16(codes + (((2 * (group + GROUPS * h) + e) ^ (row & 7)) << 4));
#pragma unroll
      for (int h = 0; h < PER; ++h) {
        if (i0 + group + GROUPS * h < nblk) {
          const uint32_t scale = (raw[h] & SCALE_BITS) * 0x10001u;
          uint32_t v[32];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            decode8(nib, c[h][e].x, scale, v + 16 * e);
            decode8(nib, c[h][e].y, scale, v + 16 * e + 4);
            decode8(nib, c[h][e].z, scale, v + 16 * e + 8);
            decode8(nib, c[h][e].w, scale, v + 16 * e + 12);
          }
          ok = mbar_wait_warp(wempty_bar(q), turn, abort_flag);
          if (!ok) break;
          tc_fence_after();
          tmem_st32(weights + lanes + q * 32, v);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(wfull_bar(q));
          q ^= GROUPS;
          if (q == group) turn ^= 1u;  // both have been written once more
        }
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(s));
      if (++s == p.stages) {
        s = 0;
        phase ^= 1u;
      }
    }
    // ------------------------------------------------------------ sums
    ok = ok && mbar_wait_warp(done_bar, 0, abort_flag);
    tc_fence_after();
    if (ADD != NO_ADAPTERS) grid_dependency_wait();
    if (ok) {
      float* part = reinterpret_cast<float*>(smem);  // the ring, whose operands are consumed
      const int toks = min(N, f.T - t0);
#pragma unroll 1
      for (int j = 8 * group; j < toks; j += 8 * GROUPS) {
        uint32_t v[8];
        tmem_ld8(tmem_base + lanes + j, v);
        tc_wait_ld();
        if (S > 1 || ADD == BY_ADAPTER) {
#pragma unroll
          for (int e = 0; e < 8; ++e) part[(j + e) * QM + row] = __uint_as_float(v[e]);
        } else {
#pragma unroll
          for (int h = 0; h < 8; h += OUT) {
            float y[OUT];
            int rows[OUT], at[OUT];
#pragma unroll
            for (int e = 0; e < OUT; ++e) {
              y[e] = __uint_as_float(v[h + e]);
              at[e] = t0 + j + h + e;
              rows[e] = j + h + e < toks && m0 + row < f.c ? m0 + row : -1;
            }
            finish<bf16, OUT, ADD != NO_ADAPTERS>(f, rows, at, y);
          }
        }
      }
    }
  }
  if (S > 1 || ADD == BY_ADAPTER) {
    cluster_sync_all();
    if (warp < PRODUCER && ok) {
      const int row = threadIdx.x & (QM - 1), toks = min(N, f.T - t0);
      const int step = GROUPS * S, first = GROUPS * rank + (int)(threadIdx.x / QM);
      if constexpr (ADD == BY_ADAPTER) {
        finish_by_adapter(f, smem_base, first, step, toks, t0, m0, row, S);
      } else if constexpr (ADD == BY_TOKEN) {
        if (toks < OUT * step || f.r > 16)
          sum_and_finish<1, true>(f, smem_base, first, step, toks, t0, m0, row, S);
        else
          sum_and_finish<OUT, true>(f, smem_base, first, step, toks, t0, m0, row, S);
      } else {
        if (toks < 2 * OUT * step)
          sum_and_finish<1, false>(f, smem_base, first, step, toks, t0, m0, row, S);
        else
          sum_and_finish<OUT, false>(f, smem_base, first, step, toks, t0, m0, row, S);
      }
    }
    __syncwarp();
    cluster_sync_all();  // no CTA leaves while another reads its sums
  }
  tc_fence_before();
  __syncthreads();
  if (warp == ISSUER) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                 "r"(p.tmem_cols)
                 : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(f.status, 0, (int)THANOS_ERR_TIMEOUT);
}

bool make_map2(CUtensorMap* map, const void* base, CUtensorMapDataType type, int64_t inner,
               int64_t rows, int64_t pitch_bytes, int box_inner, int box_rows) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  cuuint64_t gdim[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
  cuuint64_t gstr[1] = {(cuuint64_t)pitch_bytes};
  cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return enc(map, type, 2, const_cast<void*>(base), gdim, gstr, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int GROUPS, int ADD>
thanos_status_t launch_tiles(const CUtensorMap& map_w, const CUtensorMap& map_x, const TilesParams& p,
                             int tiles_t, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  THANOS_CUDA(ensure_max_dyn_smem(tiles_kernel<GROUPS, ADD>, 227 * 1024, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ceil_div(p.f.c, QM) * p.split), (unsigned)tiles_t, 1);
  cfg.blockDim = dim3(threads_of(GROUPS), 1, 1);
  cfg.dynamicSmemBytes = (size_t)p.ring_bytes + 1024 + 512;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ADD != NO_ADAPTERS ? 2 : 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, tiles_kernel<GROUPS, ADD>, map_w, map_x, p));
  return THANOS_OK;
}

}  // namespace

thanos_status_t packed_tiles(const FewParams& f, cudaStream_t stream) {
  TilesParams p = {};
  p.f = f;
  const int tiles_t = (int)ceil_div(f.T, 128);
  p.N = (int)round_up((size_t)ceil_div(f.T, tiles_t), 16);
  p.blocks = (int)ceil_div(f.b, QBLOCK);
  const int stage_bytes = QCODES + p.N * QSTAGE * 2;
  CUtensorMap map_w, map_x;
  if (!make_map2(&map_w, f.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, (int64_t)p.blocks * 32, f.c, f.ldq,
                 QSTAGE / 2, QM) ||
      !make_map2(&map_x, f.X, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, f.b, f.T, f.ldx * 2, QBLOCK, p.N))
    return THANOS_ERR_CUDA;
  const int64_t units = ceil_div(f.c, QM) * tiles_t, stages_all = ceil_div(p.blocks, 4);
  const int64_t sms = sm_count();
  // Slices of k and CTAs to an SM, by the cost of a CTA's stages: 1 where it has the SM to itself (1.1 us;
  // sixteen warps are then some 5 % faster than eight, 20 % with adapters to add), 1.75 where two share it,
  // if two stages of each fit; 4 for start and end, 1 for the sum over a cluster, 1 more for clusters of
  // eight two to an SM, which are hard to place.  32 tokens, replayed, slices 1 / 2 / 3 / 4 / 6 / 8:
  //   4096 x 4096    22.5  15.4  12.9  10.3  12.5  11.3 us
  //   11008 x 4096   22.6  20.8  17.3  20.6  22.9  26.1
  //   28672 x 8192   58.0  64.6  64.5  65.4  78.5  83.1
  const bool fit = 2 * stage_bytes <= 108 * 1024;
  int groups = 2;
  double best = 0.0;
  p.split = 0;
  for (const int S : {1, 2, 3, 4, 6, 8}) {
    if (S > stages_all) break;
    const int64_t ctas = units * S;
    const bool alone = ctas <= sms || !fit;
    const double fixed = 4.0 + (S > 1 ? 1.0 : 0.0) + (S == 8 && !alone ? 1.0 : 0.0);
    const double cost = (double)ceil_div(ctas, alone ? sms : 2 * sms) *
                        ((alone ? 1.0 : 1.75) * (double)ceil_div(stages_all, S) + fixed);
    if (p.split == 0 || cost < best) {
      best = cost;
      p.split = S;
      groups = alone ? 4 : 2;
    }
  }
  const int room = (groups == 2 ? 108 : 216) * 1024;
  p.stages = room / stage_bytes;
  if (p.stages > QMAX_STAGES) p.stages = QMAX_STAGES;
  // all of tensor memory: the CTA has to have the SM to itself, and a ring that is too large for two
  p.ring_bytes = groups == 2 ? p.stages * stage_bytes : room;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.N + 2 * groups * 32) p.tmem_cols *= 2;
  // By adapter from 17 ranks on: 16 adapters, 4096 x 4096, 128 tokens, rank 32 22.4 us (by token 29.1), rank
  // 16 of 8 adapters 19.7 (20.3), but 32 tokens 15.8 (13.6), and 11008 x 4096, 16 of rank 16, 32.0 (22.1).
  int add = f.n == 0 ? NO_ADAPTERS : BY_TOKEN;
  if (f.n > 0 && f.r % 8 == 0 && f.r > 16 && p.N <= 32 * groups * p.split)
    add = BY_ADAPTER;
  auto launch = [&](auto add_) {
    constexpr int ADD = decltype(add_)::value;
    return groups == 2 ? launch_tiles<2, ADD>(map_w, map_x, p, tiles_t, stream)
                       : launch_tiles<4, ADD>(map_w, map_x, p, tiles_t, stream);
  };
  return add == NO_ADAPTERS ? launch(std::integral_constant<int, NO_ADAPTERS>{})
         : add == BY_TOKEN  ? launch(std::integral_constant<int, BY_TOKEN>{})
                            : launch(std::integral_constant<int, BY_ADAPTER>{});
}

}  // namespace thanos
