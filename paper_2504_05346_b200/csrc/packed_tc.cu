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
// the tensor cores are a quarter busy.  64 tokens: 4096 x 4096 10.9 us, 11008 x 4096 20.6, 28672 x 8192
// 60 us.
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

// GROUPS of four warps that turn codes into weights, with two buffers each.
template <int GROUPS>
__global__ void __launch_bounds__(threads_of(GROUPS), GROUPS == 2 ? 2 : 1)
tiles_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
             const TilesParams p) {
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

  if (f.n == 0 && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *f.status = 0;
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
    if (f.n > 0) grid_dependency_wait();
    if (ok) {
      float* part = reinterpret_cast<float*>(smem);  // the ring, whose operands are consumed
      const int toks = min(N, f.T - t0);
#pragma unroll 1
      for (int j = 8 * group; j < toks; j += 8 * GROUPS) {
        uint32_t v[8];
        tmem_ld8(tmem_base + lanes + j, v);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (S > 1) part[(j + e) * QM + row] = __uint_as_float(v[e]);
          else if (j + e < toks && m0 + row < f.c)
            finish<bf16>(f, m0 + row, t0 + j + e, __uint_as_float(v[e]));
        }
      }
    }
  }
  if (S > 1) {
    cluster_sync_all();
    if (warp < PRODUCER && ok) {
      const int row = threadIdx.x & (QM - 1), toks = min(N, f.T - t0);
      for (int t = GROUPS * rank + (int)(threadIdx.x / QM); t < toks && m0 + row < f.c;
           t += GROUPS * S) {
        float v = 0.f;
        for (int u = 0; u < S; ++u) {
          float z;
          asm volatile("ld.shared::cluster.f32 %0, [%1];"
                       : "=f"(z)
                       : "r"(map_to_cta(smem_base, u) + 4u * (uint32_t)(t * QM + row))
                       : "memory");
          v += z;
        }
        finish<bf16>(f, m0 + row, t0 + t, v);
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

template <int GROUPS>
thanos_status_t launch_tiles(const CUtensorMap& map_w, const CUtensorMap& map_x, const TilesParams& p,
                             int tiles_t, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  THANOS_CUDA(ensure_max_dyn_smem(tiles_kernel<GROUPS>, 227 * 1024, done));
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
  cfg.numAttrs = p.f.n > 0 ? 2 : 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, tiles_kernel<GROUPS>, map_w, map_x, p));
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
  return groups == 2 ? launch_tiles<2>(map_w, map_x, p, tiles_t, stream)
                     : launch_tiles<4>(map_w, map_x, p, tiles_t, stream);
}

}  // namespace thanos
