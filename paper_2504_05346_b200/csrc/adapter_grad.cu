// dA_i = sum U[t]^T X[t] and dB_i = s_i sum dY[t]^T V[t] over the tokens of adapter i.
//
// A skinny contraction over tokens: 2 r flops per 16-bit value read, so reading X and dY once is the
// bound (r up to 128: at most 256 flops per 2 bytes, below the tensor cores' balance of about 500).
// A CTA owns one adapter and 128 features; tokens come in the order of sort_tokens, so a tile never
// mixes adapters (nothing that is not finite crosses from one to another) and needs no mask.
//   warps 0..3   gather 32 tokens per stage by cp.async, in the MN-major layouts of the tensor cores:
//                rows of Z (64 features x 32 tokens, 128-byte swizzle) and of R, which comes as three
//                bf16 planes side by side in n (all 24 bits: the products with Z are exact)
//   warp 4       tcgen05.mma issuer, 128 x 3 r x 16
//   warps 5..8   the sums: the tensor cores cut what they add to an accumulator, by up to 2^-23 each
//                time, so it is drained into registers, rounded to nearest, every 512 tokens; at the
//                end written (or added) to the gradient
// A cluster of up to eight CTAs splits the adapter's tokens when there are few tiles; the partial
// sums are added over distributed shared memory in rank order (same inputs, same bits).
//
// What bounds it: an SM takes in some 60 bytes per clock, and 16-byte copies that are gathered come near
// (two CTAs: 53, 777 of 1440 cycles of a stage in issuing them); the planes of R are 12 of a stage's 20
// KB at rank 64.  Tiles of 256 features, which share them among more, leave one CTA per SM and were
// slower.  2048 tokens, 4096 + 4096 features, 4 adapters of rank 16: 28 us (cold).
#include "adapter_grad.cuh"

#include "proj_gemm.cuh"
#include "tc_common.cuh"

namespace thanos {

namespace {

using namespace tc;

// ------------------------------------------------------------------------------------- sorting
constexpr int SORT_THREADS = 1024;

__global__ void __launch_bounds__(SORT_THREADS)
sort_kernel(const int32_t* __restrict__ index, int T, int n, int32_t* order, int32_t* spare,
            int32_t* __restrict__ off, int32_t* __restrict__ status) {
  __shared__ int base[256];
  __shared__ int wh[32][256];
  grid_dependents_launch();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto key_of = [&](int t) {
    const int i = index[t];
    return i >= 0 && i < n ? i : n;
  };
  int digits = 1;
  while (digits < 4 && (n >> (8 * digits)) != 0) ++digits;
  bool bad = false;  // an index that names no adapter
  int32_t* dst = (digits & 1) ? order : spare;
  int32_t* src = (digits & 1) ? spare : order;
  for (int d = 0; d < digits; ++d) {
    if (tid < 256) base[tid] = 0;
    __syncthreads();
    for (int p = tid; p < T; p += SORT_THREADS) {
      const int k = key_of(d == 0 ? p : src[p]);
      if (d == 0 && k == n && index[p] != -1) bad = true;
      atomicAdd(&base[(k >> (8 * d)) & 255], 1);
    }
    __syncthreads();
    if (warp == 0) {  // exclusive scan, eight bins a lane
      int v[8], sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = sum;
        sum += base[8 * lane + e];
      }
      int before = sum;
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += u;
      }
      before -= sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) base[8 * lane + e] = before + v[e];
    }
    __syncthreads();
    for (int p0 = 0; p0 < T; p0 += SORT_THREADS) {
      for (int e = tid; e < 32 * 256; e += SORT_THREADS) (&wh[0][0])[e] = 0;
      __syncthreads();
      const int p = p0 + tid;
      const int t = p < T ? (d == 0 ? p : src[p]) : 0;
      const int bin = p < T ? (key_of(t) >> (8 * d)) & 255 : -1;
      const unsigned same = __match_any_sync(0xffffffffu, bin);
      const int before = __popc(same & ((1u << lane) - 1u));
      if (bin >= 0 && before == 0) wh[warp][bin] = __popc(same);
      __syncthreads();
      if (tid < 256) {
        int run = base[tid];
#pragma unroll
        for (int w = 0; w < 32; ++w) {
          const int c = wh[w][tid];
          wh[w][tid] = run;
          run += c;
        }
        base[tid] = run;
      }
      __syncthreads();
      if (bin >= 0) dst[wh[warp][bin] + before] = t;
      __syncthreads();
    }
    int32_t* x = dst;
    dst = src;
    src = x;
  }
  // src == order now; first position of every adapter
  for (int p = tid; p <= T; p += SORT_THREADS) {
    const int k = p < T ? key_of(src[p]) : n;
    const int prev = p > 0 ? key_of(src[p - 1]) : -1;
    for (int i = prev + 1; i <= k; ++i) off[i] = p;
  }
  // whoever waits for this launch finds the one before it finished too
  grid_dependency_wait();
  if (bad) atomicCAS(status, 0, (int)THANOS_ERR_INVALID_ARG);
}

// ----------------------------------------------------------------------------------- gradients
constexpr int GF = 128;                  // features per CTA
constexpr int GK = 32;                   // tokens per stage
constexpr int BOX_BYTES = 64 * GK * 2;   // 64 features x GK tokens
constexpr int RBOX_BYTES = 32 * GK * 2;  // 32 columns of R x GK tokens
constexpr int GA_BYTES = 2 * BOX_BYTES;
constexpr int G_MAX_STAGES = 8;
constexpr int G_THREADS = 288;
constexpr int DRAIN_STAGES = 16;         // 512 tokens between two drains of the accumulator

struct GradParams {
  AdapterGradSide side[2];
  int tiles0, tiles;                     // feature tiles of side 0, of both
  const int32_t* order;
  const int32_t* off;
  int32_t* status;
  int n, r, r16, stages, splits, accumulate, ring_bytes, stage_bytes;
  int tmem_cols, buffers;                // accumulators: 2 where they fit half of tensor memory
};

__device__ __forceinline__ uint64_t grad_desc(uint32_t addr, uint32_t lbo, uint32_t sbo,
                                              uint32_t layout) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)layout << 61;
  return d;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
        "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
        "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float grad_ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// The stage whose copies were issued `behind` turns ago is complete for this thread.
__device__ __forceinline__ void publish(uint32_t bar, int lane) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

// RMAX: ranks whose sums a thread holds: 32, 64 (two CTAs per SM) or 128.
template <int RMAX>
__global__ void __launch_bounds__(G_THREADS, RMAX <= 64 ? 2 : 1) grad_tc_kernel(const GradParams p) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.ring_bytes);
  // full, empty (G_MAX_STAGES each), accumulator full (2), accumulator empty (2)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * G_MAX_STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 2 * G_MAX_STAGES + 5);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (G_MAX_STAGES + s); };
  auto tfull_bar = [&](int q) { return bar_base + 8u * (2 * G_MAX_STAGES + q); };
  auto tempty_bar = [&](int q) { return bar_base + 8u * (2 * G_MAX_STAGES + 2 + q); };

  const int S = p.splits;
  const int rank = S > 1 ? (int)cluster_ctarank() : 0;
  const int tile = (int)(blockIdx.x / S);
  const AdapterGradSide& sd = tile < p.tiles0 ? p.side[0] : p.side[1];
  const int f0 = (tile < p.tiles0 ? tile : tile - p.tiles0) * GF;
  const int F = sd.F, r = p.r, r16 = p.r16, N = 3 * r16;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 4);
      mbar_init(empty_bar(s), 1);
    }
    for (int q = 0; q < 2; ++q) {
      mbar_init(tfull_bar(q), 1);
      mbar_init(tempty_bar(q), 4);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(p.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int stage_bytes = p.stage_bytes;
  // the ring, the accumulators and their barriers run on from adapter to adapter
  int s = 0, s_pub = 0, q = 0;
  uint32_t phase = 0, tphase = 0;
  bool ok = true;

  grid_dependency_wait();
  for (int64_t i = blockIdx.y; i < p.n; i += gridDim.y) {
    const int lo = p.off[i], len = p.off[i + 1] - lo;
    if (len == 0) {
      // an adapter without tokens: zeros, or nothing to add
      if (!p.accumulate && rank == 0) {
        for (int e = threadIdx.x; e < GF * r; e += G_THREADS) {
          const int j = sd.by_feature ? e % r : e / GF, f = f0 + (sd.by_feature ? e / r : e % GF);
          if (f < F) sd.out[sd.by_feature ? (i * F + f) * r + j : (i * r + j) * F + f] = 0.f;
        }
      }
      continue;
    }
    const int nk = (len + GK - 1) / GK;
    const int ks0 = (int)((int64_t)nk * rank / S), ks1 = (int)((int64_t)nk * (rank + 1) / S);

    if (warp < 4) {
      // ---------------------------------------------------------- gather
      // eight lanes a row, so that a copy instruction of a warp covers four whole lines; a thread
      // takes rows r8 and r8 + 16 and, in them, every eighth 16-byte piece
      const int r8 = threadIdx.x >> 3, piece = threadIdx.x & 7;
      const int lag = p.stages > 4 ? 3 : p.stages - 1;
      int pending = 0;
      // the tokens of the next stage are looked up while this one's copies are issued
      int next[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = ks0 * GK + r8 + 16 * u;
        next[u] = at < len ? p.order[lo + at] : -1;
      }
      for (int ks = ks0; ks < ks1; ++ks) {
        int tok[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          tok[u] = next[u];
          const int at = (ks + 1) * GK + r8 + 16 * u;
          next[u] = at < len ? p.order[lo + at] : -1;
        }
        // lanes whose wait ran out go on, without waiting: the warp stays together with no vote, which
        // takes 3 %, and the stages that are overwritten belong to a call that reports the timeout
        if (ok) ok = mbar_wait(empty_bar(s), phase ^ 1u, abort_flag);
        const uint32_t st = smem_base + (uint32_t)s * stage_bytes;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int row = r8 + 16 * u;
          const int64_t t = tok[u] < 0 ? 0 : tok[u];
          const __nv_bfloat16* z = sd.Z + t * sd.ldz;
#pragma unroll
          for (int box = 0; box < 2; ++box) {
            const int f = f0 + 64 * box + 8 * piece;
            const int left = tok[u] < 0 ? 0 : (F - f) * 2;
            const uint32_t bytes = left <= 0 ? 0u : left < 16 ? (uint32_t)left : 16u;
            cp_async16(st + box * BOX_BYTES + row * 128 + ((piece ^ (row & 7)) << 4),
                       bytes ? z + f : sd.Z, bytes);
          }
          // R's row into boxes of 32 n: 64 bytes per k row, 64-byte swizzle
          const __nv_bfloat16* R = sd.R + t * N;
          for (int g8 = piece; g8 < N / 8; g8 += 8)
            cp_async16(st + GA_BYTES + (g8 >> 2) * RBOX_BYTES + row * 64 +
                           (((g8 & 3) ^ ((row >> 1) & 3)) << 4),
                       R + 8 * g8, tok[u] < 0 ? 0u : 16u);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++pending > lag) {
          if (lag == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
          else if (lag == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
          else asm volatile("cp.async.wait_group 1;" ::: "memory");
          publish(full_bar(s_pub), lane);
          if (++s_pub == p.stages) s_pub = 0;
          --pending;
        }
        if (++s == p.stages) {
          s = 0;
          phase ^= 1u;
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      while (pending-- > 0) {
        publish(full_bar(s_pub), lane);
        if (++s_pub == p.stages) s_pub = 0;
      }
    } else if (warp == 4) {
      // ---------------------------------------------------------- MMA issuer
      // an instruction has at most 256 columns
      const int n1 = min(N, 256), n2 = N - n1;
      uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16);
      idesc |= (uint32_t)(GF >> 4) << 24;
      const uint32_t id1 = idesc | (uint32_t)(n1 >> 3) << 17, id2 = idesc | (uint32_t)(n2 >> 3) << 17;
      if (elect_one()) {  // the same lane every time: it alone follows the ring
        for (int ks = ks0; ks < ks1 && ok; ++ks) {
          const bool start = (ks - ks0) % DRAIN_STAGES == 0;
          if (start) ok = mbar_wait(tempty_bar(q), tphase ^ 1u, abort_flag);
          ok = ok && mbar_wait(full_bar(s), phase, abort_flag);
          tc_fence_after();
          if (ok) {
            const uint32_t sa = smem_base + (uint32_t)s * stage_bytes, sb = sa + GA_BYTES;
            const uint32_t d = tmem_base + (uint32_t)(q * N);
#pragma unroll
            for (int k2 = 0; k2 < GK / 16; ++k2) {
              const uint64_t ad = grad_desc(sa + k2 * 2048, BOX_BYTES, 1024, 2);
              const uint32_t acc = start && k2 == 0 ? 0u : 1u;
              tc_mma_bf16(d, ad, grad_desc(sb + k2 * 1024, RBOX_BYTES, 512, 4), id1, acc);
              if (n2 > 0)
                tc_mma_bf16(d + 256, ad,
                            grad_desc(sb + 8 * RBOX_BYTES + k2 * 1024, RBOX_BYTES, 512, 4), id2, acc);
            }
            tc_commit(empty_bar(s));
          }
          if (++s == p.stages) {
            s = 0;
            phase ^= 1u;
          }
          if ((ks - ks0) % DRAIN_STAGES == DRAIN_STAGES - 1 || ks + 1 == ks1) {
            if (ok) tc_commit(tfull_bar(q));
            if (++q == p.buffers) {
              q = 0;
              tphase ^= 1u;
            }
          }
        }
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------- sums of this slice of tokens
      const int g = warp & 3;
      const uint32_t taddr = tmem_base + ((uint32_t)(32 * g) << 16);
      const int row = 32 * g + lane, f = f0 + row;
      float acc[RMAX / 16][16] = {};
      for (int ks = ks0; ks < ks1 && ok; ks += DRAIN_STAGES) {
        ok = mbar_wait_warp(tfull_bar(q), tphase, abort_flag);
        tc_fence_after();
        if (!ok) break;
#pragma unroll
        for (int j16 = 0; j16 < RMAX / 16; ++j16) {
          if (16 * j16 >= r16) break;
          const uint32_t at = taddr + (uint32_t)(q * N + 16 * j16);
          uint32_t h[16], m[16], l[16];
          tc_ld16(at, h);
          tc_ld16(at + r16, m);
          tc_ld16(at + 2 * r16, l);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e)
            acc[j16][e] += __uint_as_float(h[e]) + (__uint_as_float(m[e]) + __uint_as_float(l[e]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(q));
        if (++q == p.buffers) {
          q = 0;
          tphase ^= 1u;
        }
      }
      if (ok) {
        const float k = sd.scale ? sd.scale[i] : 1.f;
        float* part = reinterpret_cast<float*>(smem);  // the ring, whose operands are consumed
#pragma unroll
        for (int j16 = 0; j16 < RMAX / 16; ++j16) {
          if (16 * j16 >= r16) break;
          if (S > 1) {
#pragma unroll
            for (int e = 0; e < 16; ++e) part[(16 * j16 + e) * GF + row] = acc[j16][e];
          } else if (f < F) {
            float* o = sd.out + (sd.by_feature ? (i * F + f) * r + 16 * j16
                                               : (i * r + 16 * j16) * (int64_t)F + f);
            const int64_t step = sd.by_feature ? 1 : F;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if (16 * j16 + e >= r) break;
              o[e * step] = p.accumulate ? o[e * step] + k * acc[j16][e] : k * acc[j16][e];
            }
          }
        }
      }
    }
    __syncthreads();
    if (S > 1) {
      cluster_sync_all();
      const float k = sd.scale ? sd.scale[i] : 1.f;
      // ranks in turn to the CTAs, a feature a thread; the slices' sums are in flight together
#pragma unroll 1
      for (int e = threadIdx.x; e < (r - rank + S - 1) / S * GF; e += G_THREADS) {
        const int j = rank + S * (e / GF), row = e % GF, f = f0 + row;
        float part[8];
#pragma unroll
        for (int w = 0; w < 8; ++w)
          part[w] = w < S ? grad_ld_cluster(map_to_cta(smem_base, w) + (uint32_t)(j * GF + row) * 4u)
                          : 0.f;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += part[w];
        if (f < F) {
          float* o = sd.out + (sd.by_feature ? (i * F + f) * r + j : (i * r + j) * (int64_t)F + f);
          *o = p.accumulate ? *o + k * v : k * v;
        }
      }
      __syncwarp();
      cluster_sync_all();  // no CTA goes on while another may still read its partial sums
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                 "r"(p.tmem_cols)
                 : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(p.status, 0, (int)THANOS_ERR_TIMEOUT);
}

template <int RMAX>
thanos_status_t launch_grads(const GradParams& p, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  THANOS_CUDA(ensure_max_dyn_smem(grad_tc_kernel<RMAX>, 203 * 1024, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.tiles * p.splits), (unsigned)(p.n < 65535 ? p.n : 65535), 1);
  cfg.blockDim = dim3(G_THREADS, 1, 1);
  cfg.dynamicSmemBytes = (size_t)p.ring_bytes + 1024 + 256;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, grad_tc_kernel<RMAX>, p));
  return THANOS_OK;
}

}  // namespace

thanos_status_t sort_tokens(const int32_t* index, int64_t T, int64_t n, int32_t* order,
                            int32_t* spare, int32_t* off, int32_t* status, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1, 1, 1);
  cfg.blockDim = dim3(SORT_THREADS, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, sort_kernel, index, (int)T, (int)n, order, spare, off, status));
  return THANOS_OK;
}

thanos_status_t adapter_grads(const AdapterGradSide& a, const AdapterGradSide& b,
                              const int32_t* order, const int32_t* off, int64_t T, int64_t n, int r,
                              int accumulate, int32_t* status, cudaStream_t stream) {
  GradParams p = {};
  p.side[0] = a;
  p.side[1] = b;
  p.tiles0 = (int)ceil_div(a.F, GF);
  p.tiles = p.tiles0 + (int)ceil_div(b.F, GF);
  p.order = order;
  p.off = off;
  p.status = status;
  p.n = (int)n;
  p.r = r;
  p.r16 = (r + 15) / 16 * 16;
  p.accumulate = accumulate;
  const int N = 3 * p.r16;
  p.buffers = 2 * N <= 256 ? 2 : 1;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.buffers * N) p.tmem_cols *= 2;
  p.stage_bytes = GA_BYTES + (int)round_up((size_t)N, 32) * GK * 2;
  // Two CTAs share an SM, so that one gathers while the other finishes.  A CTA that needs all of
  // tensor memory has to have the SM to itself: two clusters, each with a CTA that waits for the
  // other's, would wait for ever.  Its ring is too large for two.
  const int ring = p.tmem_cols > 256 ? 200 * 1024 : 100 * 1024;
  p.stages = ring / p.stage_bytes;
  if (p.stages > G_MAX_STAGES) p.stages = G_MAX_STAGES;
  p.ring_bytes = p.tmem_cols > 256 ? ring : p.stages * p.stage_bytes;
  if (p.ring_bytes < p.r16 * GF * 4) p.ring_bytes = p.r16 * GF * 4;
  // Token slices, by the rounds that their CTAs take: two to an SM (one, where tensor memory says so)
  // and 2 % of an adapter's tokens for each CTA's start and sums, as long as a slice keeps some hundred
  // tokens.  Clusters of 5 and 7 are left out: they do not fill a cluster of SMs.  8192 tokens, 118
  // tiles, rank 64, the whole call without dX: 1 slice 232 us, 2 145, 3 183, 4 151, 5 175, 6 159, 8 165.
  const int64_t units = (int64_t)p.tiles * n, slots = (p.tmem_cols > 256 ? 1 : 2) * (int64_t)sm_count();
  p.splits = 1;
  double best = 0.0;
  for (const int k : {1, 2, 3, 4, 6, 8}) {
    if (k > 1 && T < n * k * 256) break;
    const double cost = (double)ceil_div(units * k, slots) * (1.0 / k + 0.02);
    if (k == 1 || cost < best) {
      best = cost;
      p.splits = k;
    }
  }
  return p.r16 <= 32   ? launch_grads<32>(p, stream)
         : p.r16 <= 64 ? launch_grads<64>(p, stream)
                       : launch_grads<128>(p, stream);
}

}  // namespace thanos
