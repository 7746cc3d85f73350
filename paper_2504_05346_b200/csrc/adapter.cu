// The projection with low-rank adapters, forward and backward:
//   V[t] = X[t] A_i^T,  Y[t] = X[t] W^T + s_i V[t] B_i^T
//   U[t] = s_i dY[t] B_i,  dX[t] = dY[t] W + U[t] A_i,  dA_i = sum_t U[t]^T X[t],
//   dB_i = s_i sum_t dY[t]^T V[t]
#include "adapter_grad.cuh"
#include "packed.cuh"
#include "proj_gemm.cuh"
#include "recovery.cuh"
#include "tc_common.cuh"

namespace thanos {
namespace {

// The token's adapter, or -1 for none and for values that name no adapter.
__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ index, int64_t t, int n) {
  const int i = n > 0 ? index[t] : -1;
  return i >= 0 && i < n ? i : -1;
}

// ---------------------------------------------------------------------------- 16-bit operands
using bf16 = __nv_bfloat16;

// What the tensor-core kernels need besides a call's operands.  Launched once in front of them (what
// the skinny product reads) and once beside the skinny product (what only later launches read);
// blocks by number:
//   [0, n_list)          the distinct adapters of a token tile, by first occurrence
//   next n_copy          16-byte aligned copies: rows of dY, or the adapters' B with padded ranks
//   next n_turn          B_i [c, r] -> [r, c] (the skinny product's operand in the backward pass)
//   next n_planes        backward: V as three bf16 planes for dB, and the zeros beyond the rank of U's
//   the rest             V of a few tokens, a CTA per token and four ranks
struct FrontParams {
  int32_t* status;             // cleared here, or null
  int beside;                  // runs beside the launch before it, on whose results it does not depend
  const int32_t* index;
  int32_t* count;
  int32_t* list;
  int T, nt, n, n_list;
  const bf16* copy_src;
  bf16* copy_dst;
  int64_t copy_rows, copy_ls, copy_ld;
  int copy_cols, n_copy;
  const bf16* turn_src;
  bf16* turn_dst;
  int64_t turn_ld;
  int c, r, n_turn;
  const float* Vin;
  bf16* v_planes;
  bf16* u_planes;
  int n_planes;
  const bf16* X;
  int64_t ldx;
  const bf16* A;
  float* V;
  int b;
};

constexpr int SHRINK_RANKS = 4;   // ranks of a token that one CTA computes

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), s);
    s = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(y[e] & 0xFFFF0000u), s);
  }
  return s;
}

__device__ __forceinline__ void front_block(const FrontParams& p, float* sh) {
  const int tid = threadIdx.x;
  int blk = blockIdx.x;
  if (blk < p.n_list) {
    int* ids = reinterpret_cast<int*>(sh);
    int* base = ids + 256;
    const int t = blk * p.nt + tid;
    const int i = tid < p.nt && t < p.T ? adapter_of(p.index, t, p.n) : -1;
    ids[tid] = i;
    __syncthreads();
    bool first = i >= 0;
    for (int u = 0; u < p.nt; ++u)
      if (u < tid && ids[u] == i) first = false;
    const unsigned vote = __ballot_sync(0xffffffffu, first);
    if ((tid & 31) == 0) base[tid >> 5] = __popc(vote);
    __syncthreads();
    int at = __popc(vote & ((1u << (tid & 31)) - 1u)), all = 0;
    for (int w = 0; w < 8; ++w) {
      if (w < (tid >> 5)) at += base[w];
      all += base[w];
    }
    if (first) p.list[(int64_t)blk * p.nt + at] = i;
    if (tid == 0) p.count[blk] = all;
    return;
  }
  blk -= p.n_list;
  if (blk < p.n_copy) {
    const int64_t total = p.copy_rows * p.copy_cols;
    for (int64_t e = (int64_t)blk * 256 + tid; e < total; e += (int64_t)p.n_copy * 256) {
      const int64_t row = e / p.copy_cols;
      p.copy_dst[row * p.copy_ld + (e - row * p.copy_cols)] =
          p.copy_src[row * p.copy_ls + (e - row * p.copy_cols)];
    }
    return;
  }
  blk -= p.n_copy;
  if (blk < p.n_turn) {
    // 64 rows of one B_i at a time through shared memory
    const int tiles = (p.c + 63) / 64;
    const int64_t units = (int64_t)p.n * tiles;
    for (int64_t u = blk; u < units; u += p.n_turn) {
      const int64_t i = u / tiles;
      const int c0 = (int)(u - i * tiles) * 64;
      for (int j0 = 0; j0 < p.r; j0 += 64) {
        const int nj = min(64, p.r - j0);
        __syncthreads();
        for (int e = tid; e < 64 * nj; e += 256) {
          const int row = e / nj, j = e - row * nj;
          if (c0 + row < p.c)
            sh[j * 65 + row] = to_float(p.turn_src[(i * p.c + c0 + row) * p.r + j0 + j]);
        }
        __syncthreads();
        for (int e = tid; e < 64 * nj; e += 256) {
          const int j = e >> 6, row = e & 63;
          if (c0 + row < p.c)
            p.turn_dst[(i * p.r + j0 + j) * p.turn_ld + c0 + row] =
                __float2bfloat16_rn(sh[j * 65 + row]);
        }
      }
    }
    return;
  }
  blk -= p.n_turn;
  if (blk < p.n_planes) {
    const int r16 = (p.r + 15) & ~15, lane = tid & 31;
    for (int64_t t = (int64_t)blk * 8 + (tid >> 5); t < p.T; t += 8ll * p.n_planes) {
      for (int j = lane; j < r16; j += 32) {
        bf16* v = p.v_planes + t * 3 * r16 + j;
        split3(j < p.r ? p.Vin[t * p.r + j] : 0.f, v[0], v[r16], v[2 * r16]);
        if (j >= p.r) {
          bf16* u = p.u_planes + t * 3 * r16 + j;
          u[0] = u[r16] = u[2 * r16] = __float2bfloat16_rn(0.f);
        }
      }
    }
    return;
  }
  blk -= p.n_planes;
  // V[t, j0 .. j0 + 3]: the warps take k in turns of 256, eight elements a lane
  const int groups = (p.r + SHRINK_RANKS - 1) / SHRINK_RANKS;
  const int t = blk / groups, j0 = (blk - t * groups) * SHRINK_RANKS;
  const int i = adapter_of(p.index, t, p.n);
  float s[SHRINK_RANKS] = {};
  if (i >= 0) {
    const bf16* x = p.X + (int64_t)t * p.ldx;
    const bf16* a = p.A + ((int64_t)i * p.r + j0) * p.b;
#pragma unroll 2
    for (int k = tid * 8; k < p.b; k += 2048) {
      const uint4 xv = *reinterpret_cast<const uint4*>(x + k);
#pragma unroll
      for (int j = 0; j < SHRINK_RANKS; ++j)
        if (j0 + j < p.r)
          s[j] = dot8(xv, *reinterpret_cast<const uint4*>(a + (int64_t)j * p.b + k), s[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < SHRINK_RANKS; ++j) {
    for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    if ((tid & 31) == 0) sh[j * 8 + (tid >> 5)] = s[j];
  }
  __syncthreads();
  if (tid < SHRINK_RANKS && j0 + tid < p.r) {
    float v = 0.f;
    for (int w = 0; w < 8; ++w) v += sh[tid * 8 + w];
    p.V[(int64_t)t * p.r + j0 + tid] = v;
  }
}

__global__ void __launch_bounds__(256) front_kernel(const FrontParams p) {
  __shared__ float sh[64 * 65];
  grid_dependents_launch();
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) *p.status = 0;
  front_block(p, sh);
  // whoever waits for this launch finds the one before it finished too
  if (p.beside && blockIdx.x == 0) grid_dependency_wait();
}

thanos_status_t launch_front(const FrontParams& p, int64_t shrink_blocks, cudaStream_t stream) {
  const int64_t blocks = (int64_t)p.n_list + p.n_copy + p.n_turn + p.n_planes + shrink_blocks;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(256, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  if (p.beside) {
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, front_kernel, p));
  return THANOS_OK;
}

// A handful of tokens: V on the way, in the CTAs that need it.  Every one of them reads the tokens'
// A_i, so these may be no more than a fraction of the weights that a CTA reads (1 token, 4096 x 4096,
// r = 16: 128 KB beside 256 KB; a call takes 20.0 us instead of 23.5 with a launch for V).
bool handful(const AdapterArgs& a) { return a.T <= 8 && a.T * a.r * a.b <= (1 << 17); }

// Few tokens: V by dot products in the first launch; more: one more launch on the tensor cores (4096 x
// 4096, 16 adapters of rank 16: 64 tokens 17.0 and 22.6 us, 256 tokens 34.8 and 29.4; 2 of rank 64: 32
// tokens 20.6 and 24.7, 64 tokens 31.1 and 28.8, 128 tokens 43.4 and 33.9).
bool few_tokens(const AdapterArgs& a) { return a.T <= 64; }

struct Layout {
  int32_t* status;
  float* R;          // V or U
  int32_t* count;
  int32_t* list;
  bf16* copy;        // padded B (forward) or dY (backward)
  bf16* turned;      // backward: B_i transposed
  bf16* v_planes;    // backward: V and U as three bf16 planes
  bf16* u_planes;
  int32_t* order;    // backward: tokens by adapter
  int32_t* spare;
  int32_t* off;
};

bool carve(Arena& ar, Layout& L, bool backward, int64_t T, int64_t c, int64_t b, int64_t n, int r,
           bool copy_dy) {
  const int64_t nt = proj_pair_tile(T, backward ? b : c), tiles = nt ? ceil_div(T, nt) : 0;
  L = Layout{};
  L.status = ar.take<int32_t>(64);
  L.R = ar.take<float>((size_t)T * r);
  if (nt) {
    L.count = ar.take<int32_t>((size_t)tiles);
    L.list = ar.take<int32_t>((size_t)(tiles * nt));
  }
  if (!backward && nt && r % 8) L.copy = ar.take<bf16>((size_t)n * c * round_up(r, 8));
  if (backward && copy_dy) L.copy = ar.take<bf16>((size_t)T * round_up(c, 8));
  if (backward) {
    L.turned = ar.take<bf16>((size_t)n * r * round_up(c, 8));
    L.v_planes = ar.take<bf16>((size_t)T * 3 * round_up(r, 16));
    L.u_planes = ar.take<bf16>((size_t)T * 3 * round_up(r, 16));
    L.order = ar.take<int32_t>((size_t)T);
    L.spare = ar.take<int32_t>((size_t)T);
    L.off = ar.take<int32_t>((size_t)n + 1);
  }
  return ar.ok();
}

thanos_status_t forward16(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                          cudaStream_t stream) {
  Arena ar(workspace, ws_bytes);
  Layout L;
  if (!carve(ar, L, false, a.T, a.c, a.b, a.n, a.r, false)) return THANOS_ERR_WORKSPACE;
  float* V = a.V ? a.V : L.R;
  ProjArgs g;
  g.M = (int)a.c;
  g.N = (int)a.T;
  g.K = (int)a.b;
  g.A = a.W;
  g.lda = a.ldw;
  g.B = a.in;
  g.ldb = a.ldi;
  g.status = L.status;
  g.out = a.out;
  g.ldo = a.ldo;
  const int nt = proj_pair_tile(a.T, a.c);
  if (a.packed) g.A = a.unpacked;
  if (a.n == 0) {
    THANOS_CUDA(cudaMemsetAsync(L.status, 0, 16, stream));
    if (a.packed)
      THANOS_TRY(unpack_weights(a.unpacked, a.ldw, a.dtype, *a.packed, a.c, a.b, stream));
    return proj_gemm(g, stream);
  }
  FrontParams f = {};
  f.status = L.status;
  f.index = a.index;
  f.count = L.count;
  f.list = L.list;
  f.T = (int)a.T;
  f.nt = nt;
  f.n = (int)a.n;
  f.n_list = nt ? (int)ceil_div(a.T, nt) : 0;
  f.r = a.r;
  const bool pad = nt && a.r % 8;
  if (pad) {
    f.copy_src = static_cast<const bf16*>(a.B);
    f.copy_dst = L.copy;
    f.copy_rows = a.n * a.c;
    f.copy_cols = a.r;
    f.copy_ls = a.r;
    f.copy_ld = (int64_t)round_up(a.r, 8);
    const int64_t want = ceil_div(f.copy_rows * a.r, 1024);
    f.n_copy = (int)(want < 4 * NUM_SMS ? want : 4 * NUM_SMS);
  }
  g.V = V;
  g.index = a.index;
  g.n_adapters = (int)a.n;
  g.r = a.r;
  g.tile_count = L.count;
  g.tile_list = L.list;
  if (handful(a)) {
    g.V = a.V;
    g.skinny = a.A;
    g.first = 1;
  } else if (few_tokens(a)) {
    f.X = static_cast<const bf16*>(a.in);
    f.ldx = a.ldi;
    f.A = static_cast<const bf16*>(a.A);
    f.V = V;
    f.b = (int)a.b;
    THANOS_TRY(launch_front(f, a.T * ceil_div(a.r, SHRINK_RANKS), stream));
  } else {
    ProjArgs s = g;
    s.epi = PROJ_SHRINK;
    s.first = 1;
    s.A = a.A;
    s.lda = a.b;
    s.M = (int)(a.n * a.r);
    THANOS_TRY(proj_gemm(s, stream));
    f.status = nullptr;
    f.beside = 1;
    if (f.n_list + f.n_copy > 0) THANOS_TRY(launch_front(f, 0, stream));
  }
  if (a.packed)
    THANOS_TRY(unpack_weights(a.unpacked, a.ldw, a.dtype, *a.packed, a.c, a.b, stream, true));
  g.scale = a.scale;
  g.P = pad ? static_cast<const void*>(L.copy) : a.B;
  g.ldp = pad ? (int64_t)round_up(a.r, 8) : a.r;
  g.p_adapter = a.c * g.ldp;
  g.early = !handful(a) && !a.packed;
  return proj_gemm(g, stream);
}

thanos_status_t backward16(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                           cudaStream_t stream) {
  const bool copy_dy = a.ldi % 8 != 0;
  Arena ar(workspace, ws_bytes);
  Layout L;
  if (!carve(ar, L, true, a.T, a.c, a.b, a.n, a.r, copy_dy)) return THANOS_ERR_WORKSPACE;
  const int64_t c8 = (int64_t)round_up(a.c, 8);
  const void* dY = copy_dy ? static_cast<const void*>(L.copy) : a.in;
  const int64_t lddy = copy_dy ? c8 : a.ldi;
  ProjArgs g;
  g.M = (int)a.b;
  g.N = (int)a.T;
  g.K = (int)a.c;
  g.A = a.W;
  g.lda = a.ldw;
  if (a.packed) g.A = a.unpacked;
  g.a_mn = 1;
  g.B = dY;
  g.ldb = lddy;
  g.status = L.status;
  g.out = a.out;
  g.ldo = a.ldo;
  const int nt = proj_pair_tile(a.T, a.b);
  FrontParams f = {};
  f.status = L.status;
  f.index = a.index;
  f.count = L.count;
  f.list = L.list;
  f.T = (int)a.T;
  f.nt = nt;
  f.n = (int)a.n;
  f.n_list = a.n > 0 && nt ? (int)ceil_div(a.T, nt) : 0;
  f.r = a.r;
  f.c = (int)a.c;
  if (copy_dy) {
    f.copy_src = static_cast<const bf16*>(a.in);
    f.copy_dst = L.copy;
    f.copy_rows = a.T;
    f.copy_cols = (int)a.c;
    f.copy_ls = a.ldi;
    f.copy_ld = c8;
    const int64_t want = ceil_div(a.T * a.c, 1024);
    f.n_copy = (int)(want < 4 * NUM_SMS ? want : 4 * NUM_SMS);
  }
  if (a.n > 0) {
    f.turn_src = static_cast<const bf16*>(a.B);
    f.turn_dst = L.turned;
    f.turn_ld = c8;
    const int64_t want = a.n * ceil_div(a.c, 64);
    f.n_turn = (int)(want < 4 * NUM_SMS ? want : 4 * NUM_SMS);
  }
  const bool sorts = a.dA != nullptr;
  if (sorts) {
    f.Vin = a.Vin;
    f.v_planes = L.v_planes;
    f.u_planes = L.u_planes;
    const int64_t want = ceil_div(a.T, 8);
    f.n_planes = (int)(want < 2 * NUM_SMS ? want : 2 * NUM_SMS);
  }
  // in front: the copy of dY and the turned B; the rest beside the skinny product
  FrontParams later = f;
  later.status = nullptr;
  later.beside = 1;
  later.n_copy = later.n_turn = 0;
  f.n_list = f.n_planes = 0;
  if (f.n_copy + f.n_turn > 0) THANOS_TRY(launch_front(f, 0, stream));
  else THANOS_CUDA(cudaMemsetAsync(L.status, 0, 16, stream));
  if (a.n > 0) {
    g.V = L.R;
    g.index = a.index;
    g.n_adapters = (int)a.n;
    g.r = a.r;
    g.tile_count = L.count;
    g.tile_list = L.list;
    ProjArgs s = g;
    s.epi = PROJ_SHRINK;
    s.a_mn = 0;
    s.A = L.turned;
    s.lda = c8;
    s.M = (int)(a.n * a.r);
    s.scale = a.scale;
    s.planes = sorts ? L.u_planes : nullptr;
    THANOS_TRY(proj_gemm(s, stream));
    if (later.n_list + later.n_planes > 0) THANOS_TRY(launch_front(later, 0, stream));
    if (sorts)
      THANOS_TRY(sort_tokens(a.index, a.T, a.n, L.order, L.spare, L.off, L.status, stream));
    g.P = a.A;
    g.ldp = a.b;
    g.p_adapter = (int64_t)a.r * a.b;
    g.early = copy_dy || a.packed ? 0 : 1;
  }
  if (a.out && a.packed)
    THANOS_TRY(unpack_weights(a.unpacked, a.ldw, a.dtype, *a.packed, a.c, a.b, stream, a.n > 0));
  if (a.out) THANOS_TRY(proj_gemm(g, stream));
  if (a.dA) {
    AdapterGradSide sa, sb;
    sa.Z = static_cast<const bf16*>(a.X);
    sa.ldz = a.X8 ? a.ldx8 : a.ldx;
    sa.Z8 = a.X8;
    sa.exps = a.exps;
    sa.lde = a.lde;
    sa.R = L.u_planes;
    sa.out = a.dA;
    sa.F = (int)a.b;
    sb.Z = static_cast<const bf16*>(dY);
    sb.ldz = lddy;
    sb.R = L.v_planes;
    sb.scale = a.scale;
    sb.out = a.dB;
    sb.F = (int)a.c;
    sb.by_feature = 1;
    THANOS_TRY(adapter_grads(sa, sb, L.order, L.off, a.T, a.n, a.r, a.accumulate, L.status, stream));
  }
  return THANOS_OK;
}

}  // namespace

size_t adapter_workspace_bytes(bool backward, int64_t T, int64_t c, int64_t b, int64_t n, int r,
                               thanos_dtype_t dtype, bool packed) {
  if (dtype == THANOS_F32) return adapter_f32_workspace_bytes(backward, T, c, b, n, r, packed);
  size_t need = 256 + round_up((size_t)T * (size_t)r * 4, 256);
  const int64_t nt = proj_pair_tile(T, backward ? b : c), tiles = nt ? ceil_div(T, nt) : 0;
  need += round_up((size_t)tiles * 4, 256) + round_up((size_t)(tiles * nt) * 4, 256);
  const size_t c8 = round_up((size_t)c, 8);
  if (!backward && nt && r % 8) need += round_up((size_t)n * c * round_up(r, 8) * 2, 256);
  // room for a copy of dY whose rows are not 16-byte aligned
  if (backward)
    need += round_up((size_t)T * c8 * 2, 256) + round_up((size_t)n * r * c8 * 2, 256) +
            2 * round_up((size_t)T * 3 * round_up(r, 16) * 2, 256) + 2 * round_up((size_t)T * 4, 256) +
            round_up(((size_t)n + 1) * 4, 256);
  return need;
}

thanos_status_t adapter_forward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                     cudaStream_t stream) {
  if (a.dtype == THANOS_BF16) return forward16(a, workspace, ws_bytes, stream);
  return adapter_f32(false, a, workspace, ws_bytes, stream);
}

thanos_status_t adapter_backward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                      cudaStream_t stream) {
  if (a.dtype == THANOS_BF16) return backward16(a, workspace, ws_bytes, stream);
  return adapter_f32(true, a, workspace, ws_bytes, stream);
}

}  // namespace thanos
