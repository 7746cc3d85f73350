// Log probabilities of given tokens, with the entropy and the most likely tokens, and their gradient.
//
//   m = max_j z_j,  S = sum_j exp(z_j - m),  log p_j = (z_j - m) - log S
//   H = -sum_j p_j log p_j = log S - (1 / S) sum_j exp(z_j - m) (z_j - m)
//   dz_j = -p_j (G + g_H (log p_j + H)) + g_t [j = t] + sum_i g_i [j = a_i],   G = g_t + sum_i g_i
//
// Both have memory for a floor: the forward pass reads every logit once, the backward pass reads and
// writes it once.
//
// Forward, a CTA per row (a cluster of up to eight where rows are few).  A thread keeps the largest logit
// so far and the two sums relative to it, 32 values at a time; a value costs an exponential, and an SM has
// 16 of those a clock: 30 us of the 52 that 4096 x 32000 bf16 logits take (5.0 TB/s); conversions, clamps
// and two packed additions and multiplications are issued beside them.
// The k most likely: every thread also keeps the largest of each quarter of its batches.  The k-th largest
// of 2 k bins of threads bounds the k-th largest logit from below, so only quarters that reach the bound
// are read again, and what passes is ranked by counting (half of the bins hold a logit above the bound, so
// for logits in no order some 2 k ln 2 = 1.4 k pass): 69 us with k = 16.  What is added follows the pass and
// has nothing beside it in its CTA: of a warp's time 27 % is waiting for loads and 22 % for barriers, with 68
// % of the issue slots used.
// Rows of which more pass than the list holds (constant ones, many masked ones) are searched bit by bit.
//
// Backward, 8192 values a CTA, nothing shared: 2048 x 128000 in 168 to 176 us, 6.0 to 6.2 TB/s.
#include <float.h>

#include "logprobs.cuh"
#include "tc_common.cuh"

namespace thanos {
namespace {

using namespace tc;
using bf16 = __nv_bfloat16;

constexpr int BT = 256;               // threads of a CTA of the gradient
constexpr int MAX_TOP = LOGPROBS_MAX_TOP;
constexpr int MAX_SPLIT = 8;          // CTAs of a cluster that share a row
constexpr int CANDIDATES = 512;
static_assert(CANDIDATES >= MAX_SPLIT * MAX_TOP, "holds a cluster's lists");
static_assert(2 * MAX_TOP <= 128 && MAX_TOP < BT, "bins of the fewest threads; a named column to a thread");
constexpr int U = 4;                  // vectors of a thread's batch
constexpr int QUARTERS = 4;           // a thread's batches in turn, each with a largest logit of its own
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// Exponents are cut off here: 2^-10000 is zero, and zero times a finite number stays zero where the
// entropy's sum meets a masked logit.
constexpr float FAR = -10000.f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN where either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// Two fp32 numbers in a register pair: one instruction for both.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// ------------------------------------------------------------------------------- rows and vectors
// A row of V logits as 16-byte vectors: vector v holds the columns v * VEC - shift and up.  Only the
// first and the last may reach beyond the row; they are read value by value.
template <typename T>
struct Row {
  static constexpr int VEC = 16 / sizeof(T);
  const T* z;
  int V, shift, nv, first, last;  // vectors [first, last) are whole
  __device__ Row(const T* row, int V_) : z(row), V(V_) {
    shift = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    nv = (V + shift + VEC - 1) / VEC;
    first = shift > 0 ? 1 : 0;
    last = (V + shift) / VEC;
  }
  __device__ __forceinline__ int column(int v) const { return v * VEC - shift; }
  __device__ __forceinline__ bool whole(int v) const { return v >= first && v < last; }
  __device__ __forceinline__ uint4 load(int v) const {  // whole(v)
    return *reinterpret_cast<const uint4*>(z + column(v));  // dZ may be Z: no read-only load
  }
  // Any vector; what is not of the row is -infinity.
  __device__ __noinline__ uint4 edge(int v) const {
    uint32_t w[4];
    const int c = column(v);
    auto at = [&](int e) {
      return c + e >= 0 && c + e < V ? __float_as_uint(to_float(z[c + e])) : 0xFF800000u;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VEC == 8) w[e] = at(2 * e) >> 16 | at(2 * e + 1);
      else w[e] = at(e);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ uint4 any(int v) const { return whole(v) ? load(v) : edge(v); }
  static __device__ __forceinline__ uint4 nothing() {
    const uint32_t x = VEC == 8 ? 0xFF80FF80u : 0xFF800000u;
    return make_uint4(x, x, x, x);
  }
  __device__ __forceinline__ void values(int v, float (&x)[VEC]) const { expand(any(v), x); }
  static __device__ __forceinline__ void expand(uint4 r, float (&x)[VEC]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VEC == 8) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      } else {
        x[e] = __uint_as_float(w[e]);
      }
    }
  }
  // Largest of the vector's values, NaN left out.
  static __device__ __forceinline__ float largest(const uint4* r, int n) {
    if constexpr (VEC == 8) {
      __nv_bfloat162 t = *reinterpret_cast<const __nv_bfloat162*>(&r[0].x);
      for (int u = 0; u < n; ++u) {
        const uint32_t w[4] = {r[u].x, r[u].y, r[u].z, r[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) t = __hmax2(t, *reinterpret_cast<const __nv_bfloat162*>(&w[e]));
      }
      return fmaxf(__low2float(t), __high2float(t));
    } else {
      float t = -INFINITY;
      for (int u = 0; u < n; ++u)
        t = fmaxf(t, fmaxf(fmaxf(__uint_as_float(r[u].x), __uint_as_float(r[u].y)),
                           fmaxf(__uint_as_float(r[u].z), __uint_as_float(r[u].w))));
      return t;
    }
  }
};

// Order of logits: by value, NaN above all, zeros of both signs alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (isnan(x)) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  if (o == 0xFFFFFFFFu) return NAN;
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
constexpr uint32_t NO_ORDER = 0x007FFFFFu;  // of -infinity: what is below is no number's
// A logit and its column as one number: the larger is the more likely, equal ones by column.
__device__ __forceinline__ uint64_t key_of(float x, int column) {
  return (uint64_t)order_of(x) << 32 | (uint32_t)~(uint32_t)column;
}
__device__ __forceinline__ int column_of(uint64_t key) { return (int)~(uint32_t)key; }

// ------------------------------------------------------------------------------------ running sums
struct Sums {
  float m, s, t;  // largest (at least -FLT_MAX), sum of 2^d, sum of 2^d d, with d = (z - m) log2(e)
  __device__ __forceinline__ void rebase(float to) {  // to >= m
    const float far = fmaxf((m - to) * LOG2E, FAR), r = ex2(far);
    t = r * fmaf(far, s, t);
    s *= r;
    m = to;
  }
  __device__ __forceinline__ void merge(float om, float os, float ot) {
    Sums o{om, os, ot};
    const float to = fmaxf(m, om);
    rebase(to);
    o.rebase(to);
    s += o.s;
    t += o.t;
  }
  // Over groups of 2 * from neighbouring lanes: one common largest first, then plain sums.
  __device__ __forceinline__ void join(int from) {
    float to = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o <= from) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
    rebase(to);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (o <= from) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
      }
    }
  }
};

template <typename T, int U>
__device__ __forceinline__ void take(Sums& a, const uint4 (&raw)[U], float& seen) {
  constexpr int VEC = 16 / sizeof(T);
  const float top = Row<T>::largest(raw, U);
  seen = fmaxf(seen, top);
  a.rebase(fmaxf(a.m, top));
  const uint64_t neg = pack2(-a.m, -a.m), k2 = pack2(LOG2E, LOG2E);
  uint64_t s2 = pack2(0.f, 0.f), t2 = s2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[VEC];
    Row<T>::expand(raw[u], x);
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
      float d0, d1;
      unpack2(mul2(add2(pack2(x[e], x[e + 1]), neg), k2), d0, d1);
      d0 = max_nan(d0, FAR);
      d1 = max_nan(d1, FAR);
      const uint64_t w = pack2(ex2(d0), ex2(d1));
      s2 = add2(s2, w);
      t2 = fma2(w, pack2(d0, d1), t2);
    }
  }
  float s0, s1, t0, t1;
  unpack2(s2, s0, s1);
  unpack2(t2, t0, t1);
  a.s += s0 + s1;
  a.t += t0 + t1;
}

template <int LT>  // threads
struct Shared {
  Sums warp[LT / 32];
  __align__(16) uint32_t bin[LT];
  uint32_t exact[LT];
  uint32_t bound, guess;
  int count, n_who;
  uint16_t who[LT * QUARTERS];
  uint64_t list[CANDIDATES];
  uint64_t best[MAX_TOP];
  Sums total;  // for the cluster: the warps' may still be read when it is there
};

// Columns of this CTA's vectors [v0, v1) with a logit >= bound, at most CANDIDATES of them in list; the
// count may be larger.  Only the batches of the quarters of threads in `who`.
template <int LT, typename T>
__device__ __forceinline__ void collect(const Row<T>& row, int v0, int v1, float bound, int n_who,
                                        Shared<LT>& sh) {
  constexpr int VEC = Row<T>::VEC;
  const int batches = (v1 - v0 + QUARTERS * U * LT - 1) / (QUARTERS * U * LT);
  const int shift = batches > 1 ? 32 - __clz(batches - 1) : 0;
  for (int i = threadIdx.x; i < (n_who * U) << shift; i += LT) {
    const int w = sh.who[i / U >> shift], j = i / U & ((1 << shift) - 1);
    const int v = v0 + w / QUARTERS + LT * (i % U + U * (w % QUARTERS + QUARTERS * j));
    if (v >= v1) continue;
    float x[VEC];
    row.values(v, x);
    const int c = row.column(v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (x[e] >= bound && c + e >= 0 && c + e < row.V) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < CANDIDATES) sh.list[at] = key_of(x[e], c + e);
      }
    }
  }
}

// The slow way to the k largest, for rows of which more candidates pass than the list holds: the k-th
// largest value bit by bit, then all that are larger, and of those that equal it the first ones.
template <int LT, typename T>
__device__ __noinline__ void select_slowly(const Row<T>& row, int v0, int v1, int k, uint32_t guess,
                                           Shared<LT>& sh) {
  constexpr int VEC = Row<T>::VEC;
  const int tid = threadIdx.x, lane = tid & 31;
  auto count = [&](uint32_t lo) {  // logits whose order is >= lo
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
    int n = 0;
    for (int v = v0 + tid; v < v1; v += LT) {
      float x[VEC];
      row.values(v, x);
      const int c = row.column(v);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        n += c + e >= 0 && c + e < row.V && order_of(x[e]) >= lo ? 1 : 0;
    }
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (lane == 0) atomicAdd(&sh.count, n);
    __syncthreads();
    return sh.count;
  };
  uint32_t kth = guess;
  if (count(guess) < k || (guess != 0xFFFFFFFFu && count(guess + 1u) >= k)) {
    kth = 0;
    for (int bit = 31; bit >= 0; --bit)
      if (count(kth | 1u << bit) >= k) kth |= 1u << bit;
  }
  __syncthreads();
  if (tid == 0) sh.count = 0;
  __syncthreads();
  for (int v = v0 + tid; v < v1; v += LT) {  // what is larger: fewer than k
    float x[VEC];
    row.values(v, x);
    const int c = row.column(v);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (c + e >= 0 && c + e < row.V && order_of(x[e]) > kth)
        sh.list[atomicAdd(&sh.count, 1)] = key_of(x[e], c + e);
  }
  __syncthreads();
  if (tid < 32) {
    int have = sh.count;
    __syncwarp();
    for (int v = v0; v < v1 && have < k; v += 32) {
      float x[VEC];
      const int mine = v + lane, c = row.column(mine);
      int n = 0;
      if (mine < v1) {
        row.values(mine, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) n += c + e >= 0 && c + e < row.V && order_of(x[e]) == kth;
      }
      int upto = n;
      for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += w;
      }
      int at = have + upto - n;
      if (n > 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (c + e >= 0 && c + e < row.V && order_of(x[e]) == kth) {
            if (at < k) sh.list[at] = key_of(x[e], c + e);
            ++at;
          }
        }
      }
      have += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) sh.count = min(have, k);
  }
  __syncthreads();
}

// The first k of list[0 .. n) in best, in order; what is missing is 0 (no logit has that key).
template <int LT>
__device__ void rank_list(Shared<LT>& sh, int n, int k) {
  for (int i = threadIdx.x; i < k; i += LT)
    if (i >= n) sh.best[i] = 0;
  for (int i = threadIdx.x; i < n; i += LT) {
    const uint64_t mine = sh.list[i];
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) before += sh.list[j] > mine ? 1 : 0;
    if (before < k) sh.best[before] = mine;
  }
  __syncthreads();
}

struct ForwardParams {
  const void* Z;
  int64_t ldz;
  const int64_t* target;
  float* logp;
  float* entropy;
  float* stats;
  int64_t* top_index;
  float* top_logp;
  int V, k, split;
};

// LT threads: 256, or 128 for many short rows, where what follows the pass over a row is most of the work
// (4096 x 1000 in bf16, 16 alternatives: 38.6 and 23.9 us; 2048 x 128000: 108 and 123 us).
template <typename T, int LT>
__global__ void __launch_bounds__(LT, LT == 256 ? 5 : 8) logprobs_kernel(const ForwardParams p) {
  __shared__ Shared<LT> sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int S = p.split, rank = S > 1 ? (int)cluster_ctarank() : 0;
  const int64_t r = blockIdx.x / S;
  const Row<T> row(static_cast<const T*>(p.Z) + r * p.ldz, p.V);
  const int v0 = (int)((int64_t)row.nv * rank / S), v1 = (int)((int64_t)row.nv * (rank + 1) / S);
  int64_t target = -1;
  float zt = 0.f;
  if (p.target && rank == 0 && tid == 0) {
    target = p.target[r];
    if (target >= 0 && target < p.V) zt = to_float(row.z[target]);
  }

  // ---- one pass over the row
  Sums a{-FLT_MAX, 0.f, 0.f};
  float seen[QUARTERS];
#pragma unroll
  for (int q = 0; q < QUARTERS; ++q) seen[q] = -INFINITY;
  auto turn = [&]() {
    const float first = seen[0];
#pragma unroll
    for (int q = 0; q + 1 < QUARTERS; ++q) seen[q] = seen[q + 1];
    seen[QUARTERS - 1] = first;
  };
  int batch = 0;
  const int inner = min(v1, row.last);
  for (int v = v0 + tid; v < v1; v += U * LT, ++batch) {
    uint4 raw[U];
    if (v >= row.first && v + (U - 1) * LT < inner) {
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = row.load(v + u * LT);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        raw[u] = v + u * LT < v1 ? row.any(v + u * LT) : Row<T>::nothing();
    }
    take<T, U>(a, raw, seen[0]);
    turn();
  }
  for (; batch % QUARTERS; ++batch) turn();

  // ---- sums of the CTA, in a fixed order
  const int k = p.k;
  // Bins of logits, each of as many threads as leave two bins for one alternative.  A bin stands for the
  // order of its largest, with its own number in the low bits: all different, and no more than eight
  // bits below what it stands for.
  const int held = min(v1 - v0, LT);  // threads with a vector
  int bins = 16;
  while (bins < LT && bins * held < 2 * k * LT) bins *= 2;
  const int wide = LT / bins;
  if (k > 0) {
    float most = fmaxf(fmaxf(seen[0], seen[1]), fmaxf(seen[2], seen[3]));
    for (int o = 1; o < wide; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if ((tid & (wide - 1)) == 0) {
      const int bin = tid / wide;
      sh.bin[bin] = (order_of(most) & ~(uint32_t)(LT - 1)) | (uint32_t)bin;
      sh.exact[bin] = order_of(most);
    }
  }
  a.join(16);
  if (lane == 0) sh.warp[warp] = a;
  if (tid == 0) sh.count = sh.n_who = 0;
  __syncthreads();
  a = sh.warp[lane & (LT / 32 - 1)];
  a.join(LT / 64);

  // ---- the k largest of the CTA
  if (k > 0) {
    const int mine = min(p.V, row.column(v1)) - max(0, row.column(v0));  // logits of this slice
    const int want = min(k, mine);
    // The want-th largest of the bins is no more than the want-th largest of all.
    if (tid < bins) {
      const uint32_t x = sh.bin[tid];
      const uint4* y = reinterpret_cast<const uint4*>(sh.bin);
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < bins / 4; ++j) {
        const uint4 q = y[j];
        before += (q.x > x) + (q.y > x) + (q.z > x) + (q.w > x);
      }
      if (before == want - 1) {
        sh.bound = max(x & ~(uint32_t)(LT - 1), NO_ORDER);
        sh.guess = sh.exact[tid];
      }
    }
    __syncthreads();
    const float bound = value_of(sh.bound);
#pragma unroll
    for (int q = 0; q < QUARTERS; ++q)
      if (seen[q] >= bound)
        sh.who[atomicAdd(&sh.n_who, 1)] = (uint16_t)(tid * QUARTERS + q);
    __syncthreads();
    const bool odd = isnan(a.s);  // a NaN is no thread's largest
    if (!odd) collect(row, v0, v1, bound, sh.n_who, sh);
    __syncthreads();
    if (odd || sh.count > CANDIDATES) select_slowly(row, v0, v1, want, sh.guess, sh);
    const int n = sh.count;
    rank_list(sh, n, k);
  }

  // ---- the row
  if (S > 1) {
    if (tid == 0) sh.total = a;
    cluster_sync_all();
    if (rank == 0) {
      const uint32_t sums = smem_u32(&sh.total), best = smem_u32(&sh.best[0]);
      for (int w = 1; w < S; ++w) {
        const uint32_t at = map_to_cta(sums, w);
        float q[3];
#pragma unroll
        for (int e = 0; e < 3; ++e)
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q[e]) : "r"(at + 4u * e) : "memory");
        a.merge(q[0], q[1], q[2]);
      }
      for (int i = tid; i < S * k; i += LT) {
        uint64_t key;
        asm volatile("ld.shared::cluster.u64 %0, [%1];"
                     : "=l"(key)
                     : "r"(map_to_cta(best, i / k) + 8u * (i % k))
                     : "memory");
        sh.list[i] = key;
      }
    }
    cluster_sync_all();
    if (rank != 0) return;
    if (k > 0) rank_list(sh, S * k, k);
  }
  const bool none = a.s == 0.f;  // every logit is -infinity
  const float logS = none ? 0.f : logf(a.s);
  const float m = none ? -INFINITY : a.m;
  auto logp_of = [&](float z) { return none ? -INFINITY : (z - m) - logS; };
  if (tid == 0) {
    if (p.logp)
      p.logp[r] = target < 0 ? 0.f : target >= p.V ? NAN : isnan(zt) ? zt : logp_of(zt);
    p.entropy[r] = none ? 0.f : logS - LN2 * (a.t / a.s);
    p.stats[2 * r] = m;
    p.stats[2 * r + 1] = logS;
  }
  for (int i = tid; i < k; i += LT) {
    const uint64_t key = sh.best[i];
    p.top_index[r * k + i] = column_of(key);
    p.top_logp[r * k + i] = logp_of(value_of((uint32_t)(key >> 32)));
  }
}

// ---------------------------------------------------------------------------------------- gradient
struct BackwardParams {
  const void* Z;
  int64_t ldz;
  void* dZ;
  int64_t lddz;
  const float* stats;
  const int64_t* target;
  const float* dlogp;
  const float* entropy;
  const float* dentropy;
  const int64_t* top_index;
  const float* dtop;
  int V, k, chunks;
};

constexpr int BU = 4;  // vectors of a thread

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16 from_float<bf16>(float x) { return __float2bfloat16_rn(x); }

// What a row's logits are turned into where nothing is asked of a column by name:
//   y = 2^d (bend d + turn),   d = (z - m) log2(e) - log2 S,   bend = -g_H ln 2,  turn = -(G + g_H H)
struct Slope {
  float m, low, bend, turn;
  __device__ __forceinline__ float operator()(float z) const {
    const float d = max_nan(fmaf(z - m, LOG2E, low), FAR);
    return ex2(d) * fmaf(bend, d, turn);
  }
  __device__ __forceinline__ void two(float& z0, float& z1) const {
    float d0, d1;
    unpack2(fma2(add2(pack2(z0, z1), pack2(-m, -m)), pack2(LOG2E, LOG2E), pack2(low, low)), d0, d1);
    d0 = max_nan(d0, FAR);
    d1 = max_nan(d1, FAR);
    const uint64_t f = fma2(pack2(bend, bend), pack2(d0, d1), pack2(turn, turn));
    unpack2(mul2(pack2(ex2(d0), ex2(d1)), f), z0, z1);
  }
};

// NAMED: gradients of alternatives, whose columns are put right at the end; without them the thread that
// holds the target's column does so on the way.
template <typename T, bool NAMED>
__global__ void __launch_bounds__(BT) logprobs_grad_kernel(const BackwardParams p) {
  constexpr int VEC = 16 / sizeof(T);
  __shared__ int at[MAX_TOP + 1];
  __shared__ float grad[MAX_TOP + 1];
  const int tid = threadIdx.x, lane = tid & 31;
  const int64_t r = blockIdx.x / p.chunks;
  const int chunk = (int)(blockIdx.x - r * p.chunks);
  const Row<T> row(static_cast<const T*>(p.Z) + r * p.ldz, p.V);
  T* out = static_cast<T*>(p.dZ) + r * p.lddz;
  const int v0 = chunk * (BT * BU), v1 = min(row.nv, v0 + BT * BU);
  const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.z)) & 15u) == 0;

  uint4 raw[BU];
#pragma unroll
  for (int u = 0; u < BU; ++u) {
    const int v = v0 + u * BT + tid;
    if (v < v1) raw[u] = row.any(v);
  }
  const float m = p.stats[2 * r], logS = p.stats[2 * r + 1];
  const float gh = p.dentropy ? p.dentropy[r] : 0.f, H = p.dentropy ? p.entropy[r] : 0.f;
  // G, and whether there is anything to pass on: every warp by itself
  const int64_t target = p.target ? p.target[r] : -1;
  const float own = target < 0 ? 0.f : target < p.V ? p.dlogp[r] : NAN;
  const int t = target >= 0 && target < p.V ? (int)target : -1;
  float G = own;
  bool any = G != 0.f || gh != 0.f;
  if constexpr (NAMED) {
    float sum = 0.f;
    bool some = false;
    for (int i = lane; i < p.k; i += 32) {
      const int64_t j = p.top_index[r * p.k + i];
      const bool in = j >= 0 && j < p.V;
      const float g = in ? p.dtop[r * p.k + i] : 0.f;
      if (tid < 32) {
        at[i + 1] = in ? (int)j : -1;
        grad[i + 1] = g;
      }
      sum += g;
      some |= g != 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    any = __any_sync(0xffffffffu, some) || any;
    G += sum;
    if (tid == 0) {
      at[0] = t;
      grad[0] = own;
    }
  }
  any = any && m != -INFINITY;  // nothing was likely: no gradient
  const Slope slope{m, -logS * LOG2E, -gh * LN2, -fmaf(gh, H, G)};
  float named = 0.f;
  int where = -1;
  if constexpr (NAMED) {
    __syncthreads();
    // dZ may be Z: what the named columns hold is read before anything is written
    if (any && tid <= p.k) {
      const int j = at[tid];
      if (j >= 0 && j >= row.column(v0) && j < row.column(v1)) {
        where = j;
        named = slope(to_float(row.z[j]));
        for (int i = 0; i <= p.k; ++i) named += at[i] == j ? grad[i] : 0.f;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < BU; ++u) {
    const int v = v0 + u * BT + tid;
    if (v >= v1) break;
    const int c = row.column(v);
    float y[VEC];
    Row<T>::expand(raw[u], y);
    const bool mine = !NAMED && any && t >= c && t < c + VEC;
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
      if (any) slope.two(y[e], y[e + 1]);
      else y[e] = y[e + 1] = 0.f;
    }
    if (mine) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) y[e] += c + e == t ? own : 0.f;
    }
    if (same && row.whole(v)) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (VEC == 8) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
          w[e] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
          w[e] = __float_as_uint(y[e]);
        }
      }
      *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e >= 0 && c + e < p.V) out[c + e] = from_float<T>(y[e]);
    }
  }
  if constexpr (NAMED) {
    __syncthreads();
    if (where >= 0) out[where] = from_float<T>(named);
  }
}

template <typename T, int LT>
thanos_status_t forward(const LogprobsArgs& a, cudaStream_t stream) {
  ForwardParams p = {};
  p.Z = a.Z;
  p.ldz = a.ldz;
  p.target = a.target;
  p.logp = a.logp;
  p.entropy = a.entropy;
  p.stats = a.stats;
  p.top_index = a.top_index;
  p.top_logp = a.top_logp;
  p.V = (int)a.V;
  p.k = a.k;
  // few rows: several CTAs share one, as long as each has some ten thousand bytes of it
  p.split = 1;
  while (p.split < MAX_SPLIT && a.T * p.split < 2 * NUM_SMS &&
         a.V * (int64_t)sizeof(T) / p.split >= 16384)
    p.split *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.T * p.split), 1, 1);
  cfg.blockDim = dim3(LT, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  THANOS_CUDA(cudaLaunchKernelEx(&cfg, logprobs_kernel<T, LT>, p));
  return THANOS_OK;
}

template <typename T>
thanos_status_t backward(const LogprobsGradArgs& a, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  BackwardParams p = {};
  p.Z = a.Z;
  p.ldz = a.ldz;
  p.dZ = a.dZ;
  p.lddz = a.lddz;
  p.stats = a.stats;
  p.target = a.target;
  p.dlogp = a.dlogp;
  p.entropy = a.entropy;
  p.dentropy = a.dentropy;
  p.top_index = a.top_index;
  p.dtop = a.dtop;
  p.V = (int)a.V;
  p.k = a.k;
  // a row that starts between two vectors has one more
  p.chunks = (int)ceil_div(ceil_div(a.V, VEC) + 1, BT * BU);
  if (p.dtop) logprobs_grad_kernel<T, true><<<(unsigned)(a.T * p.chunks), BT, 0, stream>>>(p);
  else logprobs_grad_kernel<T, false><<<(unsigned)(a.T * p.chunks), BT, 0, stream>>>(p);
  THANOS_CHECK_LAUNCH();
  return THANOS_OK;
}

}  // namespace

thanos_status_t logprobs_impl(const LogprobsArgs& a, cudaStream_t stream) {
  // many rows of a few thousand bytes each
  const int64_t bytes = a.V * (a.dtype == THANOS_BF16 ? 2 : 4);
  if (bytes <= 32768 && a.T >= 8 * NUM_SMS)
    return a.dtype == THANOS_BF16 ? forward<bf16, 128>(a, stream) : forward<float, 128>(a, stream);
  return a.dtype == THANOS_BF16 ? forward<bf16, 256>(a, stream) : forward<float, 256>(a, stream);
}

thanos_status_t logprobs_grad_impl(const LogprobsGradArgs& a, cudaStream_t stream) {
  return a.dtype == THANOS_BF16 ? backward<bf16>(a, stream) : backward<float>(a, stream);
}

}  // namespace thanos
