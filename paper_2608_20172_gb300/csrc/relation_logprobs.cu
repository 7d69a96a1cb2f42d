// relation_logprobs.cu -- log probabilities of given tokens, the rows' entropies and top alternatives,
// and the logits' gradient.
//
// A row x_0 .. x_{V-1} at temperature T, M = max x, t_j = (x_j - M) / T:
//   l = sum e^{t_j},  logZ = M / T + log l,  log p_j = t_j - log l,
//   H = -sum p_j log p_j = log l - sum t_j e^{t_j} / l.
// M, l and sum t e^t are taken in one pass: every thread keeps the three of its own elements, and two
// such triples join by t' = t - (M' - M) / T:  l' = l f,  (sum)' = f (sum - l (M' - M) / T),
// f = e^{-(M' - M) / T}.
// The K largest (K <= 32): every thread's maximum is known after the pass.  The K-th largest of 32 of
// these maxima, the largest of the first warps' lanes, is reached by at least K elements, so only lanes
// whose maximum is not below it can hold one of the K; their warp goes through these lanes' elements again
// (from L2: a few hundred elements of a row in place of all) and keeps its K largest in a sorted list, one
// per lane.  The lists' elements are ranked against each other.
// Gradient, of g log p_y + h H + k logZ:
//   dx_j = (1 / T) (g (delta_jy - p_j) - h p_j (log p_j + H) + k p_j).
// log p_j is x_j / T - logZ where logZ is small; other rows' CTA takes M and l again.
//
// Memory is the floor: the logits are read once (gradient: and written).  Few rows are shared by clusters
// of CTAs that join through distributed shared memory.  Measured: 2048 rows of 50257 bf16 42 us, 4.9 TB/s,
// with 20 alternatives 60 us, bound by issue (2.9 instructions per clock); one row of 32000 fp32 with 5
// alternatives 7 us, a chain of barriers; the gradient of 4096 rows of 50257 bf16 130 us, 6.3 TB/s.
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace logprobs {

using u64 = unsigned long long;

constexpr int kMaxTop = 32;
constexpr int kMaxCluster = 8;

template <typename TI>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
  }
};

// A row in groups of 16 aligned bytes: group g holds elements g N - off .. + N - 1, the first and the
// last group in part.
template <typename TI>
struct Row {
  static constexpr int N = Vec<TI>::N;
  const TI* x;
  int V, off, groups;
  __device__ __forceinline__ Row(const TI* row, int V_) : x(row), V(V_) {
    off = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(TI));
    groups = (V + off + N - 1) / N;
  }
  __device__ __forceinline__ bool whole(int g) const { return g * N >= off && g * N - off + N <= V; }
  __device__ __forceinline__ uint4 raw(int g) const {
    return *reinterpret_cast<const uint4*>(x + (g * N - off));
  }
  // the group's elements, -inf outside the row
  __device__ __forceinline__ void load(int g, float (&v)[N]) const {
    if (whole(g)) {
      Vec<TI>::unpack(raw(g), v);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = g * N - off + j;
        v[j] = c >= 0 && c < V ? (float)x[c] : -INFINITY;
      }
    }
  }
};

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
  float m = fmaxf(v[0], v[1]);
#pragma unroll
  for (int j = 2; j < N; j += 2) {
    asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(v[j]), "f"(v[j + 1]));
  }
  return m;
}

// max, sum of e^t, sum of t e^t in units of log 2 (t log2 e)
struct Sums {
  float m = -INFINITY, l = 0.f, s = 0.f;
  // to the scale of a maximum that is not below this one's
  __device__ __forceinline__ void raise(float to, float k2) {
    const float d = (m - to) * k2, f = ex2_approx(d);
    if (m == -INFINITY) {  // (nothing yet, or a NaN)
      m = to;
      return;
    }
    s = f > 0.f ? f * fmaf(l, d, s) : 0.f;
    l *= f;
    m = to;
  }
  // the sums of the warp's lanes, the same bits in each
  __device__ __forceinline__ void join_warp(float k2) {
    float to = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
    if (to != -INFINITY) raise(to, k2);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, o);
      s += __shfl_xor_sync(0xffffffffu, s, o);
    }
  }
};

// Keys that order elements by value, the largest first, equal ones by index (0: none).  -0 is 0.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 key_of(float x, int i) { return (u64)ordered(x) << 32 | (unsigned)~i; }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                   : "memory");
}
__device__ __forceinline__ uint32_t peer(const void* p, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ float peer_f(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ u64 peer_u64(uint32_t a) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

template <int kWarps>
struct Smem {
  float m[kWarps], l[kWarps], s[kWarps];
  float cm, cl, cs;          // this CTA's
  unsigned top[32];          // the largest of the first warps' maxima
  int n;                     // keys in `list`
  u64 list[kMaxCluster * kMaxTop > kWarps * kMaxTop ? kMaxCluster * kMaxTop : kWarps * kMaxTop];
  u64 best[kMaxTop];         // this CTA's K largest
};

// The rank of `key` among the n of list (no two are the same)
__device__ __forceinline__ int rank_of(u64 key, const u64* list, int n) {
  int r = 0;
  for (int i = 0; i < n; ++i) r += list[i] > key;
  return r;
}

template <typename TI, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 8 : 2)
    logprobs_kernel(const __grid_constant__ LogprobsProblem p, int n_cl) {
  constexpr int N = Vec<TI>::N;
  constexpr int kWarps = kThreads / 32;
  __shared__ Smem<kWarps> sm;
  pdl_wait_and_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = (int)blockIdx.x / n_cl, rank = n_cl > 1 ? (int)cluster_rank() : 0;
  const Row<TI> x(static_cast<const TI*>(p.logits) + (long long)row * p.s_row, p.V);
  const float T = p.temperature ? p.temperature[row] : 1.f, scale = 1.f / T, k2 = scale * kLog2e;
  const int target = p.targets[row];
  const bool bad_t = !(T > 0.f) || !isfinite(T) || !isfinite(k2), bad_y = target >= p.V;
  // this CTA's groups, and a thread's: first + thread, + kThreads, ...
  const int g0 = (int)((long long)x.groups * rank / n_cl), g1 = (int)((long long)x.groups * (rank + 1) / n_cl);
  Sums a;
  auto take = [&](const float (&v)[N]) {
    const float mx = max_of(v);
    if (mx > a.m) a.raise(mx, k2);
    const float m = a.m == -INFINITY ? 0.f : a.m;  // (masked so far: every weight is 0)
    const float2 m2 = make_float2(-m, -m), kk = make_float2(k2, k2);
    float2 l = make_float2(0.f, 0.f), s = l;
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      // (-inf would make t e^t NaN: e^t is 0 long before; a NaN stays one)
      float2 t = __fmul2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), m2), kk);
      t.x = max_nan(t.x, -300.f);
      t.y = max_nan(t.y, -300.f);
      const float2 w = make_float2(ex2_approx(t.x), ex2_approx(t.y));
      l = __fadd2_rn(l, w);
      s = __ffma2_rn(w, t, s);
    }
    a.l += l.x + l.y;
    a.s += s.x + s.y;
  };
  {
    constexpr int U = kThreads == 256 ? 2 : 4;  // loads in flight
    int g = g0 + (int)threadIdx.x;
    for (; g + (U - 1) * kThreads < g1; g += U * kThreads) {
      float v[U][N];
      uint4 w[U];
      bool all = true;
#pragma unroll
      for (int i = 0; i < U; ++i) all &= x.whole(g + i * kThreads);
      if (all) {
#pragma unroll
        for (int i = 0; i < U; ++i) w[i] = x.raw(g + i * kThreads);
#pragma unroll
        for (int i = 0; i < U; ++i) Vec<TI>::unpack(w[i], v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i) x.load(g + i * kThreads, v[i]);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) take(v[i]);
    }
    for (; g < g1; g += kThreads) {
      float v[N];
      x.load(g, v);
      take(v);
    }
  }
  const float mine = a.m;
  // the CTA's sums: a warp's at its maximum, then the warps' by every warp
  a.join_warp(k2);
  if (lane == 0) {
    sm.m[warp] = a.m; sm.l[warp] = a.l; sm.s[warp] = a.s;
  }
  // the largest maxima of the first `from` warps' lanes, 32 in all (fewer whole warps than one: no bound)
  const int K = p.top, full = (g1 - g0) / 32;
  int from = kWarps;
  while (from > full) from /= 2;
  if (K > 0) {
    unsigned rest = mine == -INFINITY ? 0u : ordered(mine);
    if (warp < from) {
      for (int i = 0; i < 32 / from; ++i) {
        const unsigned best = __reduce_max_sync(0xffffffffu, rest);
        if (lane == __ffs(__ballot_sync(0xffffffffu, rest == best)) - 1) rest = 0;
        if (lane == 0) sm.top[warp * (32 / from) + i] = best;
      }
    }
    if (threadIdx.x == 0) sm.n = 0;
  }
  __syncthreads();
  a = Sums();
  if (lane < kWarps) {
    a.m = sm.m[lane]; a.l = sm.l[lane]; a.s = sm.s[lane];
  }
  a.join_warp(k2);
  if (K > 0) {
    unsigned low = 0;
    if (from > 0) {  // the K-th of them
      const unsigned one = sm.top[lane];
      int above = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const unsigned other = __shfl_sync(0xffffffffu, one, i);
        above += other > one || (other == one && i < lane);
      }
      low = __shfl_sync(0xffffffffu, one, __ffs(__ballot_sync(0xffffffffu, above == K - 1)) - 1);
    }
    // (-inf and NaN are never kept)
    const float least = low > ordered(-FLT_MAX) ? value_of(low) : -FLT_MAX;
    // the warp's K largest among the elements of its lanes that reach the bound, one a lane
    u64 best = 0;
    unsigned who = __ballot_sync(0xffffffffu, mine >= least);
    // such lanes' groups, one to a lane each, of as many of them at a time as there are lanes for
    const int slices = (g1 - g0 + kThreads - 1) / kThreads;
    int width = 1;
    while (width < slices && width < 32) width *= 2;
    while (who) {
      int of = -1;
      for (int i = 0; i < 32 && who; i += width) {
        if (lane / width == i / width) of = __ffs(who) - 1;
        who &= who - 1;
      }
      for (int i0 = 0; i0 < slices; i0 += width) {
        const int i = i0 + lane % width, g = g0 + warp * 32 + of + i * kThreads;
        float v[N];
        if (of >= 0 && i < slices && g < g1) {
          x.load(g, v);
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] = -INFINITY;
        }
        if (!__any_sync(0xffffffffu, max_of(v) >= least)) continue;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (!__any_sync(0xffffffffu, v[j] >= least)) continue;
          const u64 key = v[j] >= least ? key_of(v[j], g * N - x.off + j) : 0;
          unsigned in = __ballot_sync(0xffffffffu, key > __shfl_sync(0xffffffffu, best, K - 1));
          while (in) {
            const u64 next = __shfl_sync(0xffffffffu, key, __ffs(in) - 1);
            in &= in - 1;
            const int at = __popc(__ballot_sync(0xffffffffu, best > next));
            const u64 up = __shfl_up_sync(0xffffffffu, best, 1);
            best = lane == at ? next : lane > at ? up : best;
          }
        }
      }
    }
    const unsigned have = __ballot_sync(0xffffffffu, lane < K && best != 0);
    int at = 0;
    if (lane == 0 && have) at = atomicAdd(&sm.n, __popc(have));
    at = __shfl_sync(0xffffffffu, at, 0) + lane;
    if (have >> lane & 1) sm.list[at] = best;
    if (threadIdx.x < kMaxTop) sm.best[threadIdx.x] = 0;
    __syncthreads();
    const int n = sm.n;
    if ((int)threadIdx.x < n) {
      const u64 mykey = sm.list[threadIdx.x];
      const int r = rank_of(mykey, sm.list, n);
      if (r < K) sm.best[r] = mykey;
    }
  }
  if (n_cl > 1) {
    if (threadIdx.x == 0) {
      sm.cm = a.m; sm.cl = a.l; sm.cs = a.s;
    }
    __syncthreads();
    cluster_sync();
    if (rank == 0) {
      a = Sums();
      if (lane < n_cl) {
        a.m = peer_f(peer(&sm.cm, lane)); a.l = peer_f(peer(&sm.cl, lane)); a.s = peer_f(peer(&sm.cs, lane));
      }
      a.join_warp(k2);
      if (K > 0) {
        const int n = n_cl * K;
        for (int e = threadIdx.x; e < n; e += kThreads) sm.list[e] = peer_u64(peer(&sm.best[e % K], e / K));
        __syncthreads();
        u64 mykey = 0;
        int r = 0;
        if ((int)threadIdx.x < n) {
          mykey = sm.list[threadIdx.x];
          r = rank_of(mykey, sm.list, n);
        }
        // (this CTA's own list has been read: sm.best can take the row's)
        __syncthreads();
        if (threadIdx.x < kMaxTop) sm.best[threadIdx.x] = 0;
        __syncthreads();
        if (mykey && r < K) sm.best[r] = mykey;
      }
    }
    cluster_sync();  // this CTA's shared memory has been read
    if (rank != 0) return;
  }
  __syncthreads();
  // rows without a finite maximum: +inf shares the probability, -inf has none, NaN is NaN
  if (!isfinite(a.m)) {
    int inf = 0, nan = 0;
    for (int c = threadIdx.x; c < p.V; c += kThreads) {
      const float v = (float)x.x[c];
      inf += v == INFINITY;
      nan |= v != v;
    }
    nan = __syncthreads_or(nan);
    if (threadIdx.x == 0) sm.n = 0;
    __syncthreads();
    if (inf) atomicAdd(&sm.n, inf);
    __syncthreads();
    a.l = nan ? NAN : a.m == INFINITY ? (float)sm.n : 0.f;
    a.s = 0.f;
  }
  const bool none = a.m == -INFINITY && a.l == 0.f;
  const float logl = bad_t ? NAN : logf(a.l);
  auto logp = [&](float v) {  // of a value of the row
    if (none && !bad_t) return -INFINITY;
    const float t = v == a.m ? 0.f : (v - a.m) * scale;
    return t - logl;
  };
  if (threadIdx.x == 0) {
    p.logz[row] = none ? (bad_t ? NAN : -INFINITY) : fmaf(a.m, scale, logl);
    p.entropy[row] = none ? (bad_t ? NAN : 0.f) : logl - kLn2 * (a.s / a.l);
    const bool nan = logl != logl;
    p.logprob[row] = bad_y || nan ? NAN : target < 0 ? 0.f : logp((float)x.x[target]);
    if ((bad_t || bad_y) && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
  }
  if ((int)threadIdx.x < K) {
    const u64 k = sm.best[threadIdx.x];
    const bool nan = logl != logl;
    p.top_tokens[(long long)row * K + threadIdx.x] = nan || !k ? -1 : (int)~(unsigned)k;
    p.top_logprobs[(long long)row * K + threadIdx.x] =
        nan ? NAN : !k ? -INFINITY : logp(value_of((unsigned)(k >> 32)));
  }
}

// Gradient: a CTA takes kChunk groups of a row.
constexpr int kGradThreads = 256, kGradU = 4, kChunk = kGradThreads * kGradU;
constexpr float kNear = 64.f;  // |logz| of the rows whose log p is x / T - logz
constexpr float kLog2eRest = 1.92596303e-8f;  // log2 e less kLog2e

// One of the CTA's threads' values: the largest (NaN: any), or the sum in a fixed order
template <bool MAX>
__device__ __forceinline__ float block_join(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? max_nan(v, y) : v + y;
  }
  __syncthreads();  // (what was joined before has been read)
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < kGradThreads / 32; ++i) v = MAX ? max_nan(v, part[i]) : v + part[i];
  return v;
}

// A whole row by one CTA with its own maximum and sum: large |logz|, infinite logits, no token, NaN.  The row
// is read before any of it is written, each element of the last pass by the thread that writes it: the output
// may be the logits.  4096 rows of 50257 bf16 that all come here take 302 us (an element at a time 475),
// ordinary ones 130; few rows wait for one CTA's three passes, one of 131072 fp32 84 us against 3.
template <typename TI, bool VEC>
__device__ __noinline__ void grad_far(const Row<TI> x, TI* out, int target, float scale, float logz, float H,
                                      float g, float h, float k, int V) {
  constexpr int N = Vec<TI>::N;
  __shared__ float part[kGradThreads / 32];
  const bool bad = logz != logz || target >= V;  // (uniform, as all that follows is but the elements)
  float m = -INFINITY, l = 0.f;
  if (!bad) {
    for (int gr = (int)threadIdx.x; gr < x.groups; gr += kGradThreads) {
      float v[N];
      x.load(gr, v);
#pragma unroll
      for (int j = 0; j < N; ++j) m = max_nan(m, v[j]);
    }
    m = block_join<true>(m, part);
  }
  // t = (x - m) / T; the largest ones' is 0, infinite ones' too
  auto t_of = [&](float v) { return v == m ? 0.f : (v - m) * scale; };
  if (!bad && m != -INFINITY) {
    for (int gr = (int)threadIdx.x; gr < x.groups; gr += kGradThreads) {
      float v[N];
      x.load(gr, v);  // (-inf outside the row: a weight of 0)
#pragma unroll
      for (int j = 0; j < N; ++j) l += ex2_approx(t_of(v[j]) * kLog2e);
    }
    l = block_join<false>(l, part);
  }
  const float logl = logf(l), inv = 1.f / l;
  for (int gr = (int)threadIdx.x; gr < x.groups; gr += kGradThreads) {
    const int at = gr * N - x.off;
    float v[N];
    x.load(gr, v);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float d = NAN;
      if (!bad && m == -INFINITY) {
        d = 0.f;
      } else if (!bad) {
        const float t = t_of(v[j]), q = ex2_approx(t * kLog2e) * inv;
        d = q == 0.f ? 0.f : q * (k - g - h * (t - logl + H));
        if (at + j == target) d += g;
        d *= scale;
      }
      v[j] = d;
    }
    if (VEC && x.whole(gr)) {
      *reinterpret_cast<uint4*>(out + at) = Vec<TI>::pack(v);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (at + j >= 0 && at + j < V) out[at + j] = (TI)v[j];
    }
  }
}

template <typename TI, bool VEC>
__global__ void __launch_bounds__(kGradThreads)
    logprobs_grad_kernel(const __grid_constant__ LogprobsGradProblem p, int chunks) {
  constexpr int N = Vec<TI>::N;
  pdl_wait_and_launch();
  const int row = (int)(blockIdx.x / (unsigned)chunks), chunk = (int)(blockIdx.x - (unsigned)row * chunks);
  const Row<TI> x(static_cast<const TI*>(p.logits) + (long long)row * p.s_row, p.V);
  TI* out = static_cast<TI*>(p.dlogits) + (long long)row * p.s_out;
  uint4 w[kGradU];
  const int first = chunk * kChunk + (int)threadIdx.x;
#pragma unroll
  for (int i = 0; i < kGradU; ++i)
    if (x.whole(first + i * kGradThreads)) w[i] = x.raw(first + i * kGradThreads);
  const float T = p.temperature ? p.temperature[row] : 1.f, scale = 1.f / T;
  const float logz = p.logz[row], H = p.entropy[row];
  const int target = p.targets[row];
  const float g = p.dlogprob && target >= 0 ? p.dlogprob[row] : 0.f;
  const float h = p.dentropy ? p.dentropy[row] : 0.f, k = p.dlogz ? p.dlogz[row] : 0.f;
  // a = log2 p_j:  dx_j = 2^a (c0 + c1 a), and g / T more for the given token.  The factors of x and logz are
  // pairs of numbers: rounded to one each, a was off by 190 u where the two were near 60 (u = 2^-24), which is
  // all of 1 - p of a token that is almost certain.
  const float s2 = scale * kLog2e, z2 = -logz * kLog2e;
  const float s2l = fmaf(scale, kLog2e, -s2) + scale * kLog2eRest, z2l = fmaf(-logz, kLog2e, -z2) - logz * kLog2eRest;
  const float c0 = target >= p.V ? NAN : (k - g - h * H) * scale;  // (no log p: the NaN leads to grad_far)
  const float c1 = -h * kLn2 * scale;
  // log p_j = x_j / T - logz is off by logz's own rounding: up to kNear by 2^-19 at most, as much as by the sum's
  // roundings; beyond, and where a coefficient leaves the type, a row's maximum is taken from its logits first.
  // (a masked token's 2^a, 0, is multiplied by c0 - 300 c1, which has to be finite)
  if (!(fabsf(logz) <= kNear) || !(fabsf(c0) <= 1e38f) || !(fabsf(c1) <= 5e35f) || !isfinite(s2)) {
    if (chunk == 0) grad_far<TI, VEC>(x, out, target, scale, logz, H, g, h, k, p.V);
    return;
  }
  auto grad = [&](float v, int c) {
    const float a = fmaxf(fmaf(v, s2, z2) + fmaf(v, s2l, z2l), -300.f);
    const float d = ex2_approx(a) * fmaf(a, c1, c0);
    return c == target ? fmaf(g, scale, d) : d;
  };
#pragma unroll
  for (int i = 0; i < kGradU; ++i) {
    const int gr = first + i * kGradThreads;
    if (gr >= x.groups) break;
    const int at = gr * N - x.off;
    if (x.whole(gr)) {
      float v[N];
      Vec<TI>::unpack(w[i], v);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 x2 = make_float2(v[j], v[j + 1]);
        float2 a = __fadd2_rn(__ffma2_rn(x2, make_float2(s2, s2), make_float2(z2, z2)),
                              __ffma2_rn(x2, make_float2(s2l, s2l), make_float2(z2l, z2l)));
        // (2^a is 0 long before -inf would make 2^a times a a NaN; a masked token's parts may be infinities of either
        // sign, whose sum is one already: no logit of a row that comes here is)
        a.x = fmaxf(a.x, -300.f);
        a.y = fmaxf(a.y, -300.f);
        const float2 d = __fmul2_rn(make_float2(ex2_approx(a.x), ex2_approx(a.y)),
                                    __ffma2_rn(a, make_float2(c1, c1), make_float2(c0, c0)));
        v[j] = d.x;
        v[j + 1] = d.y;
      }
      if ((unsigned)(target - at) < (unsigned)N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (at + j == target) v[j] = fmaf(g, scale, v[j]);
      }
      if (VEC) {
        *reinterpret_cast<uint4*>(out + at) = Vec<TI>::pack(v);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) out[at + j] = (TI)v[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (at + j >= 0 && at + j < p.V) out[at + j] = (TI)grad((float)x.x[at + j], at + j);
    }
  }
}

template <typename TI>
cudaError_t launch_t(const LogprobsProblem& p, cudaStream_t s) {
  int dev = 0, nsm = 148;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    nsm = 148;
  // Clusters while all rows' CTAs are resident at once and each keeps 4096 elements.  Of many rows eight
  // CTAs of 256 threads fit an SM, so that some read while others join their sums (2048 rows of 50257
  // bf16 with 20 alternatives: 59 us, four of 256 67, two of 512 95); of few, which end in one round, two of
  // 512 with twice the loads in flight a thread (256 rows of 131072 fp32: 25 us against 33).
  int cl = 1;
  while (cl < kMaxCluster && 2LL * cl * p.R <= nsm && p.V / (2 * cl) >= 4096) cl *= 2;
  const cudaError_t e =
      p.R > 2 * nsm ? launch_pdl(logprobs_kernel<TI, 256>, dim3((unsigned)p.R), 256, 0, s, 1, p, 1)
                    : launch_pdl(logprobs_kernel<TI, 512>, dim3((unsigned)p.R * cl), 512, 0, s, cl, p, cl);
  if (e != cudaSuccess) note_failure("log probabilities: launch");
  return e;
}

template <typename TI>
cudaError_t launch_grad_t(const LogprobsGradProblem& p, cudaStream_t s) {
  // a row's groups at any alignment
  const int groups = (p.V + 2 * Vec<TI>::N - 2) / Vec<TI>::N, chunks = (groups + kChunk - 1) / kChunk;
  const long long grid = (long long)p.R * chunks;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  // 16-byte stores where every row of the output lies like its row of logits
  const long long es = sizeof(TI);
  const bool vec = (reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.dlogits)) % 16 == 0 &&
                   (p.R == 1 || (p.s_row - p.s_out) * es % 16 == 0);
  const cudaError_t e =
      vec ? launch_pdl(logprobs_grad_kernel<TI, true>, dim3((unsigned)grid), kGradThreads, 0, s, 1, p, chunks)
          : launch_pdl(logprobs_grad_kernel<TI, false>, dim3((unsigned)grid), kGradThreads, 0, s, 1, p, chunks);
  if (e != cudaSuccess) note_failure("log probabilities, gradient: launch");
  return e;
}

}  // namespace logprobs

int logprobs_max_top() { return logprobs::kMaxTop; }

cudaError_t launch_logprobs(const LogprobsProblem& p, cudaStream_t s) {
  return p.dtype == RELATION_F32 ? logprobs::launch_t<float>(p, s) : logprobs::launch_t<__nv_bfloat16>(p, s);
}

cudaError_t launch_logprobs_grad(const LogprobsGradProblem& p, cudaStream_t s) {
  return p.dtype == RELATION_F32 ? logprobs::launch_grad_t<float>(p, s)
                                 : logprobs::launch_grad_t<__nv_bfloat16>(p, s);
}

}  // namespace rel
