// relation_paged.cu -- the Relation row of one new token per request over a paged key/value cache.
//
// The row of relation_decode.cu (Sec. 3.1; Sec. 4.2 / App. A.1): with len rows, history
// j < len - 1 and the token itself in row len - 1,
//   E_j = SiLU(q . k_j / sqrt(d)),  L^E = log sum_j e^{E_j},  S = sigmoid(q . k_self / (sqrt(d) tau_S)),
//   A = L^E - lambda log len,  g = sigmoid(A - S),
//   Y = (1 - g) v_self + g sum_j e^{E_j} v_j / sum_j e^{E_j},  logZ = logaddexp(S, A),
// where row r of request b lies in row r % page of page table[b][r / page].  G = H / H_kv query heads
// share a key/value head.
//
// Bound by memory: every cached key and value is read once, for all query heads that share it.  The
// history of all requests and key/value heads is cut into units of kUnit rows, and the units, in the
// order of requests, heads and rows, into as many equal runs as there are CTAs resident: ragged
// lengths leave no CTA idle, and nothing is launched for the rows that a table could hold.  A CTA
// takes its run head by head in one pass: every warp keeps (m, l, z) = (max E, sum e^{E - m},
// sum e^{E - m} v) over tiles of rows that stay in registers, merged at the head's end.  A head that
// lies within one run is finished there; of a head that several runs share, each leaves its (m, l, z)
// in the workspace and the second launch joins them.
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace paged {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxD = 128;
constexpr int kUnit = 64;      // rows of a unit
constexpr int kMaxCtas = 640;  // runs (the workspace holds two partial results of each)
constexpr int kPart = 2 + kMaxD;

template <typename TI>
__device__ __forceinline__ float ldf(const TI* p) {
  return (float)*p;
}

// 16 bytes of a row as fp32
template <typename TI>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&x)[8]) {
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(ww[e] << 16);
      x[2 * e + 1] = __uint_as_float(ww[e] & 0xffff0000u);
    }
  }
};

// Elements c .. c + N - 1 of a row of d, zeros past its end
template <typename TI, bool VEC>
__device__ __forceinline__ uint4 load_group(const TI* row, int c, int d) {
  constexpr int N = Vec<TI>::N;
  if constexpr (VEC) {
    if (c < d) return __ldg(reinterpret_cast<const uint4*>(row + c));
    return make_uint4(0, 0, 0, 0);
  } else {
    union {
      uint4 w;
      unsigned short h[8];
      unsigned int f[4];
    } u;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (sizeof(TI) == 2)
        u.h[e] = c + e < d ? reinterpret_cast<const unsigned short*>(row)[c + e] : 0;
      else
        u.f[e] = c + e < d ? reinterpret_cast<const unsigned int*>(row)[c + e] : 0;
    }
    return u.w;
  }
}

__device__ __forceinline__ float silu(float u) { return u / (1.0f + expf(-u)); }

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// A request's length, 0 (reported) where it lies outside [0, cols * page]
__device__ __forceinline__ int length_of(const PagedProblem& p, int b, bool report) {
  const int len = p.lengths[b];
  if (len >= 0 && len <= p.cols * p.page) return len;
  if (report && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
  return 0;
}
// Units of a head: also one where there is no history
__device__ __forceinline__ int units_of(int len) {
  return len > 1 ? (len - 2) / kUnit + 1 : 1;
}

// Element offset of row r of request b's head 0
__device__ __forceinline__ long long row_at(const PagedProblem& p, int b, int r) {
  const int j = r / p.page;
  int id = __ldg(p.table + (long long)b * p.t_stride + j);
  if (id < 0 || id >= p.n_pages) {  // reported, and read as page 0
    if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    id = 0;
  }
  return (long long)id * p.sP + (long long)(r - j * p.page) * p.sR;
}

// Units per head of all requests, and of those before request b: b_stop, or (b_stop < 0) the one
// that holds the first unit of run `at`.
struct Sums {
  long long before, all;
  int b;
};
__device__ __forceinline__ Sums scan_requests(const PagedProblem& p, long long at, int b_stop,
                                              bool report) {
  __shared__ long long part[kWarps], found[2];
  __shared__ int found_b;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (p.B + kThreads - 1) / kThreads;
  const int lo = min(p.B, (int)threadIdx.x * per), hi = min(p.B, lo + per);
  long long x = 0;
  for (int b = lo; b < hi; ++b) x += units_of(length_of(p, b, report));
  long long s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += t;
  }
  if (lane == 31) part[warp] = s;
  __syncthreads();
  long long before = s - x, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  if (b_stop >= 0) {  // by request
    if (lo <= b_stop && b_stop < hi) {
      for (int b = lo; b < b_stop; ++b) before += units_of(length_of(p, b, false));
      found[0] = before;
      found_b = b_stop;
    }
  } else {  // by run: unit floor(at * U / runs) of the U units of all heads (none for an idle CTA)
    const long long U = all * p.HG, u = at * U / min((long long)gridDim.x, U);
    long long n = before;
    for (int b = lo; b < hi; ++b) {
      const long long e = n + units_of(length_of(p, b, false));
      if (n * p.HG <= u && u < e * p.HG) {
        found[0] = n;
        found_b = b;
      }
      n = e;
    }
  }
  __syncthreads();
  return {found[0], all, found_b};
}

// Column c of a finished row
template <typename TI>
__device__ __forceinline__ void epilogue(const PagedProblem& p, int b, int h, int len, float qk,
                                         float M, float L, float Z, int c, float vi) {
  const float S = 1.0f / (1.0f + expf(-(qk * p.inv_sqrt_d) / p.tau_s));
  float g = 0.f, lz = S, fz = 0.f;
  if (len > 1) {
    const float A = M + logf(L) - p.lambda * logf((float)len);
    g = 1.0f / (1.0f + expf(S - A));
    lz = A > S ? A + log1pf(expf(S - A)) : S + log1pf(expf(A - S));  // NaN stays NaN
    fz = Z / L;
  }
  const bool idle = len < 1;
  reinterpret_cast<TI*>(p.out)[(long long)b * p.qsB + (long long)h * p.qsH + c] =
      (TI)(idle ? 0.f : fmaf(g, fz - vi, vi));
  if (c == 0) p.logz[(long long)b * p.H + h] = idle ? -INFINITY : lz;
}

// q . k_self by one warp
template <typename TI>
__device__ __forceinline__ float self_dot(const PagedProblem& p, const TI* q, const TI* k, int lane) {
  float s = 0.f;
  for (int c = lane; c < p.d; c += 32) s = fmaf(ldf(q + c), ldf(k + c), s);
  return warp_sum(s);
}

template <int GG>
struct Smem {
  float z[kWarps][GG][kMaxD], m[kWarps][GG], l[kWarps][GG];
  float self[GG];
};

constexpr int ctas_per_sm(int GG) { return GG == 1 ? 4 : GG == 2 ? 3 : 2; }

// LPR lanes per row, 32 / LPR rows per load, GG query heads at once.
template <typename TI, int LPR, int GG, bool VEC>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(GG))
    run_kernel(PagedProblem p, float* part) {
  constexpr int VE = Vec<TI>::N, RPL = 32 / LPR;
  constexpr int NI = LPR == 4 ? 4 : 8;  // loads of a tile's keys
  constexpr int R = RPL * NI;           // rows of a tile
  constexpr int DUP = LPR > NI ? LPR / NI : 1;  // lanes that end up with the same row's score
  static_assert(R <= 32, "a lane per row");
  __shared__ Smem<GG> sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = lane / LPR, c0 = (lane % LPR) * VE;
  const int my = (lane % LPR) / DUP * RPL + group;  // the tile's row whose score this lane gets
  pdl_wait();
  const Sums at = scan_requests(p, blockIdx.x, -1, blockIdx.x == 0);
  // as many runs as CTAs, or one for each unit where there are fewer of these
  const long long U = at.all * p.HG, N = min((long long)gridDim.x, U);
  if ((long long)blockIdx.x >= N) return;
  const long long r0 = (long long)blockIdx.x * U / N, r1 = ((long long)blockIdx.x + 1) * U / N;
  int b = at.b;
  long long base = at.before * p.HG;  // the request's first unit
  const int heads = p.H / p.Hk, groups = p.HG / p.Hk;
  for (long long u = r0; u < r1;) {
    int len = length_of(p, b, false), n_u = units_of(len);
    while (u >= base + (long long)n_u * p.HG) {
      base += (long long)n_u * p.HG;
      ++b;
      len = length_of(p, b, false);
      n_u = units_of(len);
    }
    const int hg = (int)((u - base) / n_u), kh = hg / groups, g0 = hg % groups * GG;
    const int ng = min(GG, heads - g0);
    const long long s0 = base + (long long)hg * n_u, s1 = s0 + n_u;  // the head's units
    const long long e = min(r1, s1);
    const int ra = (int)(u - s0) * kUnit, rb = min((int)(e - s0) * kUnit, max(len - 1, 0));
    const bool whole = u == s0 && e == s1;
    const TI* kb = reinterpret_cast<const TI*>(p.k) + (long long)kh * p.sC;
    const TI* vb = reinterpret_cast<const TI*>(p.v) + (long long)kh * p.sC;
    const int h0 = kh * heads + g0;
    const TI* qb = reinterpret_cast<const TI*>(p.q) + (long long)b * p.qsB + (long long)h0 * p.qsH;
    float q[GG][VE], z[GG][VE], m[GG], l[GG];
#pragma unroll
    for (int g = 0; g < GG; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        q[g][i] = g < ng && c0 + i < p.d ? ldf(qb + (long long)g * p.qsH + c0 + i) * p.inv_sqrt_d : 0.f;
        z[g][i] = 0.f;
      }
    }
    for (int j = ra + warp * R; j < rb; j += kWarps * R) {
      // rows past the end read the last one, and are left out below
      const long long mine = row_at(p, b, min(j + lane % R, rb - 1));
      uint4 kr[NI], vr[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const long long off = __shfl_sync(0xffffffffu, mine, i * RPL + group);
        kr[i] = load_group<TI, VEC>(kb + off, c0, p.d);
        vr[i] = load_group<TI, VEC>(vb + off, c0, p.d);
      }
      float P[GG];
#pragma unroll
      for (int g = 0; g < GG; ++g) {
        float s[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          float x[VE];
          Vec<TI>::unpack(kr[i], x);
          s[i] = 0.f;
#pragma unroll
          for (int t = 0; t < VE; ++t) s[i] = fmaf(q[g][t], x[t], s[i]);
        }
        // the sums over a row's lanes, halving the rows per lane while there are any
        int cnt = NI;
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) {
          if (cnt > 1) {
            cnt >>= 1;
#pragma unroll
            for (int i = 0; i < NI / 2; ++i) {
              if (i >= cnt) break;
              const bool up = lane & o;
              const float give = up ? s[i] : s[i + cnt], keep = up ? s[i + cnt] : s[i];
              s[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
          } else {
            s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
          }
        }
        const bool in = j + my < rb;
        const float E = silu(s[0]), mx = in ? E : -INFINITY;
        if (__any_sync(0xffffffffu, mx > m[g])) {
          const float mn = fmaxf(m[g], warp_max(mx)), sc = m[g] == -INFINITY ? 0.f : expf(m[g] - mn);
          m[g] = mn;
          l[g] *= sc;
#pragma unroll
          for (int t = 0; t < VE; ++t) z[g][t] *= sc;
        }
        P[g] = in ? expf(E - m[g]) : 0.f;
        if (lane % DUP == 0) l[g] += P[g];
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float x[VE];
        Vec<TI>::unpack(vr[i], x);
#pragma unroll
        for (int g = 0; g < GG; ++g) {
          const float w = __shfl_sync(0xffffffffu, P[g], group * LPR + i * DUP);
#pragma unroll
          for (int t = 0; t < VE; ++t) z[g][t] = fmaf(w, x[t], z[g][t]);
        }
      }
    }
    // the warp's row groups, then the warps
#pragma unroll
    for (int g = 0; g < GG; ++g) {
      l[g] = warp_sum(l[g]);
#pragma unroll
      for (int t = 0; t < VE; ++t) {
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) z[g][t] += __shfl_xor_sync(0xffffffffu, z[g][t], o);
        if (group == 0 && c0 + t < p.d) sm.z[warp][g][c0 + t] = z[g][t];
      }
      if (lane == 0) {
        sm.m[warp][g] = m[g];
        sm.l[warp][g] = l[g];
      }
    }
    long long self = 0;
    if (whole && len > 0) {
      self = row_at(p, b, len - 1);
      for (int g = warp; g < ng; g += kWarps) {
        const float s = self_dot<TI>(p, qb + (long long)g * p.qsH, kb + self, lane);
        if (lane == 0) sm.self[g] = s;
      }
    }
    __syncthreads();
    const int c = threadIdx.x;
    if (c < p.d) {
      const float vi = whole && len > 0 ? ldf(vb + self + c) : 0.f;
      for (int g = 0; g < ng; ++g) {
        float M = -INFINITY, L = 0.f, Z = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.m[w][g]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float a = sm.l[w][g] == 0.f ? 0.f : expf(sm.m[w][g] - M);
          L = fmaf(a, sm.l[w][g], L);
          Z = fmaf(a, sm.z[w][g][c], Z);
        }
        if (whole) {
          epilogue<TI>(p, b, h0 + g, len, len > 0 ? sm.self[g] : 0.f, M, L, Z, c, vi);
        } else {  // slot 0: the run's first head (begun before it), 1: its last
          float* o = part + (((long long)blockIdx.x * 2 + (u == s0)) * GG + g) * kPart;
          if (c == 0) {
            o[0] = M;
            o[1] = L;
          }
          o[2 + c] = Z;
        }
      }
    }
    __syncthreads();  // sm is written again
    u = e;
  }
}

// Heads that several runs share: a CTA per (request, query head).
template <typename TI>
__global__ void __launch_bounds__(kThreads) join_kernel(PagedProblem p, const float* part, int most,
                                                        int GG) {
  __shared__ float self;
  const int b = blockIdx.x / p.H, h = blockIdx.x % p.H, c = threadIdx.x;
  const int heads = p.H / p.Hk, groups = p.HG / p.Hk;
  const int kh = h / heads, hg = kh * groups + (h - kh * heads) / GG, g = (h - kh * heads) % GG;
  pdl_wait_and_launch();
  const Sums at = scan_requests(p, 0, b, false);
  const int len = length_of(p, b, false);
  const long long U = at.all * p.HG, n_u = units_of(len), s0 = at.before * p.HG + hg * n_u;
  const long long runs = min((long long)most, U);
  // the runs that hold the head's first and last unit
  const int k0 = (int)(((s0 + 1) * runs - 1) / U), k1 = (int)(((s0 + n_u) * runs - 1) / U);
  if (k0 == k1) return;  // (finished there)
  const long long row = row_at(p, b, len - 1) + (long long)kh * p.sC;
  if (c < 32) {
    const float s = self_dot<TI>(p, reinterpret_cast<const TI*>(p.q) + (long long)b * p.qsB +
                                        (long long)h * p.qsH,
                                 reinterpret_cast<const TI*>(p.k) + row, c);
    if (c == 0) self = s;
  }
  __syncthreads();
  if (c >= p.d) return;
  const float vi = ldf(reinterpret_cast<const TI*>(p.v) + row + c);
  auto at_run = [&](int k) {
    const bool begun = (long long)k * U / runs > s0;  // before the run
    return part + (((long long)k * 2 + !begun) * GG + g) * kPart;
  };
  float M = -INFINITY, L = 0.f, Z = 0.f;
  for (int k = k0; k <= k1; ++k) M = fmaxf(M, at_run(k)[0]);
  for (int k = k0; k <= k1; ++k) {
    const float* x = at_run(k);
    const float a = x[1] == 0.f ? 0.f : expf(x[0] - M);
    L = fmaf(a, x[1], L);
    Z = fmaf(a, x[2 + c], Z);
  }
  epilogue<TI>(p, b, h, len, self, M, L, Z, c, vi);
}

template <typename TI, int LPR, int GG, bool VEC>
cudaError_t launch_k(const PagedProblem& p, float* part, cudaStream_t s) {
  int dev = 0, nsm = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
    note_failure("paged decode: device attributes");
    return e;
  }
  const int per = ctas_per_sm(GG), runs = nsm * per < kMaxCtas ? nsm * per : kMaxCtas;
  e = launch_pdl(run_kernel<TI, LPR, GG, VEC>, dim3(runs), kThreads, 0, s, 1, p, part);
  if (e != cudaSuccess) { note_failure("paged decode: launch"); return e; }
  e = launch_pdl(join_kernel<TI>, dim3((unsigned)p.B * p.H), kThreads, 0, s, 1, p,
                 (const float*)part, runs, GG);
  if (e != cudaSuccess) note_failure("paged decode: join launch");
  return e;
}

// Query heads taken together: the group rounded up to a power of two, at most 8
int heads_at_once(int G) { return G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8; }

template <typename TI, int LPR>
cudaError_t launch_lpr(PagedProblem p, bool vec, float* part, cudaStream_t s) {
  const int G = p.H / p.Hk, gg = heads_at_once(G);
  p.HG = p.Hk * ((G + gg - 1) / gg);
  if (vec) {
    switch (gg) {
      case 1: return launch_k<TI, LPR, 1, true>(p, part, s);
      case 2: return launch_k<TI, LPR, 2, true>(p, part, s);
      case 4: return launch_k<TI, LPR, 4, true>(p, part, s);
      default: return launch_k<TI, LPR, 8, true>(p, part, s);
    }
  }
  switch (gg) {
    case 1: return launch_k<TI, LPR, 1, false>(p, part, s);
    case 2: return launch_k<TI, LPR, 2, false>(p, part, s);
    case 4: return launch_k<TI, LPR, 4, false>(p, part, s);
    default: return launch_k<TI, LPR, 8, false>(p, part, s);
  }
}

template <typename TI>
cudaError_t launch_t(const PagedProblem& p, float* part, cudaStream_t s) {
  constexpr int VE = Vec<TI>::N, most = kMaxD / VE;
  uintptr_t low = reinterpret_cast<uintptr_t>(p.k) | reinterpret_cast<uintptr_t>(p.v);
  for (long long x : {p.sP, p.sR, p.sC}) low |= (uintptr_t)(x * (long long)sizeof(TI));
  const bool vec = low % 16 == 0 && p.d % VE == 0;
  const int n = (p.d + VE - 1) / VE;
  if (n <= most / 4) return launch_lpr<TI, most / 4>(p, vec, part, s);
  if (n <= most / 2) return launch_lpr<TI, most / 2>(p, vec, part, s);
  return launch_lpr<TI, most>(p, vec, part, s);
}

}  // namespace paged

size_t paged_workspace_bytes(int H, int Hk) {
  return (size_t)paged::kMaxCtas * 2 * paged::heads_at_once(H / Hk) * paged::kPart * sizeof(float);
}

cudaError_t launch_paged(const PagedProblem& p, void* workspace, cudaStream_t s) {
  float* part = static_cast<float*>(workspace);
  if (p.dtype == RELATION_F32) return paged::launch_t<float>(p, part, s);
  return paged::launch_t<__nv_bfloat16>(p, part, s);
}

}  // namespace rel
