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
// Bound by memory: every cached key and value is gone through once for up to eight query heads that
// share it, and once more for each further eight (32 requests to 4096 rows, 8 key heads of 128 bf16: 8
// query heads each 68 us, 9 108, 16 114).  The history of all requests and key/value heads is cut into
// units of kUnit rows, and the units, in the order of requests, heads and rows, into as many equal runs
// as there are CTAs resident: ragged lengths leave no CTA idle, and nothing is launched for the rows
// that a table could hold.  A CTA takes its run head by head in one pass: every warp keeps
// (m, l, z) = (max E, sum e^{E - m}, sum e^{E - m} v) over tiles of rows that stay in registers, merged
// at the head's end.  A head that lies within one run is finished there; of a head that several runs
// share, each leaves its (m, l, z) in the workspace, the one with its end q . k_self and v_self, and the
// second launch joins them.
// Measured, 32 requests of 1 to 4096 rows, 8 key heads, both launches: bf16 of 128 51 us (81 % of the
// copy bandwidth), of 64 38, of 80 43, of 128 with 2, 4, 8 query heads each 62, 63, 69; fp32 of 128 with
// 1, 2, 4, 8 query heads each 93, 99, 146, 205 (90, 84, 57, 41 %: with 8 the products take 20 % of the
// FMA pipe, and 8 warps an SM, by 246 registers, wait for their loads).  32 requests to 8192 rows of
// 16 x 128 bf16 188 us (97 %); one request of 2048 rows, 12 x 64, 8 us.
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace paged {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxD = 128;
constexpr int kUnit = 64;      // rows of a unit
constexpr int kMaxCtas = 640;  // runs (the workspace holds two partial results of each)
constexpr int kPart = 2 + kMaxD;      // floats of a partial result: m, l, z
constexpr int kOwn = kMaxD + 8;       // of what the run with a shared head's end adds: v_self, q . k_self

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

// 2^x by the special function unit (2 ulp), and through it e^x, whose argument's rounding adds
// |x| 2^-24: the weights e^{E - m} are at most 1 and lose what is far below the largest.
__device__ __forceinline__ float fast_exp(float x) { return ex2_approx(x * 1.4426950408889634f); }
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// (a denominator past 2^126 gives 0 in place of at most 1e-36)
__device__ __forceinline__ float silu(float u) { return __fdividef(u, 1.0f + fast_exp(-u)); }
// The running maximum is raised only where a score exceeds it by more than this: weights up to
// e^kSlack are as exact as those below 1, and a raise touches every accumulator.
constexpr float kSlack = 6.f;

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
// Units of a head: its rows' and one for what every head costs (a head of few rows takes as long as a
// unit of 64 rows, 2300 to 6500 cycles by its width); none without history, where the join writes the row.
// (With a unit for each such row, a batch of 32 with two of them waited 12 of 49 us for the CTA that
// had them.)
__device__ __forceinline__ int units_of(int len) { return len > 1 ? (len - 2) / kUnit + 2 : 0; }

__device__ __forceinline__ int page_of(const PagedProblem& p, int r) {
  return rel::page_of(r, p.page, p.page_mul, p.page_shift);
}
// The page id of row r of request b, and with it the element offset of the row's head 0.  In two
// steps, so that a loop can ask for an id a tile before it uses it.
__device__ __forceinline__ int id_at(const PagedProblem& p, int b, int r) {
  return __ldg(p.table + (long long)b * p.t_stride + page_of(p, r));
}
__device__ __forceinline__ long long row_of(const PagedProblem& p, int id, int r) {
  if (id < 0 || id >= p.n_pages) {  // reported, and read as page 0
    if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    id = 0;
  }
  return (long long)id * p.sP + (long long)(r - page_of(p, r) * p.page) * p.sR;
}
__device__ __forceinline__ long long row_at(const PagedProblem& p, int b, int r) {
  return row_of(p, id_at(p, b, r), r);
}

// a / b for a, b >= 0 (b > 0): in 32 bits where both fit
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return (unsigned)a / (unsigned)b;
  return a / b;
}

// The units of all heads, U = all * HG, cut into `runs` runs: the first `more` of them hold one unit
// more than the others.
struct Cut {
  long long U, each;
  int runs, more;
  __device__ __forceinline__ Cut(long long U, int ctas) : U(U) {
    runs = (int)min((long long)ctas, U);
    each = quotient(U, max(runs, 1));
    more = (int)(U - each * runs);
  }
  __device__ __forceinline__ long long begin(int k) const { return k * each + min(k, more); }
  __device__ __forceinline__ int owner(long long u) const {
    const long long big = more * (each + 1);
    return (int)(u < big ? quotient(u, each + 1) : more + quotient(u - big, each));
  }
};

// A head that run k begins inside of, where it is the first to do so: run k - 1 holds the head's start,
// run `last` its end (request -1: there is no such head).
struct Split {
  int b, hg, last, len;
};

// Where run `run` of at most `ctas` begins: the request, its length and the units (per head) before it;
// and the cut.
struct Place {
  int b, len;
  long long before;
  Cut cut;
};
__device__ __forceinline__ Place find_place(const PagedProblem& p, int run, int ctas) {
  __shared__ long long part[kWarps], found;
  __shared__ int found_b, found_len;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (p.B + kThreads - 1) / kThreads;
  const int lo = min(p.B, (int)threadIdx.x * per), hi = min(p.B, lo + per);
  long long x = 0;
  int len = 0;  // the thread's last request's
  for (int b = lo; b < hi; ++b) x += units_of(len = length_of(p, b, false));
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
  const Cut cut(all * p.HG, ctas);
  if (run < cut.runs) {
    const long long u = cut.begin(run);
    if (before * p.HG <= u && u < (before + x) * p.HG) {  // (one thread's requests hold it)
      int b = lo;
      for (; b < hi - 1; ++b) {
        const int own = length_of(p, b, false), n = units_of(own);
        if (u < (before + n) * p.HG) {
          len = own;
          break;
        }
        before += n;
      }
      found = before;
      found_b = b;
      found_len = len;
    }
  }
  __syncthreads();
  return {found_b, found_len, found, cut};
}

// A row's gate g and logZ from q . k_self and the history's M and L
struct Gate {
  float g, lz;
};
__device__ __forceinline__ Gate gate_of(const PagedProblem& p, int len, float qk, float M, float L) {
  const float S = 1.0f / (1.0f + expf(-(qk * p.inv_sqrt_d) / p.tau_s));
  if (len < 2) return {0.f, S};
  const float A = M + logf(L) - p.lambda * logf((float)len);
  // (logaddexp written so that NaN stays NaN)
  return {1.0f / (1.0f + expf(S - A)),
          A > S ? A + log1pf(expf(S - A)) : S + log1pf(expf(A - S))};
}

// (1 - g) v + g z for 0 < g < 1.  With an infinite v the one product would be one of a difference of
// infinities; the sum has the infinity's value (and NaN where z or g has it).
__device__ __forceinline__ float mix(float g, float z, float v) {
  return fabsf(v) < INFINITY ? fmaf(g, z - v, v) : fmaf(0.f, g, z + v);
}

// q . k_self by one warp
template <typename TI>
__device__ __forceinline__ float self_dot(const PagedProblem& p, const TI* q, const TI* k, int lane) {
  float s = 0.f;
  for (int c = lane; c < p.d; c += 32) s = fmaf(ldf(q + c), ldf(k + c), s);
  return warp_sum(s);
}

// The warps' results of a head's part of a run, for up to GG query heads.
template <int GG>
struct Smem {
  float z[kWarps][GG][kMaxD], m[kWarps][GG], l[kWarps][GG];
  float self[GG];
};

// The rows that a warp takes, as (m, l, z) of GG query heads, on the CUDA cores.  LPR lanes per row,
// 32 / LPR rows per load; scores are summed over a row's lanes with half the rows handed over at
// every step, so that a lane ends up with one row's.  Any type, head size and alignment.
template <typename TI, int LPR, int GG_, bool VEC>
struct Lanes {
  using T = TI;
  static constexpr int GG = GG_;
  static constexpr bool kVec = VEC;
  // per SM, by the registers (unaligned bf16 with 8 query heads spills 276 to 316 bytes even so)
  static constexpr int kCtas = GG == 1 ? 4 : GG == 2 ? 3 : 2;
  static constexpr int VE = Vec<TI>::N, RPL = 32 / LPR;
  static constexpr int NI = LPR == 4 ? 4 : 8;  // loads of a tile's keys
  static constexpr int R = RPL * NI;           // rows of a tile
  static constexpr int DUP = LPR > NI ? LPR / NI : 1;  // lanes that end up with the same row's score
  static constexpr int kRing = 0;  // bytes of a CTA's ring
  static_assert(R <= 32, "a lane per row");
  float q[GG][VE], z[GG][VE], m[GG], l[GG];

  __device__ __forceinline__ void start(const PagedProblem& p, const TI* qb, int ng, int lane) {
    const int c0 = (lane % LPR) * VE;
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
  }
  // rows j .. min(j + R, rb) - 1, of which this lane has looked up row j + lane % R (offset mine)
  __device__ __forceinline__ void tile(const PagedProblem& p, const TI* kb, const TI* vb,
                                       long long mine, int j, int rb, int lane) {
    const int group = lane / LPR, c0 = (lane % LPR) * VE;
    const int my = (lane % LPR) / DUP * RPL + group;  // the tile's row whose score this lane gets
    uint4 kr[NI], vr[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const long long off = __shfl_sync(0xffffffffu, mine, i * RPL + group);
      kr[i] = load_group<TI, VEC>(kb + off, c0, p.d);
      vr[i] = load_group<TI, VEC>(vb + off, c0, p.d);
    }
    // No value of a row past the end: its weight is 0, and 0 times an infinity would be NaN.  Before the
    // scores or after them, by the registers (us before and after them, 32 requests to 4096 rows, 8 key
    // heads of 128: unaligned bf16 with 1, 2, 8 query heads each 99 and 109, 107 and 142, 237 and 224; fp32
    // in 16-byte groups with 4 170 and 146).
    auto cut = [&] {
      if (j + R <= rb) return;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (j + i * RPL + group >= rb) vr[i] = make_uint4(0, 0, 0, 0);
    };
    constexpr bool kEarly = sizeof(TI) == 2 && !VEC && GG <= 2;
    if constexpr (kEarly) cut();
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
      if (__any_sync(0xffffffffu, mx > m[g] + kSlack)) {
        const float mn = fmaxf(m[g], warp_max(mx)), sc = m[g] == -INFINITY ? 0.f : expf(m[g] - mn);
        m[g] = mn;
        l[g] *= sc;
#pragma unroll
        for (int t = 0; t < VE; ++t) z[g][t] *= sc;
      }
      P[g] = in ? fast_exp(E - m[g]) : 0.f;
      if (lane % DUP == 0) l[g] += P[g];
    }
    if constexpr (!kEarly) cut();
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
  // this warp's tiles of rows ra .. rb - 1; `more` asks for what else it wants once the first page ids
  // are on their way
  template <typename F>
  __device__ __forceinline__ void run(const PagedProblem& p, int b, const TI* qb, int ng, const TI* kb,
                                      const TI* vb, int ra, int rb, uint4*, int warp, int lane, F more) {
    start(p, qb, ng, lane);
    // rows past the end read the last one, and are left out of the tile
    auto row = [&](int j) { return min(j + lane % R, rb - 1); };
    int j = ra + warp * R;
    int id = j < rb ? id_at(p, b, row(j)) : 0;
    more();
    for (; j < rb; j += kWarps * R) {
      const long long mine = row_of(p, id, row(j));
      id = j + kWarps * R < rb ? id_at(p, b, row(j + kWarps * R)) : 0;
      tile(p, kb, vb, mine, j, rb, lane);
    }
  }
  __device__ __forceinline__ void finish(const PagedProblem& p, Smem<GG>& sm, int warp, int lane) {
    const int group = lane / LPR, c0 = (lane % LPR) * VE;
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
  }
};

// D += A B on the tensor core: A 16 x 16 by rows, B 16 x 8 by columns, bf16; D 16 x 8 fp32.  With
// r = lane / 4, t = lane % 4 a lane holds A[r][2t, 2t + 1], A[r + 8][..], A[r][2t + 8, 2t + 9],
// A[r + 8][..]; B[2t, 2t + 1][r], B[2t + 8, 2t + 9][r]; D[r][2t, 2t + 1], D[r + 8][..].
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                    uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A sum's parts by the weights' leading bits and by what these leave.  The leading weights are positive,
// so that an infinite value makes their part what the whole is; the others are of either sign, or 0.
__device__ __forceinline__ float whole_of(float hi, float lo) {
  return fabsf(hi) < INFINITY ? hi + lo : hi;
}

// The same for 2 to 8 query heads that share bf16 keys (16-byte groups), on the tensor core, 16 rows
// at a time.  What the products sum over and what they leave in a column may be permuted freely, so
// that the keys and values go from memory to the products in the registers they were loaded to:
//   scores  A = Q (head r), B = K^T: row r of 8, channels: lane t's 16-byte groups t, t + 4, .. of
//           the row, 4 elements of a group per product, the same elements of Q's row in A;
//   Y       A = P (head r), B = V: rows 2t, 2t + 1, 2t + 8, 2t + 9, column r of product (i, e) is
//           channel 8 (r + 8 i) + e, element e of the group that lane r loaded; two rows' elements
//           are brought into one register by a byte permutation.
// (tcgen05 products have at least 64 rows, of which 8 would be used, and read their operands from
// shared memory; the reading of K and V bounds this, not the products.)  A's rows 8 to 15 hold what
// the rounding of P to bf16 drops, itself rounded to bf16: P has 16 bits, and both parts of Y are
// summed in fp32.  A tile comes by cp.async S tiles ahead into the warp's own part of shared memory.
// There a row's 16-byte groups are permuted so that the eight lanes of an access meet no bank twice:
// of keys by bit 2 with the row's parity, of values by bits 1 and 2 with the row's bits 1 and 2.
template <int DK>  // 32-channel groups of a row
struct Tensor {
  using T = __nv_bfloat16;
  static constexpr int GG = 8, R = 16;
  static constexpr bool kVec = true;
  static constexpr int DV = (DK + 1) / 2;  // 64-channel groups of a row
  static constexpr int kRow = 8 * DV;      // 16-byte groups of a row in shared memory
  static constexpr int kStage = 2 * R * kRow;
  static constexpr int S = DK <= 2 ? 3 : 2;  // stages
  static constexpr int kRing = kWarps * S * kStage * 16;
  static constexpr int kCtas = DK <= 2 ? 4 : 3;
  uint32_t q[DK][4];  // the lane's groups of head r's query
  float z[DV][8][4], m, l;

  __device__ __forceinline__ void start(const PagedProblem& p, const T* qb, int ng, int lane) {
    const int r = lane >> 2, t = lane & 3;
    const T* x = qb + (long long)min(r, ng - 1) * p.qsH + 8 * t;  // (d is a multiple of 8)
    const bool whole = (reinterpret_cast<uintptr_t>(x) & 15u) == 0;
#pragma unroll
    for (int i = 0; i < DK; ++i) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r < ng && 32 * i + 8 * t < p.d)
        w = whole ? load_group<T, true>(x, 32 * i, 32 * i + 8) : load_group<T, false>(x, 32 * i, 32 * i + 8);
      q[i][0] = w.x;
      q[i][1] = w.y;
      q[i][2] = w.z;
      q[i][3] = w.w;
    }
#pragma unroll
    for (int i = 0; i < DV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) z[i][e][k] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  // A tile into a stage, kRow lanes to a row, so that an access meets as few lines as there are; lane
  // l has looked up row l % 16 (element offset off).
  __device__ __forceinline__ void fetch(const PagedProblem& p, const T* kb, const T* vb, long long off,
                                        uint4* stage, int lane) const {
    constexpr int PER = 32 / kRow;  // rows of an access
    const int c = lane % kRow, r0 = lane / kRow;
    const uint32_t base = smem_u32(stage);
    const bool in = 8 * c < p.d;
#pragma unroll
    for (int k = 0; k < R / PER; ++k) {
      const int row = r0 + PER * k;
      const long long at = __shfl_sync(0xffffffffu, off, row) + 8 * c;
      if (in) {
        cp16(base + 16 * (row * kRow + (c ^ (row & 1) << 2)), kb + at);
        cp16(base + 16 * ((R + row) * kRow + (c ^ (row >> 1 & 3) << 1)), vb + at);
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void run(const PagedProblem& p, int b, const T* qb, int ng, const T* kb,
                                      const T* vb, int ra, int rb, uint4* ring, int warp, int lane,
                                      F more) {
    constexpr int step = kWarps * R;
    uint4* mine = ring + warp * S * kStage;
    int j = ra + warp * R;
    if (p.d < 64 * DV) {  // channels past the row's end: zeros (the results were in their place)
      for (int i = lane; i < S * kStage; i += 32) mine[i] = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
    // rows past the end read the last one, and are left out of the tile
    const int own = lane & 15;
    auto id = [&](int at) { return at < rb ? id_at(p, b, min(at + own, rb - 1)) : 0; };
    int next[S + 1];
#pragma unroll
    for (int st = 0; st <= S; ++st) next[st] = id(j + st * step);
    more();
#pragma unroll
    for (int st = 0; st < S; ++st) {
      const int at = j + st * step;
      if (at < rb) fetch(p, kb, vb, row_of(p, next[st], min(at + own, rb - 1)), mine + st * kStage, lane);
      cp_commit();
    }
    int ahead = next[S];
    start(p, qb, ng, lane);
    for (int st = 0; j < rb; j += step, st = st + 1 == S ? 0 : st + 1) {
      const int at = j + S * step;
      const int later = id(at + step);
      cp_wait<S - 1>();
      __syncwarp();
      uint4* stage = mine + st * kStage;
      if (j + R <= rb)
        tile<true>(p, stage, j, rb, lane);
      else
        tile<false>(p, stage, j, rb, lane);
      __syncwarp();
      if (at < rb) fetch(p, kb, vb, row_of(p, ahead, min(at + own, rb - 1)), stage, lane);
      cp_commit();
      ahead = later;
    }
    cp_wait<0>();
  }
  template <bool FULL>
  __device__ __forceinline__ void tile(const PagedProblem& p, const uint4* stage, int j, int rb,
                                       int lane) {
    const int r = lane >> 2, t = lane & 3;
    const uint4* ks = stage + r * kRow + t;
    const uint4* vs = stage + (R + 2 * t) * kRow + (r ^ 2 * t);
    float E[4], mx = -INFINITY;
    bool in[4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DK; ++i) {
        const uint4 k = ks[8 * n * kRow + 4 * (i ^ (r & 1))];
        mma(s, q[i][0], 0, q[i][1], 0, k.x, k.y);
        mma(s, q[i][2], 0, q[i][3], 0, k.z, k.w);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        in[2 * n + k] = FULL || j + 8 * n + 2 * t + k < rb;
        E[2 * n + k] = silu(s[k] * p.inv_sqrt_d);
        if (in[2 * n + k]) mx = fmaxf(mx, E[2 * n + k]);
      }
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    if (__any_sync(0xffffffffu, mx > m + kSlack)) {
      const float mn = fmaxf(m, mx), sc = m == -INFINITY ? 0.f : expf(m - mn);
      m = mn;
      l *= sc;
#pragma unroll
      for (int i = 0; i < DV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) z[i][e][k] *= sc;
    }
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float a = in[2 * n] ? fast_exp(E[2 * n] - m) : 0.f;
      const float c = in[2 * n + 1] ? fast_exp(E[2 * n + 1] - m) : 0.f;
      l += a + c;
      hi[n] = pack_bf16x2(a, c);
      lo[n] = pack_bf16x2(a - __uint_as_float(hi[n] << 16), c - __uint_as_float(hi[n] & 0xffff0000u));
    }
#pragma unroll
    for (int i = 0; i < DV; ++i) {
      uint32_t v[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint4 x = vs[((k & 1) + 8 * (k >> 1)) * kRow + 8 * i];
        if (!FULL && !in[k]) x = make_uint4(0, 0, 0, 0);  // (0 times an infinity would be NaN)
        v[k][0] = x.x; v[k][1] = x.y; v[k][2] = x.z; v[k][3] = x.w;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int sel = e & 1 ? 0x7632 : 0x5410;
        mma(z[i][e], hi[0], lo[0], hi[1], lo[1], __byte_perm(v[0][e / 2], v[1][e / 2], sel),
            __byte_perm(v[2][e / 2], v[3][e / 2], sel));
      }
    }
  }
  __device__ __forceinline__ void finish(const PagedProblem& p, Smem<GG>& sm, int warp, int lane) {
    const int r = lane >> 2, t = lane & 3;
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (t == 0) {
      sm.m[warp][r] = m;
      sm.l[warp][r] = l;
    }
#pragma unroll
    for (int i = 0; i < DV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          sm.z[warp][r][8 * (2 * t + k + 8 * i) + e] = whole_of(z[i][e][k], z[i][e][k + 2]);
  }
};

// The key and value of request b's last row into shared memory, by one warp: on their way while the
// history is summed.  (Read after it, they put two trips to memory at every head's end: 500 requests to
// 64 rows, 8 x 128 bf16, 42 us, so 37; 256 to 300 rows 48 and 44; 32 to 4096 rows 58 either way, in fp32
// 103 and 105, 8 x 80 80 and 84.)
template <typename TI, bool VEC>
__device__ __forceinline__ void fetch_self(const PagedProblem& p, int b, int len, const TI* kb,
                                           const TI* vb, TI (&row)[2][kMaxD], int lane) {
  const long long at = row_at(p, b, len - 1);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const TI* x = (i ? vb : kb) + at;
    if constexpr (VEC) {
      constexpr int VE = Vec<TI>::N;
      if (lane * VE < p.d) cp16(smem_u32(&row[i][lane * VE]), x + lane * VE);  // (d <= 32 VE)
    } else {
      for (int c = lane; c < p.d; c += 32) row[i][c] = x[c];
    }
  }
  cp_commit();
}

template <typename Core>
__global__ void __launch_bounds__(kThreads, Core::kCtas)
    run_kernel(PagedProblem p, Split* splits, float* own, float* part) {
  using TI = typename Core::T;
  constexpr int GG = Core::GG;
  // the ring, and then in its place the results
  extern __shared__ uint4 ring[];
  Smem<GG>& sm = *reinterpret_cast<Smem<GG>*>(ring);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  const int k = (int)blockIdx.x;
  const Place at = find_place(p, k, gridDim.x);
  if (k >= at.cut.runs) {
    if (threadIdx.x == 0) splits[k].b = -1;
    return;
  }
  const long long r0 = at.cut.begin(k), r1 = at.cut.begin(k + 1);
  int b = at.b, len = at.len, n_u = units_of(len);
  long long base = at.before * p.HG;  // the request's first unit
  int hg = (int)quotient(r0 - base, n_u);
  // (the record of the head that the run may begin inside of: completed at the end)
  __shared__ Split split;
  __shared__ long long split_end;
  __shared__ __align__(16) TI self[2][kMaxD];  // the token's own key and value
  if (threadIdx.x == 0) {
    const long long s0 = base + (long long)hg * n_u;
    split = {k > 0 && s0 < r0 && at.cut.begin(k - 1) <= s0 ? b : -1, hg, 0, len};
    split_end = s0 + n_u;
  }
  const int heads = p.H / p.Hk, groups = p.HG / p.Hk;
  for (long long u = r0; u < r1;) {
    const int kh = hg / groups, g0 = hg % groups * p.GG, ng = min(p.GG, heads - g0);
    const long long s0 = base + (long long)hg * n_u, s1 = s0 + n_u;  // the head's units
    const long long e = min(r1, s1);
    const int ra = (int)(u - s0) * kUnit, rb = min((int)(e - s0) * kUnit, len - 1);
    const bool whole = u == s0 && e == s1;
    const TI* kb = reinterpret_cast<const TI*>(p.k) + (long long)kh * p.sC;
    const TI* vb = reinterpret_cast<const TI*>(p.v) + (long long)kh * p.sC;
    const int h0 = kh * heads + g0;
    const TI* qb = reinterpret_cast<const TI*>(p.q) + (long long)b * p.qsB + (long long)h0 * p.qsH;
    const bool ends = e == s1;  // the token's own row is this run's
    Core core;
    core.run(p, b, qb, ng, kb, vb, ra, rb, ring, warp, lane, [&] {
      if (ends && warp == kWarps - 1) fetch_self<TI, Core::kVec>(p, b, len, kb, vb, self, lane);
    });
    cp_wait<0>();
    if (Core::kRing > 0) __syncthreads();
    core.finish(p, sm, warp, lane);
    if (GG > 1 && Core::kRing == 0) __syncthreads();
    else __syncwarp();  // (the warp that fetched the row takes the only head)
    if (ends) {
      for (int g = kWarps - 1 - warp; g < ng; g += kWarps) {
        const float s = self_dot<TI>(p, qb + (long long)g * p.qsH, self[0], lane);
        if (lane == 0) sm.self[g] = s;
      }
    }
    __syncthreads();
    // a head per thread: the warps' weights, the gate
    if ((int)threadIdx.x < ng) {
      const int g = threadIdx.x;
      float M = -INFINITY, L = 0.f, a[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.m[w][g]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float l = sm.l[w][g];
        a[w] = l == 0.f ? 0.f : expf(sm.m[w][g] - M);
        L = fmaf(a[w], l, L);
      }
      const float scale = whole ? 1.0f / L : 1.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sm.m[w][g] = a[w] * scale;
      if (whole) {
        const Gate gate = gate_of(p, len, sm.self[g], M, L);
        sm.self[g] = gate.g;
        p.logz[(long long)b * p.H + h0 + g] = gate.lz;
      } else {
        float* o = part + (((long long)k * 2 + (u == s0)) * p.GG + g) * kPart;
        o[0] = M;
        o[1] = L;
        if (ends) own[k * kOwn + kMaxD + g] = sm.self[g];
      }
    }
    __syncthreads();
    TI* out = reinterpret_cast<TI*>(p.out) + (long long)b * p.qsB + (long long)h0 * p.qsH;
    // a column per thread, two heads at a time where a row takes half of them
    const int half = p.d <= kThreads / 2, c = threadIdx.x & (kThreads >> half) - 1;
    if (c < p.d) {
      const float vi = ends ? ldf(&self[1][c]) : 0.f;
      if (ends && !whole && (int)threadIdx.x == c) own[k * kOwn + c] = vi;
      for (int g = threadIdx.x != c; g < ng; g += 1 + half) {
        float Z = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) Z = fmaf(sm.m[w][g], sm.z[w][g][c], Z);
        if (whole)
          out[(long long)g * p.qsH + c] = (TI)mix(sm.self[g], Z, vi);
        else  // slot 0: the run's first head (begun before it), 1: its last
          part[(((long long)k * 2 + (u == s0)) * p.GG + g) * kPart + 2 + c] = Z;
      }
    }
    __syncthreads();  // sm is written again
    u = e;
    if (++hg == p.HG && u < r1) {
      base += (long long)n_u * p.HG;
      hg = 0;
      do n_u = units_of(len = length_of(p, ++b, false));
      while (n_u == 0);
    }
  }
  if (threadIdx.x == 0) {
    if (split.b >= 0) split.last = at.cut.owner(split_end - 1);
    splits[k] = split;
  }
}

// Request b without history: y = v_self and logZ = S, or zero and -inf (idle); a head per warp.
template <typename TI>
__device__ __forceinline__ void first_row(const PagedProblem& p, int b, int h) {
  const int len = length_of(p, b, h == 0), lane = threadIdx.x & 31;
  if (len > 1 || h >= p.H) return;
  const TI* q = reinterpret_cast<const TI*>(p.q) + (long long)b * p.qsB + (long long)h * p.qsH;
  TI* out = reinterpret_cast<TI*>(p.out) + (long long)b * p.qsB + (long long)h * p.qsH;
  const long long at = (len > 0 ? row_at(p, b, 0) : 0) + (long long)(h / (p.H / p.Hk)) * p.sC;
  const TI* v = reinterpret_cast<const TI*>(p.v) + at;
  float lz = -INFINITY;
  for (int c = lane; c < p.d; c += 32) out[c] = len > 0 ? v[c] : (TI)0.f;
  if (len > 0)
    lz = gate_of(p, len, self_dot<TI>(p, q, reinterpret_cast<const TI*>(p.k) + at, lane), 0.f, 1.f).lz;
  if (lane == 0) p.logz[(long long)b * p.H + h] = lz;
}

// The heads that several runs share: a CTA per run (of `most`) that might be the second of one, and
// query head, the runs' weights a thread each, their z with kAhead loads in flight, the first with
// the weights'.  Behind them a warp per request and head, for the requests without history.
template <typename TI>
__global__ void __launch_bounds__(kThreads, 8)
    join_kernel(PagedProblem p, const Split* splits, const float* own, const float* part, int most) {
  constexpr int kAhead = 16;
  __shared__ float red[kWarps], w[kThreads], lw[kThreads];
  const int c = threadIdx.x, warp = c >> 5, lane = c & 31;
  const int k0 = (int)blockIdx.x / p.GG, g = (int)blockIdx.x % p.GG;  // run, head
  const int heads = p.H / p.Hk, groups = p.HG / p.Hk;
  pdl_wait_and_launch();
  if (k0 >= most - 1) {
    const int i = (int)blockIdx.x - (most - 1) * p.GG, per = (p.H + kWarps - 1) / kWarps;
    first_row<TI>(p, i / per, i % per * kWarps + warp);
    return;
  }
  const Split at = splits[k0 + 1];
  if (at.b < 0) return;
  const int kh = at.hg / groups, in_group = at.hg % groups * p.GG + g;
  if (in_group >= heads) return;
  const int b = at.b, h = kh * heads + in_group, n = at.last - k0 + 1;
  // the first of them begins the head (its second slot), the others begin with it
  const long long step = 2LL * p.GG * kPart;
  const float* first = part + (long long)k0 * step + g * kPart;
  const float* begun = first + (long long)p.GG * kPart;
  auto at_run = [&](int i) { return i == 0 ? begun : first + i * step; };
  const bool in = c < p.d;
  const float vi = in ? own[at.last * kOwn + c] : 0.f, qk = own[at.last * kOwn + kMaxD + g];
  float zk[kAhead];
#pragma unroll
  for (int e = 0; e < kAhead; ++e) zk[e] = e < n && in ? at_run(e)[2 + c] : 0.f;
  float M = -INFINITY;
  for (int i = c; i < n; i += kThreads) M = fmaxf(M, at_run(i)[0]);
  M = warp_max(M);
  if (lane == 0) red[warp] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) M = fmaxf(M, red[i]);
  float L = 0.f, Z = 0.f;
  for (int i0 = 0; i0 < n; i0 += kThreads) {  // kThreads runs' weights at a time
    if (i0 > 0) __syncthreads();
    if (i0 + c < n) {
      const float* x = at_run(i0 + c);
      w[c] = x[1] == 0.f ? 0.f : expf(x[0] - M);
      lw[c] = x[1];
    }
    __syncthreads();
    const int m = min(kThreads, n - i0);
    for (int i = 0; i < m; i += kAhead) {
      if (i0 + i > 0) {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) zk[e] = i + e < m && in ? at_run(i0 + i + e)[2 + c] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        if (i + e >= m) break;
        L = fmaf(w[i + e], lw[i + e], L);
        Z = fmaf(w[i + e], zk[e], Z);
      }
    }
  }
  if (!in) return;
  const Gate gate = gate_of(p, at.len, qk, M, L);
  reinterpret_cast<TI*>(p.out)[(long long)b * p.qsB + (long long)h * p.qsH + c] =
      (TI)mix(gate.g, Z / L, vi);
  if (c == 0) p.logz[(long long)b * p.H + h] = gate.lz;
}

template <typename Core>
cudaError_t launch_core(const PagedProblem& p, float* part, cudaStream_t s) {
  int dev = 0, nsm = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
    note_failure("paged decode: device attributes");
    return e;
  }
  constexpr int smem = Core::kRing > (int)sizeof(Smem<Core::GG>) ? Core::kRing : (int)sizeof(Smem<Core::GG>);
  if (smem > 40 * 1024 &&  // (48 KB, less what the kernel declares)
      (e = cudaFuncSetAttribute(run_kernel<Core>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) !=
          cudaSuccess) {
    note_failure("paged decode: shared memory");
    return e;
  }
  const int runs = nsm * Core::kCtas < kMaxCtas ? nsm * Core::kCtas : kMaxCtas;
  Split* splits = reinterpret_cast<Split*>(part);
  float* own = part + kMaxCtas * sizeof(Split) / sizeof(float);
  part = own + kMaxCtas * kOwn;
  e = launch_pdl(run_kernel<Core>, dim3(runs), kThreads, smem, s, 1, p, splits, own, part);
  if (e != cudaSuccess) { note_failure("paged decode: launch"); return e; }
  e = launch_pdl(join_kernel<typename Core::T>,
                 dim3((unsigned)((runs - 1) * p.GG + p.B * ((p.H + kWarps - 1) / kWarps))), kThreads, 0, s,
                 1, p, (const Split*)splits, (const float*)own, (const float*)part, runs);
  if (e != cudaSuccess) note_failure("paged decode: join launch");
  return e;
}

// Query heads taken together: the group rounded up to a power of two, at most 8
int heads_at_once(int G) { return G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8; }

template <typename TI, int LPR, bool VEC>
cudaError_t launch_lanes(const PagedProblem& p, float* part, cudaStream_t s) {
  // (bf16 in 16-byte groups with shared keys takes the tensor core)
  if constexpr (sizeof(TI) == 2 && VEC) return launch_core<Lanes<TI, LPR, 1, VEC>>(p, part, s);
  else switch (p.GG) {
    case 1: return launch_core<Lanes<TI, LPR, 1, VEC>>(p, part, s);
    case 2: return launch_core<Lanes<TI, LPR, 2, VEC>>(p, part, s);
    case 4: return launch_core<Lanes<TI, LPR, 4, VEC>>(p, part, s);
    default: return launch_core<Lanes<TI, LPR, 8, VEC>>(p, part, s);
  }
}

template <typename TI>
cudaError_t launch_t(PagedProblem p, float* part, cudaStream_t s) {
  constexpr int VE = Vec<TI>::N, most = kMaxD / VE;
  const int G = p.H / p.Hk, n = (p.d + VE - 1) / VE;
  p.GG = heads_at_once(G);
  p.HG = p.Hk * ((G + p.GG - 1) / p.GG);
  page_division(p.page, &p.page_mul, &p.page_shift);
  uintptr_t low = reinterpret_cast<uintptr_t>(p.k) | reinterpret_cast<uintptr_t>(p.v);
  for (long long x : {p.sP, p.sR, p.sC}) low |= (uintptr_t)(x * (long long)sizeof(TI));
  if (low % 16 == 0 && p.d % VE == 0) {
    if constexpr (sizeof(TI) == 2) {
      if (G > 1 && p.d <= 32) return launch_core<Tensor<1>>(p, part, s);
      if (G > 1 && p.d <= 64) return launch_core<Tensor<2>>(p, part, s);
      if (G > 1 && p.d <= 96) return launch_core<Tensor<3>>(p, part, s);
      if (G > 1) return launch_core<Tensor<4>>(p, part, s);
    }
    if (n <= most / 4) return launch_lanes<TI, most / 4, true>(p, part, s);
    if (n <= most / 2) return launch_lanes<TI, most / 2, true>(p, part, s);
    return launch_lanes<TI, most, true>(p, part, s);
  }
  if (n <= most / 4) return launch_lanes<TI, most / 4, false>(p, part, s);
  if (n <= most / 2) return launch_lanes<TI, most / 2, false>(p, part, s);
  return launch_lanes<TI, most, false>(p, part, s);
}

}  // namespace paged

size_t paged_workspace_bytes(int H, int Hk) {
  using namespace paged;
  const size_t floats = kOwn + 2 * heads_at_once(H / Hk) * kPart;
  return kMaxCtas * (sizeof(Split) + floats * sizeof(float));
}

cudaError_t launch_paged(const PagedProblem& p, void* workspace, cudaStream_t s) {
  float* part = static_cast<float*>(workspace);
  if (p.dtype == RELATION_F32) return paged::launch_t<float>(p, part, s);
  return paged::launch_t<__nv_bfloat16>(p, part, s);
}

}  // namespace rel
