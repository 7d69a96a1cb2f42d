// relation_sample.cu -- the next token of every row from its logits and a given uniform number.
//
// With scale = 1 / temperature and M the row's largest logit, token j weighs
//   w_j = exp((x_j - M) scale)  (fp32),   q_j = floor(2^40 w_j),
// a whole number, so that sums of weights are exact and the same in any order: the token depends
// neither on the batch nor on how a row is shared out.  (What is cut off is below 2^-40 of the
// largest weight per token; an fp32 sum would lose 2^-24 of itself.)  In the order of descending w,
// equal ones by ascending index, the rules keep a beginning of the row:
//   top-k   the first k
//   top-p   of these the shortest beginning that holds floor(p Q_k) of their mass Q_k
//   min-p   of these the tokens with w_j >= min_p
// and the token is the first in index order whose running sum over the kept ones exceeds floor(u Q).
// temperature 0 takes the largest logit (w_j = 1 there and 0 elsewhere, k = 1).
//
// A cluster of CTAs shares a row: each holds its slice of the weights in shared memory, so that the
// logits are read once.  A cut is found from above: a histogram of the weights' leading bits, of
// which every bin knows its count and its exact mass, names the bin in which the cut lies; while that
// bin holds more than kList tokens, further digits of the key (w_j, index), which no two tokens
// share, narrow it; then its tokens are ranked against each other.  What the CTAs have to know of
// each other goes through distributed shared memory.
// Two CTAs fit an SM (64 KB of weights each at most); issue slots and the waits for the cluster bound
// it.  us a call: 256 rows of 131072 fp32, top-p 160 (0.84 TB/s); 64 rows of 50257 bf16, all parameters
// 26; one row of 32000 fp32 without cuts 5.5, with top-k and top-p 11.5.
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace sample {

namespace cg = cooperative_groups;

using u64 = unsigned long long;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 32 * 1024;  // tokens of a CTA,
constexpr int kShort = 16 * 1024;     // and of one that shares an SM with another
constexpr int kIndexBits = 22;        // of the key: 30 bits of w, then the index from the top down
constexpr int kFirst = 87;            // the exponent of 2^-40, below which a weight is 0
constexpr int kDigit = 8;             // further digits
constexpr int kList = 1024;           // tokens of a bin that every CTA goes through by itself,
constexpr int kRanked = 32;           // and that are ranked against each other
constexpr int kFew = kThreads / 4;    // tokens from the top on that settle top-k and top-p together

// A slice of at most 2^(32 - LOW) tokens: its bins' sums of LOW-bit numbers stay below 2^32.
constexpr int low_bits(bool wide) { return wide ? 17 : 18; }
constexpr int bins_of(int low) { return ((127 - kFirst) << (23 - low)) + 1; }

template <int LOW>
struct Smem {
  static constexpr int kBins = bins_of(LOW);
  union {
    unsigned hist[2][kBins];            // this CTA's bins: tokens, sums of the low bits
    struct {                            // later:
      u64 all[kList];                   // keys of the cluster's tokens in the cut's bin
      union {
        struct {
          unsigned part[4][1 << kDigit];  // a digit's histogram: tokens, the masses in 14-bit parts,
          unsigned d_count[1 << kDigit];  // its sums
          u64 d_mass[1 << kDigit];
        };
        u64 extra[kThreads];            // kept mass of every run that lies in that bin
      };
    };
  };
  unsigned count[kBins];              // the cluster's bins: tokens and masses
  u64 mass[kBins];
  u64 list[2][kList];                 // this CTA's tokens in the cut's bin, of the first and second cut
  int sizes[2][kMaxCluster], n_list;  // every CTA's number of them
  u64 few[kRanked];                   // the last of them
  u64 scan_mass[kWarps], total;
  unsigned scan_count[kWarps];
  u64 kept[kMaxCluster];              // of every CTA: its kept mass,
  float max[kMaxCluster];             // its largest logit (NaN: it has one)
  float red[kWarps];
  // what the threads tell each other
  unsigned bin, inside, above_count;
  u64 above_mass, key, key_mass, wanted;
};

// floor(2^40 w) for 0 <= w <= 1 from the bits of w.  (The conversion instruction to 64 bits bounds a
// pass over the weights: 64 rows of 131072 take 35 us with it.)
__device__ __forceinline__ u64 fixed_of(float w) {
  const unsigned bits = __float_as_uint(w);
  const int left = (int)(bits >> 23) - 110;
  const unsigned top = (bits & 0x7fffffu) | 0x800000u;
  return left >= 0 ? (u64)top << left : (u64)(top >> min(-left, 31));
}
// floor(p mass).  (By one thread: in all of them, the chip's few fp64 units take 2000 cycles.)
__device__ __forceinline__ long long share_of(float p, u64 mass) {
  return (long long)floor((double)p * (double)(long long)mass);
}
__device__ __forceinline__ u64 key_of(float w, int j) {
  return (u64)__float_as_uint(w) << kIndexBits | (u64)((1 << kIndexBits) - 1 - j);
}
__device__ __forceinline__ u64 weight_of_key(u64 key) {
  return fixed_of(__uint_as_float((unsigned)(key >> kIndexBits)));
}

// A bin is the weights that agree in all but their LOW last bits, w = 2^(E - 150) (top + low) with
// the leading one in top.  In units of 2^-40, rounded down, that is
// top << (E - 110) + low << (E - 110), or for E < 110 (top >> (110 - E)) + (low >> (110 - E)): top
// ends in LOW zeros, and a low that is shifted past them adds nothing.
template <int LOW>
__device__ __forceinline__ unsigned low_part(unsigned bits) {
  const int right = 110 - (int)(bits >> 23);
  const unsigned low = bits & ((1u << LOW) - 1);
  return right > 0 ? low >> right : low;
}
template <int LOW>
__device__ __forceinline__ u64 mass_of(int bin, unsigned count, u64 low) {
  const unsigned bits = ((unsigned)bin << LOW) + ((unsigned)kFirst << 23);
  const int right = 110 - (int)(bits >> 23);
  const unsigned top = (bits & 0x7fffffu) | 0x800000u;
  return right > 0 ? (u64)count * (top >> right) + low : ((u64)count * top + low) << -right;
}

// This thread's exclusive sums over the block.
template <typename S>
__device__ __forceinline__ void block_scan(S& sm, unsigned& c, u64& m) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned cs = c;
  u64 ms = m;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, cs, o);
    const u64 y = __shfl_up_sync(0xffffffffu, ms, o);
    if (lane >= o) {
      cs += x;
      ms += y;
    }
  }
  __syncthreads();  // the sums of the last scan have been read
  if (lane == 31) {
    sm.scan_count[warp] = cs;
    sm.scan_mass[warp] = ms;
  }
  __syncthreads();
  if (warp == 0 && lane < kWarps) {
    const unsigned c0 = sm.scan_count[lane];
    const u64 m0 = sm.scan_mass[lane];
    unsigned x = c0;
    u64 y = m0;
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
      const unsigned xo = __shfl_up_sync(0xffffu, x, o);
      const u64 yo = __shfl_up_sync(0xffffu, y, o);
      if (lane >= o) {
        x += xo;
        y += yo;
      }
    }
    sm.scan_count[lane] = x - c0;
    sm.scan_mass[lane] = y - m0;
  }
  __syncthreads();
  c = cs - c + sm.scan_count[warp];
  m = ms - m + sm.scan_mass[warp];
}

// A histogram's bins from the highest down, a run of them per thread, and the sums above this
// thread's.
struct Bins {
  const unsigned* count;
  const u64* mass;
  int first, last;  // from, and down to but without
  unsigned c;
  u64 m;
  template <typename S>
  __device__ __forceinline__ Bins(S& sm, const unsigned* count, const u64* mass, int bins,
                                  unsigned above_count, u64 above_mass, u64* total)
      : count(count), mass(mass), c(0), m(0) {
    const int per = (bins + kThreads - 1) / kThreads;
    first = bins - 1 - (int)threadIdx.x * per;
    last = max(first - per, -1);
    for (int d = first; d > last; --d) {
      c += count[d];
      m += mass[d];
    }
    const u64 own = m;
    block_scan(sm, c, m);
    if (total && threadIdx.x == kThreads - 1) *total = m + own;
    c += above_count;
    m += above_mass;
  }
  // The bin in which the running count (by_mass: mass) reaches `want`, into sm.bin, sm.inside (its
  // tokens) and sm.above_*; sm.inside 0: in none.
  template <typename S>
  __device__ __forceinline__ void find(S& sm, bool by_mass, u64 want) const {
    if (threadIdx.x == 0) sm.inside = 0;
    __syncthreads();
    unsigned ca = c;
    u64 ma = m;
    for (int d = first; d > last; --d) {
      const unsigned n = count[d];
      const u64 q = mass[d];
      if (by_mass ? ma < want && want <= ma + q : ca < want && want <= (u64)ca + n) {
        sm.bin = d;
        sm.inside = n;
        sm.above_count = ca;
        sm.above_mass = ma;
      }
      ca += n;
      ma += q;
    }
    __syncthreads();
  }
};

// Sum the CTAs' bins: each CTA adds up its share of them and hands it to all.
template <typename S, typename F>
__device__ __forceinline__ void add_bins(cg::cluster_group& cl, S& sm, unsigned* count, u64* mass,
                                         int bins, F own) {
  const int C = (int)cl.num_blocks(), share = (bins + C - 1) / C, b0 = (int)cl.block_rank() * share;
  cl.sync();
  for (int i = b0 + (int)threadIdx.x; i < min(bins, b0 + share); i += kThreads) {
    unsigned c = 0;
    u64 m = 0;
    own(i, c, m);
    for (int r = 0; r < C; ++r) {
      cl.map_shared_rank(count, r)[i] = c;
      cl.map_shared_rank(mass, r)[i] = m;
    }
  }
  cl.sync();
}

// Sums of fixed_of in 32-bit operations: floor(2^20 w) is what remains of w 2^20 + 2^23 when the sum
// is cut to its 24 bits, and the rest of w 2^20 gives the next 20 bits in the same way; both numbers
// are added up with the bits of 2^23, which `value` takes off again.  At most 2^11 weights.
struct Mass {
  unsigned hi = 0, lo = 0, n = 0;
  __device__ __forceinline__ void add(float w) {
    const float t = __fmaf_rz(w, 1048576.f, 8388608.f);
    const float f = __fmaf_rn(t, 1048576.f, -8796093022208.f);  // 2^20 floor(2^20 w)
    const float r = __fadd_rz(__fmaf_rn(w, 1099511627776.f, -f), 8388608.f);
    hi += __float_as_uint(t);
    lo += __float_as_uint(r);
    ++n;
  }
  __device__ __forceinline__ u64 value() const {
    const unsigned bias = n * 0x4b000000u;
    return ((u64)(hi - bias) << 20) + (lo - bias);
  }
};

// A thread's run of the slice, w[i0 .. i1).
struct Run {
  int i0, i1, len;
};

__device__ __forceinline__ void clear(unsigned* x, int n) {
  for (int i = threadIdx.x; i < n; i += kThreads) x[i] = 0;
}
// A key's digit at `shift` into the digit's histogram.
template <typename S>
__device__ __forceinline__ void count_digit(S& sm, u64 key, int shift, int bits) {
  const unsigned d = (unsigned)(key >> shift) & ((1u << bits) - 1);
  const u64 q = weight_of_key(key);
  atomicAdd(&sm.part[0][d], 1u);
  atomicAdd(&sm.part[1][d], (unsigned)q & 0x3fff);
  atomicAdd(&sm.part[2][d], (unsigned)(q >> 14) & 0x3fff);
  atomicAdd(&sm.part[3][d], (unsigned)(q >> 28));
}
template <typename S>
__device__ __forceinline__ u64 part_mass(const S& sm, int i) {
  return (u64)sm.part[1][i] + ((u64)sm.part[2][i] << 14) + ((u64)sm.part[3][i] << 28);
}

// The key of the cut that lies in sm.bin, among sm.inside tokens, and the mass down to and with it.
// *above (if set) gets the mass of this thread's run down to the cut, without weights below min_p.
template <int LOW>
__device__ __forceinline__ u64 find_key(cg::cluster_group& cl, Smem<LOW>& sm, const float* w,
                                        const Run& run, int j0, int which, bool by_mass, u64 want,
                                        float min_p, u64* mass, u64* above) {
  const int tid = threadIdx.x, C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  u64 prefix = sm.bin + ((u64)kFirst << (23 - LOW));  // the key's bits from `shift` up
  int shift = kIndexBits + LOW;
  unsigned above_count = sm.above_count;
  u64 above_mass = sm.above_mass;
  while (sm.inside > kList) {
    const int bits = min(kDigit, shift);
    shift -= bits;
    __syncthreads();
    clear(&sm.part[0][0], 4 << kDigit);
    __syncthreads();
    for (int i = run.i0; i < run.i1; ++i) {
      const u64 key = key_of(w[i], j0 + i);
      if (key >> (shift + bits) == prefix) count_digit(sm, key, shift, bits);
    }
    add_bins(cl, sm, sm.d_count, sm.d_mass, 1 << kDigit, [&](int i, unsigned& c, u64& m) {
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        if (r >= C) break;
        const Smem<LOW>* o = cl.map_shared_rank(&sm, r);
        c += o->part[0][i];
        m += part_mass(*o, i);
      }
    });
    Bins(sm, sm.d_count, sm.d_mass, 1 << kDigit, above_count, above_mass, nullptr)
        .find(sm, by_mass, want);
    prefix = prefix << bits | sm.bin;
    above_count = sm.above_count;
    above_mass = sm.above_mass;
  }
  // The bin's tokens, of all CTAs, and the run's mass above it.  (Mostly the weight's bits alone
  // tell where a token lies.)
  if (tid == 0) sm.n_list = 0;
  __syncthreads();
  u64* list = sm.list[which];
  Mass sum;
  if (shift >= kIndexBits) {
    const int right = shift - kIndexBits;
    const unsigned high = (unsigned)prefix;
#pragma unroll 4
    for (int i = run.i0; i < run.i1; ++i) {
      const float x = w[i];
      const unsigned bits = __float_as_uint(x) >> right;
      if (bits == high) list[atomicAdd(&sm.n_list, 1)] = key_of(x, j0 + i);
      if (above) sum.add(bits > high && !(x < min_p) ? x : 0.f);
    }
  } else {
    for (int i = run.i0; i < run.i1; ++i) {
      const float x = w[i];
      const u64 key = key_of(x, j0 + i), high = key >> shift;
      if (high == prefix) list[atomicAdd(&sm.n_list, 1)] = key;
      if (above) sum.add(high > prefix && !(x < min_p) ? x : 0.f);
    }
  }
  __syncthreads();
  const int mine = sm.n_list;
  if (tid < C) cl.map_shared_rank(&sm, tid)->sizes[which][rank] = mine;
  cl.sync();
  int total = 0;  // <= kList
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) {
    if (r >= C) break;
    const int m = sm.sizes[which][r];
    const u64* from = cl.map_shared_rank(list, r);
    for (int i = tid; i < m; i += kThreads) sm.all[total + i] = from[i];
    total += m;
  }
  // from here on every CTA by itself: further digits of these tokens,
  unsigned left = total;
  while (left > kRanked) {
    const int bits = min(kDigit, shift);
    shift -= bits;
    clear(&sm.part[0][0], 4 << kDigit);
    __syncthreads();
    for (int i = tid; i < total; i += kThreads) {
      const u64 key = sm.all[i];
      if (key >> (shift + bits) == prefix) count_digit(sm, key, shift, bits);
    }
    __syncthreads();
    if (tid < 32) {  // one warp, 8 bins a lane, from the highest down
      constexpr int kPer = (1 << kDigit) / 32;
      const int first = (1 << kDigit) - 1 - tid * kPer;
      unsigned c = 0;
      u64 m = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        c += sm.part[0][first - i];
        m += part_mass(sm, first - i);
      }
      unsigned ca = c;
      u64 ma = m;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned x = __shfl_up_sync(0xffffffffu, ca, o);
        const u64 y = __shfl_up_sync(0xffffffffu, ma, o);
        if (tid >= o) {
          ca += x;
          ma += y;
        }
      }
      ca += above_count - c;
      ma += above_mass - m;
      for (int i = 0; i < kPer; ++i) {
        const unsigned n = sm.part[0][first - i];
        const u64 q = part_mass(sm, first - i);
        if (by_mass ? ma < want && want <= ma + q : ca < want && want <= (u64)ca + n) {
          sm.bin = first - i;
          sm.inside = n;
          sm.above_count = ca;
          sm.above_mass = ma;
        }
        ca += n;
        ma += q;
      }
    }
    __syncthreads();
    prefix = prefix << bits | sm.bin;
    above_count = sm.above_count;
    above_mass = sm.above_mass;
    left = sm.inside;
  }
  // and the last ones' ranks
  if (tid == 0) sm.n_list = 0;
  __syncthreads();
  for (int i = tid; i < total; i += kThreads) {
    const u64 key = sm.all[i];
    if (key >> shift == prefix) sm.few[atomicAdd(&sm.n_list, 1)] = key;
  }
  __syncthreads();
  if (tid < (int)left) {
    const u64 key = sm.few[tid], q = weight_of_key(key);
    unsigned c = above_count;
    u64 m = above_mass;
    for (int i = 0; i < (int)left; ++i) {
      const u64 other = sm.few[i];
      if (other > key) {
        ++c;
        m += weight_of_key(other);
      }
    }
    if (by_mass ? m < want && want <= m + q : c + 1 == want) {
      sm.key = key;
      sm.key_mass = m + q;
    }
  }
  if (above) sm.extra[tid] = 0;
  __syncthreads();
  const u64 found = sm.key;
  *mass = sm.key_mass;
  if (above) {
    for (int i = tid; i < mine; i += kThreads) {
      const u64 key = list[i];
      const int at = (1 << kIndexBits) - 1 - (int)(key & ((1 << kIndexBits) - 1)) - j0;
      if (key >= found && !(__uint_as_float((unsigned)(key >> kIndexBits)) < min_p))
        atomicAdd(&sm.extra[at / run.len], weight_of_key(key));
    }
    __syncthreads();
    *above = sum.value() + sm.extra[tid];
  }
  __syncthreads();  // (sm.key and the digit's histogram are written again)
  return found;
}

// Both cuts where the bins down to the one with the k-th token, sm.bin, hold at most kFew tokens: these
// are ranked against each other, four threads to a token.  The last kept token's key; *above gets the
// kept mass of this thread's run, without weights below min_p.
template <int LOW>
__device__ __forceinline__ u64 find_few(cg::cluster_group& cl, Smem<LOW>& sm, const float* w,
                                        const Run& run, int j0, unsigned k, float top_p, float min_p,
                                        u64* above) {
  const int tid = threadIdx.x, C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const unsigned low = ((unsigned)sm.bin << LOW) + ((unsigned)kFirst << 23);
  if (tid == 0) sm.n_list = 0;
  __syncthreads();
  u64* list = sm.list[0];
#pragma unroll 4
  for (int i = run.i0; i < run.i1; ++i)
    if (__float_as_uint(w[i]) >= low) list[atomicAdd(&sm.n_list, 1)] = key_of(w[i], j0 + i);
  __syncthreads();
  const int mine = sm.n_list;
  if (tid < C) cl.map_shared_rank(&sm, tid)->sizes[0][rank] = mine;
  cl.sync();
  int total = 0;
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) {
    if (r >= C) break;
    const int m = sm.sizes[0][r];
    if (tid >= total && tid < total + m) sm.all[tid] = cl.map_shared_rank(list, r)[tid - total];
    total += m;
  }
  sm.extra[tid] = 0;
  __syncthreads();
  const int g = tid >> 2;
  const u64 key = g < total ? sm.all[g] : ~0ull, q = g < total ? weight_of_key(key) : 0;
  unsigned c = 0;
  u64 m = 0;
#pragma unroll 4
  for (int i = tid & 3; i < total; i += 4) {
    const u64 other = sm.all[i];
    if (other > key) {
      ++c;
      m += weight_of_key(other);
    }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    c += __shfl_xor_sync(0xffffffffu, c, o);
    m += __shfl_xor_sync(0xffffffffu, m, o);
  }
  const bool one = (tid & 3) == 0 && g < total && c < k;
  if (one && c + 1 == k) sm.wanted = (u64)max(share_of(top_p, m + q), 1LL);
  __syncthreads();
  const u64 want = sm.wanted;
  if (one && m < want && (c + 1 == k || want <= m + q)) sm.key = key;
  __syncthreads();
  const u64 found = sm.key;
  for (int i = tid; i < mine; i += kThreads) {
    const u64 own = list[i];
    const int at = (1 << kIndexBits) - 1 - (int)(own & ((1 << kIndexBits) - 1)) - j0;
    if (own >= found && !(__uint_as_float((unsigned)(own >> kIndexBits)) < min_p))
      atomicAdd(&sm.extra[at / run.len], weight_of_key(own));
  }
  __syncthreads();
  *above = sm.extra[tid];
  return found;
}

// The larger of two, NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The slice into shared memory as fp32, and its largest (NaN if it holds one).  16-byte groups
// between the first and the last boundary; `w` starts where such a group falls on one, too.
template <typename TI>
__device__ __forceinline__ float load_slice(const TI* x, int n, float* w) {
  constexpr int G = 16 / (int)sizeof(TI);
  const int tid = threadIdx.x;
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15u)) % 16 / sizeof(TI)));
  const int groups = (n - head) / G;
  float mx = -INFINITY;
  auto take = [&](float v) { mx = max_nan(mx, v); };
  for (int i = tid; i < head; i += kThreads) take(w[i] = (float)x[i]);
  for (int i = head + groups * G + tid; i < n; i += kThreads) take(w[i] = (float)x[i]);
  const uint4* xs = reinterpret_cast<const uint4*>(x + head);
  float* ws = w + head;
  constexpr int kAhead = 4;
  for (int g0 = tid; g0 < groups; g0 += kAhead * kThreads) {
    uint4 r[kAhead];
#pragma unroll
    for (int t = 0; t < kAhead; ++t)
      if (g0 + t * kThreads < groups) r[t] = __ldg(xs + g0 + t * kThreads);
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      const int g = g0 + t * kThreads;
      if (g >= groups) break;
      const uint32_t u[4] = {r[t].x, r[t].y, r[t].z, r[t].w};
      float v[G];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(TI) == 4) {
          v[e] = __uint_as_float(u[e]);
        } else {
          v[2 * e] = __uint_as_float(u[e] << 16);
          v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int e = 0; e < G; e += 4) {
        *reinterpret_cast<float4*>(ws + g * G + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        take(v[e]);
        take(v[e + 1]);
        take(v[e + 2]);
        take(v[e + 3]);
      }
    }
  }
  return mx;
}

template <typename TI, int LOW>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleProblem p, int slice) {
  using S = Smem<LOW>;
  extern __shared__ __align__(16) unsigned char raw[];
  S& sm = *reinterpret_cast<S*>(raw);
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int row = (int)blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int j0 = min(p.V, rank * slice), n = min(slice, p.V - j0);
  cl.barrier_arrive();  // (waited for before the first access to another CTA's shared memory)
  pdl_wait_and_launch();
  const float temperature = p.temperature ? p.temperature[row] : 1.f, u = p.u[row];
  const bool greedy = temperature == 0.f;
  const float scale = greedy ? 1.f : __fdiv_rn(1.f, temperature);
  const int k = greedy ? 1 : p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f;
  float min_p = p.min_p ? p.min_p[row] : 0.f;
  min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;  // (NaN: no cut, as a NaN top_p)
  const bool valid = temperature >= 0.f && temperature < INFINITY && u >= 0.f && u <= 1.f;
  const bool by_k = k > 0 && k < p.V, by_p = top_p < 1.f;
  // the slice, and the row's largest logit
  const TI* x = reinterpret_cast<const TI*>(p.logits) + (long long)row * p.s_row + j0;
  float* w = reinterpret_cast<float*>(raw + (sizeof(S) + 15) / 16 * 16);
  w += (4 - (16 - (reinterpret_cast<uintptr_t>(x) & 15u)) % 16 / sizeof(TI) % 4) % 4;
  float mx = load_slice<TI>(x, n, w);
  if (by_k || by_p)
    for (int i = tid; i < 2 * S::kBins; i += kThreads) (&sm.hist[0][0])[i] = 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  if (lane == 0) sm.red[warp] = mx;
  __syncthreads();
  cl.barrier_wait();
  if (tid < C) {  // to every CTA
#pragma unroll
    for (int i = 0; i < kWarps; ++i) mx = max_nan(mx, sm.red[i]);
    cl.map_shared_rank(&sm, tid)->max[rank] = mx;
  }
  cl.sync();
  float M = -INFINITY;
  for (int r = 0; r < C; ++r) M = max_nan(M, sm.max[r]);
  const bool nan = M != M;
  if (!valid || nan || M == -INFINITY) {  // (the same in every CTA of the cluster)
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      p.logprob[row] = valid && !nan ? -INFINITY : NAN;
      p.logz[row] = valid && !nan ? -INFINITY : NAN;
      if (!valid && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    }
    return;
  }
  // the weights.  Every thread takes a run of the slice of odd length, so that neither the lanes'
  // accesses collide nor the index order is lost.
  const int len = (slice + kThreads - 1) / kThreads | 1, i0 = min(n, tid * len), i1 = min(n, i0 + len);
  const Run run{i0, i1, len};
  // (greedy: a difference times infinity)
  const float slope = greedy ? INFINITY : scale;
  u64 sum = 0;
  auto weight_of = [&](int i) {
    const float v = w[i];
    return w[i] = v == M ? 1.f : expf(__fmul_rn(__fsub_rn(v, M), slope));
  };
  if (by_k || by_p) {
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
      const unsigned bits = __float_as_uint(weight_of(i));
      const int bin = (int)(bits >> LOW) - (kFirst << (23 - LOW));
      if (bin >= 0) {
        atomicAdd(&sm.hist[0][bin], 1u);
        if (by_p) atomicAdd(&sm.hist[1][bin], low_part<LOW>(bits));  // (counts alone find the k-th)
      }
    }
  } else {
    Mass kept;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
      const float e = weight_of(i);
      kept.add(e < min_p ? 0.f : e);
    }
    sum = kept.value();
  }
  u64 least = 0;
  if (by_k || by_p) {
    add_bins(cl, sm, sm.count, sm.mass, S::kBins, [&](int i, unsigned& c, u64& m) {
      unsigned cs[kMaxCluster], ls[kMaxCluster];  // (all in flight)
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        const S* o = cl.map_shared_rank(&sm, min(r, C - 1));
        cs[r] = o->hist[0][i];
        ls[r] = o->hist[1][i];
      }
      u64 low = 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        c += r < C ? cs[r] : 0;
        low += r < C ? ls[r] : 0;
      }
      m = mass_of<LOW>(i, c, low);
    });
    const Bins bins(sm, sm.count, sm.mass, S::kBins, 0, 0, &sm.total);
    __syncthreads();
    u64 mass = sm.total;
    bool summed = false;
    if (by_k) bins.find(sm, false, (u64)k);
    const unsigned inside = by_k ? sm.inside : 0;
    if (by_p && inside && sm.above_count + inside <= kFew) {
      // (one row of 32000, k 50, p 0.9: 11.6 us, 13.0 with two cuts one after the other)
      least = find_few<LOW>(cl, sm, w, run, j0, (unsigned)k, top_p, min_p, &sum);
      summed = true;
    } else {
      if (inside) {
        least = find_key<LOW>(cl, sm, w, run, j0, 0, false, (u64)k, min_p, &mass, by_p ? nullptr : &sum);
        summed = !by_p;
      }
      if (by_p) {
        if (tid == 0) sm.wanted = (u64)max(share_of(top_p, mass), 1LL);
        __syncthreads();
        const u64 want = sm.wanted;
        bins.find(sm, true, want);
        least = find_key<LOW>(cl, sm, w, run, j0, 1, true, want, min_p, &mass, &sum);
        summed = true;
      }
    }
    if (!summed) {  // fewer than k tokens with a weight
      Mass kept;
      for (int i = i0; i < i1; ++i) kept.add(w[i] < min_p ? 0.f : w[i]);
      sum = kept.value();
    }
  }
  // the kept weights in the order of the indices
  const unsigned least_w = (unsigned)(least >> kIndexBits);
  const int last_j = (1 << kIndexBits) - 1 - (int)(least & ((1 << kIndexBits) - 1));
  auto weight = [&](int i) -> u64 {
    const unsigned bits = __float_as_uint(w[i]);
    const bool in = bits > least_w || (bits == least_w && j0 + i <= last_j);
    return in && !(w[i] < min_p) ? fixed_of(w[i]) : 0;
  };
  u64 before = sum;
  unsigned none = 0;
  block_scan(sm, none, before);
  if (tid == kThreads - 1) sm.total = before + sum;
  __syncthreads();
  if (tid < C) cl.map_shared_rank(&sm, tid)->kept[rank] = sm.total;
  cl.sync();  // (the last access to another CTA's shared memory)
  u64 total = 0;
  for (int r = 0; r < C; ++r) {
    if (r < rank) before += sm.kept[r];
    total += sm.kept[r];
  }
  if (tid == 0) sm.wanted = (u64)min(share_of(u, total), (long long)total - 1);
  __syncthreads();
  const u64 target = sm.wanted;
  const unsigned hit = __ballot_sync(0xffffffffu, before <= target && target < before + sum);
  if (!hit) return;
  // the warp goes through the run that was hit
  const int owner = __ffs(hit) - 1, stop = __shfl_sync(0xffffffffu, i1, owner);
  before = __shfl_sync(0xffffffffu, before, owner);
  for (int i = __shfl_sync(0xffffffffu, i0, owner); i < stop; i += 32) {
    const u64 own = i + lane < stop ? weight(i + lane) : 0;
    u64 upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 t = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += t;
    }
    if (before + upto - own <= target && target < before + upto) {
      const float log_sum = logf(__fmul_rn((float)(long long)total, 1.f / 1099511627776.f));
      p.token[row] = j0 + i + lane;
      p.logprob[row] = logf(w[i + lane]) - log_sum;
      p.logz[row] = __fadd_rn(__fmul_rn(M, scale), log_sum);
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
    if (before > target) break;
  }
}

template <typename TI, int LOW>
cudaError_t launch_low(const SampleProblem& p, int cluster, int slice, cudaStream_t s) {
  // The limit is the kernel's, for every host thread: set to the longest slice's need, whatever this call
  // launches with (a limit by the call could be lowered by another thread before the launch).
  constexpr int fixed = ((int)sizeof(Smem<LOW>) + 15) / 16 * 16;
  constexpr int longest = fixed + ((LOW == low_bits(true) ? kMaxSlice : kShort) + 4) * (int)sizeof(float);
  static_assert(longest <= 227 * 1024, "shared memory of a CTA");
  const int smem = fixed + (slice + 4) * (int)sizeof(float);
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<TI, LOW>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, longest);
  if (e != cudaSuccess) { note_failure("sample: shared memory"); return e; }
  e = launch_pdl(sample_kernel<TI, LOW>, dim3((unsigned)p.R * cluster), kThreads, smem, s, cluster, p,
                 slice);
  if (e != cudaSuccess) note_failure("sample: launch");
  return e;
}

template <typename TI>
cudaError_t launch_t(const SampleProblem& p, cudaStream_t s) {
  // As many CTAs per row as the GPU holds at once over all rows (two per SM), but 4096 tokens each and
  // no more than kShort, where there is a choice: what a CTA waits for its cluster costs the same
  // whatever its slice, so that longer slices in one round beat shorter ones in two (64 rows of 50257:
  // 35 us with 8 CTAs a row, 27 with 4).  (Of slices past kShort one CTA fits an SM; they come with
  // the largest cluster whatever fits.)
  int dev = 0, nsm = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
    note_failure("sample: device attributes");
    return e;
  }
  auto up = [](int a, int b) { return (a + b - 1) / b; };
  const int fit = 2 * nsm / p.R, need = up(p.V, kShort - 8), most = up(p.V, 4096);
  int cluster = fit < need ? need : fit;
  cluster = cluster < most ? cluster : most;
  cluster = cluster < 1 ? 1 : cluster < kMaxCluster ? cluster : kMaxCluster;
  const int slice = ((p.V + cluster - 1) / cluster + 7) / 8 * 8;
  if (slice <= kShort) return launch_low<TI, low_bits(false)>(p, cluster, slice, s);
  return launch_low<TI, low_bits(true)>(p, cluster, slice, s);
}

}  // namespace sample

int sample_max_vocabulary() { return sample::kMaxCluster * sample::kMaxSlice; }

cudaError_t launch_sample(const SampleProblem& p, cudaStream_t s) {
  if (p.dtype == RELATION_F32) return sample::launch_t<float>(p, s);
  return sample::launch_t<__nv_bfloat16>(p, s);
}

}  // namespace rel
