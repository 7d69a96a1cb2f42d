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
// logits are read once.  The cuts are found by a radix search over the composite key (w_j, index),
// which no two tokens share: per digit a histogram of counts and masses of the tokens that agree with
// the digits found so far, summed over the cluster through distributed shared memory.
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
constexpr int kMaxSlice = 40 * 1024;  // tokens of a CTA (with Smem 221 of its 227 KB)
constexpr int kIndexBits = 22;        // of the composite key: 30 bits of w, then the index
constexpr int kKeyBits = 30 + kIndexBits;
constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int kSlots = 3;             // a mass in 14-bit parts, whose sums stay below 2^32

struct Smem {
  unsigned hist[1 + kSlots][kBins];  // this CTA's: counts, parts of the masses
  unsigned count[kBins];             // the cluster's
  u64 mass[kBins];
  u64 scan[2][kWarps];
  u64 warp_sum[kWarps], total;
  float red[kWarps];
  float max;
  int nan;
  u64 above_count, above_mass;       // of the digit that was found,
  unsigned digit;                    // and the digit
};

__device__ __forceinline__ u64 fixed_of(float w) {
  return __float2ull_rz(w * 1099511627776.f);  // 2^40 w: the product is exact
}
__device__ __forceinline__ u64 key_of(float w, int j) {
  return (u64)__float_as_uint(w) << kIndexBits | (u64)((1 << kIndexBits) - 1 - j);
}

__device__ __forceinline__ u64 warp_sum(u64 x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The digit at `shift` of the boundary's key among this row's tokens with key >= least whose higher
// digits are `prefix`: the boundary is the first token in descending order at which the running
// count (by_mass: mass), beginning with `above`, reaches `want`.
__device__ __forceinline__ void find_digit(cg::cluster_group& cl, Smem& sm, const float* w, int n,
                                           int j0, u64 least, u64 prefix, int shift, int bits,
                                           bool by_mass, u64 want, u64 above_count,
                                           u64 above_mass) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int i = tid; i < (1 + kSlots) * kBins; i += kThreads) (&sm.hist[0][0])[i] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kThreads) {
    const float x = w[i];
    const u64 key = key_of(x, j0 + i);
    if (key < least || key >> (shift + bits) != prefix) continue;
    const unsigned d = (unsigned)(key >> shift) & ((1u << bits) - 1);
    const u64 q = fixed_of(x);
    atomicAdd(&sm.hist[0][d], 1u);
    atomicAdd(&sm.hist[1][d], (unsigned)q & 0x3fff);
    atomicAdd(&sm.hist[2][d], (unsigned)(q >> 14) & 0x3fff);
    atomicAdd(&sm.hist[3][d], (unsigned)(q >> 28));
  }
  cl.sync();
  // each CTA adds up its share of the bins and hands them to all
  const int C = (int)cl.num_blocks(), share = kBins / C, b0 = (int)cl.block_rank() * share;
  for (int i = tid; i < share; i += kThreads) {
    unsigned c = 0;
    u64 m = 0;
    for (int r = 0; r < C; ++r) {
      const Smem* o = cl.map_shared_rank(&sm, r);
      c += o->hist[0][b0 + i];
      m += (u64)o->hist[1][b0 + i] + ((u64)o->hist[2][b0 + i] << 14) + ((u64)o->hist[3][b0 + i] << 28);
    }
    for (int r = 0; r < C; ++r) {
      Smem* o = cl.map_shared_rank(&sm, r);
      o->count[b0 + i] = c;
      o->mass[b0 + i] = m;
    }
  }
  cl.sync();
  // from the highest bin down: thread t holds bins kBins - 1 - t per .. 
  constexpr int per = kBins / kThreads;
  u64 c = 0, m = 0;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const int d = kBins - 1 - (tid * per + i);
    c += sm.count[d];
    m += sm.mass[d];
  }
  u64 cs = c, ms = m;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 a = __shfl_up_sync(0xffffffffu, cs, o), b = __shfl_up_sync(0xffffffffu, ms, o);
    if (lane >= o) {
      cs += a;
      ms += b;
    }
  }
  if (lane == 31) {
    sm.scan[0][warp] = cs;
    sm.scan[1][warp] = ms;
  }
  __syncthreads();
  u64 ca = above_count + cs - c, ma = above_mass + ms - m;  // above this thread's bins
  for (int i = 0; i < warp; ++i) {
    ca += sm.scan[0][i];
    ma += sm.scan[1][i];
  }
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const int d = kBins - 1 - (tid * per + i);
    const u64 before = by_mass ? ma : ca, own = by_mass ? sm.mass[d] : sm.count[d];
    if (before < want && want <= before + own) {
      sm.digit = d;
      sm.above_count = ca;
      sm.above_mass = ma;
    }
    ca += sm.count[d];
    ma += sm.mass[d];
  }
  __syncthreads();
}

// The boundary's key; *mass = the sum of the weights down to and with it.
__device__ __forceinline__ u64 find_key(cg::cluster_group& cl, Smem& sm, const float* w, int n,
                                        int j0, u64 least, bool by_mass, u64 want, u64* mass) {
  u64 prefix = 0, above_count = 0, above_mass = 0;
  int shift = kKeyBits;
  while (shift > 0) {
    const int bits = min(kDigit, shift);
    shift -= bits;
    find_digit(cl, sm, w, n, j0, least, prefix, shift, bits, by_mass, want, above_count, above_mass);
    prefix = prefix << bits | sm.digit;
    above_count = sm.above_count;
    above_mass = sm.above_mass;
  }
  *mass = above_mass + sm.mass[sm.digit];
  return prefix;
}

template <typename TI>
__device__ __forceinline__ float value(const TI* p) {
  return (float)*p;
}

template <typename TI>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleProblem p, int slice) {
  extern __shared__ __align__(16) unsigned char raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  float* w = reinterpret_cast<float*>(raw + sizeof(Smem));
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int row = (int)blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int j0 = min(p.V, rank * slice), n = min(slice, p.V - j0);
  pdl_wait_and_launch();
  const float temperature = p.temperature ? p.temperature[row] : 1.f, u = p.u[row];
  const bool greedy = temperature == 0.f;
  const float scale = greedy ? 1.f : __fdiv_rn(1.f, temperature);
  int k = greedy ? 1 : p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f;
  const float min_p = p.min_p ? fminf(p.min_p[row], 1.f) : 0.f;
  const bool valid = temperature >= 0.f && temperature < INFINITY && u >= 0.f && u <= 1.f;
  // the slice, and the row's largest logit
  const TI* x = reinterpret_cast<const TI*>(p.logits) + (long long)row * p.s_row + j0;
  float mx = -INFINITY;
  bool bad = false;
  for (int i = tid; i < n; i += kThreads) {
    const float v = value(x + i);
    w[i] = v;
    mx = fmaxf(mx, v);
    bad |= v != v;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  if (lane == 0) sm.red[warp] = mx;
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    for (int i = 1; i < kWarps; ++i) mx = fmaxf(mx, sm.red[i]);
    sm.max = mx;
    sm.nan = bad;
  }
  cl.sync();
  float M = -INFINITY;
  bool nan = false;
  for (int r = 0; r < C; ++r) {
    const Smem* o = cl.map_shared_rank(&sm, r);
    M = fmaxf(M, o->max);
    nan |= o->nan != 0;
  }
  if (!valid || nan || M == -INFINITY) {  // (the same in every CTA of the cluster)
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      p.logprob[row] = valid && !nan ? -INFINITY : NAN;
      p.logz[row] = valid && !nan ? -INFINITY : NAN;
      if (!valid && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    }
    cl.sync();  // sm.max has been read
    return;
  }
  for (int i = tid; i < n; i += kThreads) {
    const float v = w[i];
    w[i] = v == M ? 1.f : greedy ? 0.f : expf(__fmul_rn(__fsub_rn(v, M), scale));
  }
  __syncthreads();
  u64 least = 0, mass = ~0ull;
  if (k > 0 && k < p.V) least = find_key(cl, sm, w, n, j0, 0, false, (u64)k, &mass);
  if (top_p < 1.f) {
    if (mass == ~0ull) {  // of all tokens
      u64 s = 0;
      for (int i = tid; i < n; i += kThreads) s += fixed_of(w[i]);
      s = warp_sum(s);
      if (lane == 0) sm.warp_sum[warp] = s;
      __syncthreads();
      if (tid == 0) {
        for (int i = 1; i < kWarps; ++i) s += sm.warp_sum[i];
        sm.total = s;
      }
      cl.sync();
      mass = 0;
      for (int r = 0; r < C; ++r) mass += cl.map_shared_rank(&sm, r)->total;
      cl.sync();  // sm.total has been read
    }
    const long long want = (long long)floor((double)top_p * (double)(long long)mass);
    least = find_key(cl, sm, w, n, j0, least, true, (u64)max(want, 1LL), &mass);
  }
  // kept weights of every warp's stretch, then of every CTA
  const int seg = (slice / kWarps + 31) / 32 * 32 + 32, i0 = min(n, warp * seg), i1 = min(n, i0 + seg);
  auto weight = [&](int i) -> u64 {
    const float v = w[i];
    return key_of(v, j0 + i) >= least && !(v < min_p) ? fixed_of(v) : 0;
  };
  u64 s = 0;
  for (int i = i0 + lane; i < i1; i += 32) s += weight(i);
  s = warp_sum(s);
  if (lane == 0) sm.warp_sum[warp] = s;
  __syncthreads();
  if (tid == 0) {
    u64 t = 0;
    for (int i = 0; i < kWarps; ++i) t += sm.warp_sum[i];
    sm.total = t;
  }
  cl.sync();
  u64 total = 0, before = 0;
  for (int r = 0; r < C; ++r) {
    const u64 t = cl.map_shared_rank(&sm, r)->total;
    if (r < rank) before += t;
    total += t;
  }
  const u64 target =
      (u64)min((long long)floor((double)u * (double)(long long)total), (long long)total - 1);
  for (int i = 0; i < warp; ++i) before += sm.warp_sum[i];
  if (before <= target && target < before + s) {  // this warp's stretch
    for (int i = i0; i < i1; i += 32) {
      const u64 own = i + lane < i1 ? weight(i + lane) : 0;
      u64 run = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += t;
      }
      if (before + run - own <= target && target < before + run) {
        const float sum = logf(__fmul_rn((float)(long long)total, 1.f / 1099511627776.f));
        p.token[row] = j0 + i + lane;
        p.logprob[row] = logf(w[i + lane]) - sum;
        p.logz[row] = __fadd_rn(__fmul_rn(M, scale), sum);
      }
      before += __shfl_sync(0xffffffffu, run, 31);
      if (before > target) break;
    }
  }
  cl.sync();  // the other CTAs' shared memory has been read
}

template <typename TI>
cudaError_t launch_t(const SampleProblem& p, cudaStream_t s) {
  int cluster = 1;  // at least 4096 tokens per CTA
  while (cluster < kMaxCluster && p.V > 4096 * cluster) cluster *= 2;
  const int slice = (p.V / cluster + 7) / 8 * 8 + 8;
  const int smem = (int)sizeof(Smem) + slice * (int)sizeof(float);
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<TI>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       smem);
  if (e != cudaSuccess) { note_failure("sample: shared memory"); return e; }
  e = launch_pdl(sample_kernel<TI>, dim3((unsigned)p.R * cluster), kThreads, smem, s, cluster, p, slice);
  if (e != cudaSuccess) note_failure("sample: launch");
  return e;
}

}  // namespace sample

int sample_max_vocabulary() { return sample::kMaxCluster * (sample::kMaxSlice - 16); }

cudaError_t launch_sample(const SampleProblem& p, cudaStream_t s) {
  if (p.dtype == RELATION_F32) return sample::launch_t<float>(p, s);
  return sample::launch_t<__nv_bfloat16>(p, s);
}

}  // namespace rel
