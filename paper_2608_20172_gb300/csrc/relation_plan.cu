// relation_plan.cu -- block tables, slots and positions of one serving step, from the requests'
// lengths and counts, on the GPU.
//
// Request b holds L_b rows in ceil(L_b / page) pages and brings c_b new tokens (c_b < 0: it has
// ended).  With need_b = ceil((L_b + c_b) / page) - ceil(L_b / page) and given_b = ceil(L_b / page)
// of an ended request,
//   starts_b = sum_{a < b} max(c_a, 0)          (exclusive sums over the requests)
//   N_b = sum_{a < b} need_a,  G_b = sum_{a < b} given_a
// the j-th new page of b is entry head + N_b + j of the ring of free pages, the j-th page of an
// ended b becomes entry head + count + G_b + j, and token t of b goes to position
// L_b + t - starts_b, whose slot is its page's id times the page size plus its row.
//
// Bound by latency: a step's output is a few bytes per token.  One launch and no dependence between
// CTAs: each repeats the scans over all requests, a thread for one of 512 or for four of 2048 at a
// time, and takes its share of the tokens, new pages and returned pages, finding a token's request by
// bisection in the scanned sums.  One call after the other in a graph, a step of 64 requests takes
// 6.1 us (7.1 with four requests to a thread), 131072 tokens of 2048 requests 9.4 us (18.6 with 512
// requests at a time, a token at a time and divisions by the page size and the number of pages).
#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace plan {

constexpr int kThreads = 512;
constexpr int kPerThread = 4;  // tokens of a thread, at once

struct Sums {
  unsigned long long a, b;
};
// Exclusive block sums of two numbers; *all = the sums over the block.
__device__ __forceinline__ Sums block_scan(Sums x, Sums* part, Sums* all) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Sums s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long a = __shfl_up_sync(0xffffffffu, s.a, o);
    const unsigned long long b = __shfl_up_sync(0xffffffffu, s.b, o);
    if (lane >= o) {
      s.a += a;
      s.b += b;
    }
  }
  __syncthreads();  // part is free
  if (lane == 31) part[warp] = s;
  __syncthreads();
  Sums before{0, 0}, t{0, 0};
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const Sums y = part[w];
    if (w < warp) {
      before.a += y.a;
      before.b += y.b;
    }
    t.a += y.a;
    t.b += y.b;
  }
  *all = t;
  return {before.a + s.a - x.a, before.b + s.b - x.b};
}

// A chunk's requests.  Request i's tokens are end[i - 1] .. end[i] - 1 (from 0 below the chunk's
// first), and likewise its pages.
template <int EACH>  // requests of a thread
struct Chunk {
  static constexpr int kChunk = EACH * kThreads;
  int end_[kChunk + 1];    // running sums of the tokens (at most 2^31 - 1),
  int need_[kChunk + 1];   // of the new pages
  int given_[kChunk + 1];  // and of the returned ones, each after the sum before the chunk
  int length[kChunk];      // rows; -1 where the request is not served
};

// The first request of the chunk whose running sum exceeds x, for kPerThread numbers at once.
template <int K>
__device__ __forceinline__ void owners_of(const int* end, int n, const int (&x)[K], int (&lo)[K]) {
  int hi[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    lo[k] = 0;
    hi[k] = n - 1;
  }
  for (int step = n; step > 1; step = (step + 1) >> 1) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int mid = (lo[k] + hi[k]) >> 1;
      const bool left = lo[k] >= hi[k] || end[mid] > x[k];
      hi[k] = left ? mid : hi[k];
      lo[k] = left ? lo[k] : mid + 1;
    }
  }
}

template <int EACH>
__global__ void __launch_bounds__(kThreads) plan_kernel(PlanProblem p) {
  constexpr int kEach = EACH, kChunk = Chunk<EACH>::kChunk;
  __shared__ Chunk<EACH> ch;
  __shared__ Sums part[kThreads / 32];
  __shared__ int taken_s;
  const int tid = threadIdx.x, stride = (int)gridDim.x * kThreads;
  const int first = (int)blockIdx.x * kThreads + tid;
  const bool lead = blockIdx.x == 0;
  const long long cap = (long long)p.cols * p.page;  // rows of a table row
  if (tid == 0) taken_s = 0;
  auto pages_of = [&](int rows) {  // ceil(rows / page)
    const int j = page_of(rows, p.page, p.page_mul, p.page_shift);
    return j + (rows > j * p.page);
  };
  pdl_wait_and_launch();
  int head = p.state[0], avail = p.state[1];
  if (head < 0 || head >= p.n_pages || avail < 0 || avail > p.n_pages) {
    if (lead && tid == 0 && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    head = avail = 0;
  }
  auto ring_at = [&](unsigned i) {  // entry head + i, i <= n_pages
    const unsigned j = (unsigned)head + i;
    return j >= (unsigned)p.n_pages ? j - (unsigned)p.n_pages : j;
  };
  long long tokens = 0;       // of the requests before this chunk,
  int needed = 0, given = 0;  // their new pages and returned pages
  for (int b0 = 0; b0 < p.B; b0 += kChunk) {
    const int n = min(kChunk, p.B - b0), i0 = tid * kEach;
    int L[kEach], c[kEach];
    unsigned long long mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool in = i0 + i < n;
      L[i] = in ? p.lengths[b0 + i0 + i] : 0;
      c[i] = in ? p.counts[b0 + i0 + i] : 0;
      mine += (unsigned)max(c[i], 0);
    }
    Sums all;
    long long start = tokens + (long long)block_scan({mine, 0}, part, &all).a;
    const long long all_tokens = (long long)all.a;
    if (tid == 0) {
      ch.end_[0] = (int)min(tokens, 0x7fffffffLL);
      ch.need_[0] = needed;
      ch.given_[0] = given;
    }
    int need[kEach], back[kEach];
    bool fits[kEach];
    Sums pages{0, 0};
    long long at = start;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int fresh = max(c[i], 0);
      const bool valid = L[i] >= 0 && L[i] <= cap;
      const int held = valid ? pages_of(L[i]) : 0;
      at += fresh;
      fits[i] = valid && c[i] >= 0 && L[i] + (long long)fresh <= cap && at <= p.n_tokens;
      need[i] = fits[i] ? pages_of(L[i] + fresh) - held : 0;
      back[i] = c[i] < 0 ? held : 0;
      pages.a += (unsigned)need[i];
      pages.b += (unsigned)back[i];
    }
    const Sums before = block_scan(pages, part, &all);
    int need_end = needed + (int)before.a, given_end = given + (int)before.b;
    at = start;
    int taken = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int fresh = max(c[i], 0);
      const bool valid = L[i] >= 0 && L[i] <= cap;
      need_end += need[i];
      given_end += back[i];
      const bool served = fits[i] && (need[i] == 0 || need_end <= avail);
      const int from = (int)min(at, 0x7fffffffLL);
      at += fresh;
      const int to = (int)min(at, 0x7fffffffLL), k = i0 + i;
      ch.end_[k + 1] = to;
      ch.need_[k + 1] = need_end;
      ch.given_[k + 1] = given_end;
      ch.length[k] = served || c[i] < 0 ? L[i] : -1;
      if (lead && k < n) {
        const int b = b0 + k;
        p.starts[b] = from;
        if (b == p.B - 1) p.starts[p.B] = to;
        p.lengths_out[b] = c[i] < 0 && valid ? 0 : served ? L[i] + fresh : L[i];
        if (need_end <= avail) taken = need_end;
        if (p.dev_status) {
          if (!valid) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
          else if (c[i] > 0 && !served)
            atomicCAS(p.dev_status, (int)RELATION_OK, (int)RELATION_ERR_CAPACITY);
        }
      }
    }
    if (lead && taken) atomicMax(&taken_s, taken);
    __syncthreads();
    // tokens [tokens, tokens + all_tokens) of the buffer
    const int t1 = (int)min(tokens + all_tokens, (long long)p.n_tokens);
    for (long long tb = tokens + first; tb < t1; tb += (long long)kPerThread * stride) {
      int t[kPerThread], i[kPerThread], pos[kPerThread], id[kPerThread];
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) t[k] = (int)min(tb + (long long)k * stride, (long long)t1 - 1);
      owners_of(ch.end_ + 1, n, t, i);
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) {
        const int len = ch.length[i[k]];
        pos[k] = len < 0 ? -1 : len + t[k] - ch.end_[i[k]];
        id[k] = 0;
        if (len >= 0) {
          const int j = page_of(pos[k], p.page, p.page_mul, p.page_shift), old = pages_of(len);
          id[k] = j < old ? p.table[(long long)(b0 + i[k]) * p.t_stride + j]
                          : p.ring[ring_at((unsigned)(ch.need_[i[k]] + j - old))];
        }
      }
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) {
        if (tb + (long long)k * stride >= t1) break;
        const int row = pos[k] - page_of(max(pos[k], 0), p.page, p.page_mul, p.page_shift) * p.page;
        p.slots[t[k]] = pos[k] < 0 ? -1 : (long long)id[k] * p.page + row;
        p.positions[t[k]] = pos[k];
      }
    }
    // new pages into the tables
    const int need_all = needed + (int)all.a, given_all = given + (int)all.b;
    for (long long m = (long long)needed + first; m < min(need_all, avail); m += stride) {
      int i[1];
      owners_of(ch.need_ + 1, n, {(int)m}, i);
      const int len = ch.length[i[0]];
      if (len < 0) continue;
      p.table[(long long)(b0 + i[0]) * p.t_stride + pages_of(len) + ((int)m - ch.need_[i[0]])] =
          p.ring[ring_at((unsigned)m)];
    }
    // pages of ended requests into the ring (more than there are: dropped, and reported below)
    for (long long m = (long long)given + first; m < min(given_all, p.n_pages - avail); m += stride) {
      int i[1];
      owners_of(ch.given_ + 1, n, {(int)m}, i);
      p.ring[ring_at((unsigned)(avail + m))] =
          p.table[(long long)(b0 + i[0]) * p.t_stride + ((int)m - ch.given_[i[0]])];
    }
    tokens += all_tokens;
    needed = need_all;
    given = given_all;
    __syncthreads();  // the chunk is written again
  }
  for (long long t = tokens + first; t < p.n_tokens; t += stride) {
    p.slots[t] = -1;
    p.positions[t] = -1;
  }
  if (lead && tid == 0) {
    const int taken = taken_s;
    long long count = (long long)avail - taken + given;
    if ((long long)avail + given > p.n_pages) {
      if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
      count = p.n_pages - taken;
    }
    p.state_out[0] = (int)ring_at((unsigned)taken);
    p.state_out[1] = (int)count;
  }
}

}  // namespace plan

cudaError_t launch_plan(PlanProblem p, cudaStream_t s) {
  page_division(p.page, &p.page_mul, &p.page_shift);
  int dev = 0, nsm = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
    note_failure("page plan: device attributes");
    return e;
  }
  const int per = plan::kThreads * plan::kPerThread;
  const int want = p.n_tokens / per + (p.n_tokens % per != 0);
  const dim3 grid((unsigned)(want < nsm ? want : nsm));
  e = p.B <= plan::kThreads ? launch_pdl(plan::plan_kernel<1>, grid, plan::kThreads, 0, s, 1, p)
                            : launch_pdl(plan::plan_kernel<4>, grid, plan::kThreads, 0, s, 1, p);
  if (e != cudaSuccess) note_failure("page plan: launch");
  return e;
}

}  // namespace rel
