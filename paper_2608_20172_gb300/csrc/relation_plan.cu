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
// CTAs: each repeats the scans over all requests (kThreads at a time, in shared memory) and takes
// its share of the tokens, new pages and returned pages, finding a token's request by bisection in
// the scanned sums.
#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace plan {

constexpr int kThreads = 512;
constexpr int kPerThread = 4;  // tokens per thread that another CTA is started for

// Exclusive block sum; *total = the sum over the block.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long x,
                                                         unsigned long long* part,
                                                         unsigned long long* total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned long long s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += t;
  }
  __syncthreads();  // part is free
  if (lane == 31) part[warp] = s;
  __syncthreads();
  unsigned long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const unsigned long long t = part[w];
    if (w < warp) before += t;
    all += t;
  }
  *total = all;
  return before + s - x;
}

// A chunk's requests
struct Chunk {
  int end[kThreads];          // tokens up to and with the request (at most 2^31 - 1)
  int need_end[kThreads];     // new pages up to and with it
  int given_end[kThreads];    // returned pages
  int start[kThreads], length[kThreads];
  int need0[kThreads], given0[kThreads];
  bool served[kThreads];
};

// The first request of the chunk whose running sum exceeds x.
__device__ __forceinline__ int owner_of(const int* end, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (end[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) plan_kernel(PlanProblem p) {
  __shared__ Chunk ch;
  __shared__ unsigned long long part[kThreads / 32];
  __shared__ int taken_s;
  const int tid = threadIdx.x, stride = (int)gridDim.x * kThreads;
  const int first = (int)blockIdx.x * kThreads + tid;
  const bool lead = blockIdx.x == 0;
  const long long cap = (long long)p.cols * p.page;  // rows of a table row
  if (tid == 0) taken_s = 0;
  pdl_wait_and_launch();
  int head = p.state[0], avail = p.state[1];
  if (head < 0 || head >= p.n_pages || avail < 0 || avail > p.n_pages) {
    if (lead && tid == 0 && p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    head = avail = 0;
  }
  long long tokens = 0;       // of the requests before this chunk,
  int needed = 0, given = 0;  // their new pages and returned pages
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid, n = min(kThreads, p.B - b0);
    const int L = b < p.B ? p.lengths[b] : 0, c = b < p.B ? p.counts[b] : 0;
    const bool valid = L >= 0 && L <= cap;
    const int fresh = max(c, 0);
    unsigned long long all_tokens, all_pages;
    const long long start = tokens + (long long)block_scan(fresh, part, &all_tokens);
    const long long end = start + fresh;
    const int held = valid ? L / p.page + (L % p.page != 0) : 0;
    const bool fits = valid && c >= 0 && L + (long long)fresh <= cap && end <= p.n_tokens;
    const long long want = (L + (long long)fresh + p.page - 1) / p.page;
    const int need = fits ? (int)want - held : 0;
    const int back = c < 0 && b < p.B ? held : 0;
    const unsigned long long both =
        block_scan((unsigned)need | (unsigned long long)(unsigned)back << 32, part, &all_pages);
    const int need0 = needed + (int)(both & 0xffffffffu), given0 = given + (int)(both >> 32);
    const bool served = fits && (need == 0 || need0 + need <= avail);
    ch.start[tid] = (int)min(start, 0x7fffffffLL);
    ch.end[tid] = (int)min(end, 0x7fffffffLL);
    ch.length[tid] = L;
    ch.need0[tid] = need0;
    ch.need_end[tid] = need0 + need;
    ch.given0[tid] = given0;
    ch.given_end[tid] = given0 + back;
    ch.served[tid] = served;
    if (lead && b < p.B) {
      p.starts[b] = ch.start[tid];
      if (b == p.B - 1) p.starts[p.B] = ch.end[tid];
      p.lengths_out[b] = c < 0 && valid ? 0 : served ? L + fresh : L;
      if (need0 + need <= avail) atomicMax(&taken_s, need0 + need);
      if (p.dev_status) {
        if (!valid) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
        else if (c > 0 && !served)
          atomicCAS(p.dev_status, (int)RELATION_OK, (int)RELATION_ERR_CAPACITY);
      }
    }
    __syncthreads();
    // tokens [tokens, tokens + all_tokens) of the buffer
    const long long t1 = min(tokens + (long long)all_tokens, (long long)p.n_tokens);
    for (long long t = tokens + first; t < t1; t += stride) {
      const int i = owner_of(ch.end, n, (int)t);
      long long slot = -1;
      int pos = -1;
      if (ch.served[i]) {
        const int len = ch.length[i];
        pos = len + (int)t - ch.start[i];
        const int j = pos / p.page, old = len / p.page + (len % p.page != 0);
        const int id = j < old ? p.table[(long long)(b0 + i) * p.t_stride + j]
                               : p.ring[((long long)head + ch.need0[i] + j - old) % p.n_pages];
        slot = (long long)id * p.page + pos % p.page;
      }
      p.slots[t] = slot;
      p.positions[t] = pos;
    }
    // new pages into the tables
    const int new_end = needed + (int)(all_pages & 0xffffffffu);
    for (long long m = (long long)needed + first; m < new_end; m += stride) {
      const int i = owner_of(ch.need_end, n, (int)m);
      if (!ch.served[i]) continue;
      const int len = ch.length[i], old = len / p.page + (len % p.page != 0);
      p.table[(long long)(b0 + i) * p.t_stride + old + ((int)m - ch.need0[i])] =
          p.ring[((long long)head + m) % p.n_pages];
    }
    // pages of ended requests into the ring
    const int given_end = given + (int)(all_pages >> 32);
    for (long long m = (long long)given + first; m < given_end; m += stride) {
      if (avail + m >= p.n_pages) break;  // more pages than there are (reported below)
      const int i = owner_of(ch.given_end, n, (int)m);
      p.ring[((long long)head + avail + m) % p.n_pages] =
          p.table[(long long)(b0 + i) * p.t_stride + ((int)m - ch.given0[i])];
    }
    tokens += (long long)all_tokens;
    needed = new_end;
    given = given_end;
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
    p.state_out[0] = (int)(((long long)head + taken) % p.n_pages);
    p.state_out[1] = (int)count;
  }
}

}  // namespace plan

cudaError_t launch_plan(const PlanProblem& p, cudaStream_t s) {
  int dev = 0, nsm = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
    note_failure("page plan: device attributes");
    return e;
  }
  const int per = plan::kThreads * plan::kPerThread;
  const int want = p.n_tokens / per + (p.n_tokens % per != 0);
  e = launch_pdl(plan::plan_kernel, dim3((unsigned)(want < nsm ? want : nsm)), plan::kThreads, 0, s,
                 1, p);
  if (e != cudaSuccess) note_failure("page plan: launch");
  return e;
}

}  // namespace rel
