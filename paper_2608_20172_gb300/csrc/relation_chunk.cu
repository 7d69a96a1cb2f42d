// relation_chunk.cu -- the Relation rows of several new tokens per request over a paged key/value cache.
//
// A token at zero-based position p of request b, against rows 0 .. p of the request (row r in page
// table[b][r / page_size]), as in relation_paged.cu:
//   E_j = SiLU(q . k_j / sqrt(d)) for j < p,  L^E = log sum_j e^{E_j},  S = sigmoid(q . k_p / (sqrt(d) tau_S)),
//   A = L^E - lambda log(p + 1),  g = sigmoid(A - S),
//   Y = (1 - g) v_p + g sum_j e^{E_j} v_j / sum_j e^{E_j},  logZ = logaddexp(S, A).
// G = H / H_kv query heads share a key/value head.
//
// A tile is 128 (fp32: 64) (token, query head of one key head) pairs of a request, token-major: shared heads and
// short chunks fill it together.  The host knows neither counts nor positions, so a first small kernel lays
// out the work: the tiles of all requests, each cut along its keys into pieces of the mean length of as many
// pieces as CTAs fit the GPU and a rest, which is started last, in an order that keeps the tiles of a request's head side by
// side (they read the same keys) with the longest first, the requests with the longest history before the
// others.  A tile of one piece is finished by its CTA; of others every piece leaves its rows' (m, l, z), which a last kernel joins.
//
// bf16: the tensor-core forward's scan (relation_tc_fwd.cu, scan.cuh) with keys and values fetched from
// their pages by TMA, a box of rows that lie in one page at a time (cp.async, row by row, for pages whose
// size is no multiple of 8).  fp32: register tiles on the CUDA cores.
//
// Bound by the hand-off between scan and products (tensor cores 33 %, special functions 49 % busy).
// Measured: 4 pieces of prompts, 6933 tokens of 16 x 128 bf16 that see 8970 rows on average, 620 us, 0.82
// PFLOP/s; 48 requests, half of them decoding, 6174 tokens of 32 query heads over 8 x 80 that see 2094 rows in
// pages of 24, 390 us (of 64 354); 5 tokens behind 2048 rows of 12 x 64 16 us, dependent trips; fp32, 451
// tokens of 8 query heads over 4 x 72 43 us, 3646 tokens of 8 x 128 that see 4764 rows 2.12 ms, 33 TFLOP/s.
#include <cudaTypedefs.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "scan.cuh"

namespace rel {
namespace chunk {

constexpr int kUnit = 64;  // keys that are loaded together; pieces are made of them
constexpr int kPlanThreads = 1024;
constexpr int kJoinRows = 8;  // rows of a tile that the last kernel joins together
constexpr int kSorted = 512;  // requests that the plan brings into an order of its own

// The workspace: what the plan says, and the pieces' partial results.
struct alignas(16) Item {  // a CTA's work: a piece of a tile for one key head
  int b, s0, row0, rows;   // request, its first token, the tile's first row within it, the tile's rows
  int head, u0, u1, slot;  // units u0 .. u1 - 1; slot: of the partial result, -1: the tile's only piece
};
constexpr int kToTheEnd = 0x7fffffff;  // u1 of a tile's last piece
struct alignas(16) Split {  // a tile of several pieces
  int b, s0, row0, rows, pieces, slot, pad0, pad1;  // slot: the first key head's first
};
struct Plan {
  int* head;     // {items, tiles of several pieces, the most row groups (kJoinRows) that one of these has}
  int* first;    // [B + 1] first tile of a request, in the plan's order
  int4* tiles;   // [max_tiles] request in that order, first row, pieces (twice, and whether the last is a
                 // rest), units of keys and then the first slot
  int2* upto;    // [max_tiles + 1] pieces before a tile: all but the rests, the rests
  Split* split;  // [max_split]
  Item* items;   // [max_items]
  float4* stats; // [slots][rows] m, l, self evidence, whether the piece has it
  float* z;      // [slots][rows][width]
  int max_tiles, max_items, max_split, slots, rows, width;
  int tile, target, least;  // rows of a tile; pieces aimed at; units that a piece has at least
  int small;                // every CTA lays the work out by itself (few requests and tiles)
};

// Request b's tokens, as far as the buffer holds them
__device__ __forceinline__ int2 tokens_of(const ChunkProblem& p, int b) {
  const int s0 = min(max(p.starts[b], 0), p.N), s1 = min(max(p.starts[b + 1], s0), p.N);
  return make_int2(s0, s1);
}
__device__ __forceinline__ int tiles_of(int2 tokens, int G, int tile) {  // (a power of two)
  return (int)(((long long)(tokens.y - tokens.x) * G + tile - 1) >> (31 - __clz(tile)));
}
// Units of keys that a tile's last row sees, which is the most where positions ascend
__device__ __forceinline__ int units_of(const ChunkProblem& p, int2 tokens, int row0, int G, int tile) {
  const int pos = p.positions[tokens.x + min((row0 + tile - 1) / G, tokens.y - tokens.x - 1)];
  return pos < 0 || pos >= p.limit ? 1 : pos / kUnit + 1;
}
// Units of a piece: the mean of all pieces' if there were `target`, so that there are at most that many
// more of them than tiles.  A tile is cut into pieces of exactly that and what is left, which is started
// after all others: it fills the time between the ends of these (equal pieces of a tile would end in a
// second round).  Less than `least` is no piece of its own.
__device__ __forceinline__ int piece_of(const Plan& w, unsigned long long units) {
  const unsigned long long up = units + w.target - 1;  // (a division in 64 bits takes long)
  const unsigned long long mean = up >> 32 ? up / w.target : (unsigned)up / (unsigned)w.target;
  return (int)min(max((unsigned long long)w.least, mean), 1ull << 30);
}

struct Cut {
  int pieces, rest;  // pieces, whether the last is shorter than the others
};
__device__ __forceinline__ Cut cut_of(int units, int per, int least) {
  int n = (units + per - 1) / per;
  if (n > 1 && units - (n - 1) * per < least) --n;
  return {n, n > 1 && units - (n - 1) * per < per};
}

// Four sums at once, exclusively over the threads of a block; their totals for all
__device__ __forceinline__ int4 add4(int4 a, int4 b) {
  return make_int4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}
__device__ __forceinline__ int4 shfl4(int4 a, int from) {
  return make_int4(__shfl_sync(0xffffffffu, a.x, from), __shfl_sync(0xffffffffu, a.y, from),
                   __shfl_sync(0xffffffffu, a.z, from), __shfl_sync(0xffffffffu, a.w, from));
}
__device__ __forceinline__ int4 warp_scan(int4 s, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int4 y = make_int4(__shfl_up_sync(0xffffffffu, s.x, o), __shfl_up_sync(0xffffffffu, s.y, o),
                             __shfl_up_sync(0xffffffffu, s.z, o), __shfl_up_sync(0xffffffffu, s.w, o));
    if (lane >= o) s = add4(s, y);
  }
  return s;
}
__device__ __forceinline__ int4 block_scan(int4 x, int4* part, int4* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int4 none = make_int4(0, 0, 0, 0);
  const int4 s = warp_scan(x, lane);
  __syncthreads();  // (the scan before has been read)
  if (lane == 31) part[warp] = s;
  __syncthreads();
  const int4 t = warp_scan(lane < warps ? part[lane] : none, lane);
  int4 before = shfl4(t, max(warp - 1, 0));
  if (warp == 0) before = none;
  *total = shfl4(t, 31);
  return make_int4(before.x + s.x - x.x, before.y + s.y - x.y, before.z + s.z - x.z, before.w + s.w - x.w);
}

__global__ void __launch_bounds__(kPlanThreads)
    plan_kernel(const __grid_constant__ ChunkProblem p, const __grid_constant__ Plan w) {
  // (what fits is kept in shared memory: a trip to global memory takes a tenth of a small plan)
  __shared__ int4 part[32];
  __shared__ unsigned long long work;
  __shared__ int most, length[kSorted], order[kSorted], first_s[kSorted + 1];
  __shared__ int2 tokens_s[kSorted], upto_s[kPlanThreads + 1];
  pdl_wait_and_launch();
  const int G = p.H / p.Hk, T = blockDim.x;
  const bool sorted = p.B <= kSorted && p.B <= T;
  int* first = sorted ? first_s : w.first;
  int tiles = 0;
  int4 total;
  if (threadIdx.x == 0) {
    work = 0;
    most = 0;
  }
  // the longest requests first (their tiles would end last otherwise)
  if (sorted) {
    const int b = threadIdx.x;
    int2 t = make_int2(0, 0);
    int mine = 0;
    if (b < p.B) {
      t = tokens_of(p, b);
      tokens_s[b] = t;
      if (t.y > t.x) mine = units_of(p, t, (t.y - t.x) * G - 1, G, 1);
      length[b] = mine;
    }
    __syncthreads();
    int rank = 0;
    if (b < p.B) {
      for (int i = 0; i < p.B; ++i) rank += length[i] > mine || (length[i] == mine && i < b);
      order[rank] = b;
    }
    __syncthreads();
  }
  auto request = [&](int i) { return sorted ? order[i] : i; };
  auto tokens = [&](int b) { return sorted ? tokens_s[b] : tokens_of(p, b); };
  for (int b0 = 0; b0 < p.B; b0 += T) {
    const int b = b0 + (int)threadIdx.x;
    const int n = b < p.B ? tiles_of(tokens(request(b)), G, w.tile) : 0;
    const int at = tiles + block_scan(make_int4(n, 0, 0, 0), part, &total).x;
    if (b < p.B) first[b] = at;
    tiles += total.x;
  }
  if (threadIdx.x == 0) first[p.B] = tiles;
  __syncthreads();
  tiles = min(tiles, w.max_tiles);  // (requests whose tokens overlap: not laid out past the workspace)
  const bool once = tiles <= T;     // a thread has a tile at most
  int2* upto = once ? upto_s : w.upto;
  unsigned long long mine = 0;
  int4 t = make_int4(0, 0, 0, 0);
  for (int i = threadIdx.x; i < tiles; i += T) {
    int lo = 0, hi = p.B;  // the last request whose first tile is not after this one
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= i) lo = mid; else hi = mid;
    }
    const int row0 = (i - first[lo]) * w.tile;
    t = make_int4(lo, row0, 1, units_of(p, tokens(request(lo)), row0, G, w.tile));
    if (!once) w.tiles[i] = t;
    mine += t.w;
  }
  for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&work, mine);
  __syncthreads();
  const int per_piece = piece_of(w, work * p.Hk);
  int4 sum = make_int4(0, 0, 0, 0);  // pieces but the rests, tiles of several, their slots, rests
  for (int i0 = 0; i0 < tiles; i0 += T) {
    const int i = i0 + (int)threadIdx.x;
    if (i < tiles && !once) t = w.tiles[i];
    const Cut c = i < tiles ? cut_of(t.w, per_piece, w.least) : Cut{0, 0};
    const bool several = c.pieces > 1;
    const int4 at = add4(sum, block_scan(make_int4(c.pieces - c.rest, several, several ? c.pieces * p.Hk : 0, c.rest),
                                         part, &total));
    sum = add4(sum, total);
    if (i < tiles) {
      const int b = request(t.x);
      const int2 tok = tokens(b);
      t.z = 2 * c.pieces + c.rest;
      t.w = several ? at.z : -1;
      if (!once) w.tiles[i] = t;
      upto[i] = make_int2(at.x, at.w);
      if (several) {
        const int rows = min(w.tile, (tok.y - tok.x) * G - t.y);
        w.split[at.y] = {b, tok.x, t.y, rows, c.pieces, at.z, 0, 0};
        atomicMax(&most, (rows + kJoinRows - 1) / kJoinRows);
      }
    }
  }
  if (threadIdx.x == 0) {
    upto[tiles] = make_int2(sum.x, sum.w);
    w.head[0] = (sum.x + sum.w) * p.Hk;
    w.head[1] = sum.y;
  }
  __syncthreads();
  if (threadIdx.x == 0) w.head[2] = most;
  for (int i = threadIdx.x; i < tiles; i += T) {
    if (!once) t = w.tiles[i];
    const int b = request(t.x);
    const int2 tok = tokens(b);
    const int end = min(first[t.x + 1], tiles), from = upto[first[t.x]].x, per = upto[end].x - from;
    const int later = upto[end].x - upto[i + 1].x, rows = min(w.tile, (tok.y - tok.x) * G - t.y);
    const int pieces = t.z >> 1, rest = t.z & 1, rests = sum.x * p.Hk + upto[i].y * p.Hk;
    for (int h = 0; h < p.Hk; ++h)
      for (int k = 0; k < pieces; ++k)
        w.items[rest && k == pieces - 1 ? rests + h : from * p.Hk + h * per + later + k] = {
            b, tok.x, t.y, rows, h, k * per_piece, k == pieces - 1 ? kToTheEnd : (k + 1) * per_piece,
            t.w < 0 ? -1 : t.w + h * pieces + k};
  }
}

// The same for up to 32 requests and 32 tiles, by one warp and for one CTA, the tiles in their order: lane =
// request, then lane = tile.  The first CTA writes down what the last kernel reads.
__device__ __forceinline__ Item plan_small(const ChunkProblem& p, const Plan& w) {
  const int lane = threadIdx.x & 31, G = p.H / p.Hk;
  int2 tok = lane < p.B ? tokens_of(p, lane) : make_int2(0, 0);
  const int n_tiles = lane < p.B ? tiles_of(tok, G, w.tile) : 0;
  const int upto = warp_scan(make_int4(n_tiles, 0, 0, 0), lane).x;
  const int tiles = min(__shfl_sync(0xffffffffu, upto, 31), min(w.max_tiles, 32));
  int b = 0, before = 0;  // this lane's tile: its request
  for (int i = 0; i < p.B; ++i) {
    const int u = __shfl_sync(0xffffffffu, upto, i);
    if (lane >= u) { b = i + 1; before = u; }
  }
  b = min(b, p.B - 1);
  tok = make_int2(__shfl_sync(0xffffffffu, tok.x, b), __shfl_sync(0xffffffffu, tok.y, b));
  const bool is = lane < tiles;
  const int row0 = (lane - before) * w.tile, units = is ? units_of(p, tok, row0, G, w.tile) : 0;
  const int rows = is ? min(w.tile, (tok.y - tok.x) * G - row0) : 0;
  const unsigned long long all = (unsigned long long)__reduce_add_sync(0xffffffffu, (unsigned)units) * p.Hk;
  const int per_piece = piece_of(w, all);
  const Cut c = is ? cut_of(units, per_piece, w.least) : Cut{0, 0};
  const bool several = c.pieces > 1;
  const int4 mine = make_int4((c.pieces - c.rest) * p.Hk, several, several ? c.pieces * p.Hk : 0, c.rest * p.Hk);
  const int4 end = warp_scan(mine, lane);
  const int slot = several ? end.z - mine.z : -1;
  if (blockIdx.x == 0) {
    if (several) w.split[end.y - 1] = {b, tok.x, row0, rows, c.pieces, slot, 0, 0};
    const int most = __reduce_max_sync(0xffffffffu, several ? (rows + kJoinRows - 1) / kJoinRows : 0);
    if (lane == 31) {
      w.head[1] = end.y;
      w.head[2] = most;
    }
  }
  // the tile that holds this CTA's item: among the pieces but the rests, or the rests after them
  const int firsts = __shfl_sync(0xffffffffu, end.x, 31);
  const bool rest = (int)blockIdx.x >= firsts;
  const int upto_mine = rest ? firsts + end.w : end.x, own = rest ? mine.w : mine.x;
  const unsigned past = __ballot_sync(0xffffffffu, upto_mine > (int)blockIdx.x);
  const int of = past ? __ffs(past) - 1 : 31;
  const int at = (int)blockIdx.x - __shfl_sync(0xffffffffu, upto_mine - own, of);
  const int pieces = __shfl_sync(0xffffffffu, c.pieces, of), whole = pieces - __shfl_sync(0xffffffffu, c.rest, of);
  const int first = __shfl_sync(0xffffffffu, slot, of);
  Item it = {__shfl_sync(0xffffffffu, b, of), __shfl_sync(0xffffffffu, tok.x, of),
             __shfl_sync(0xffffffffu, row0, of), __shfl_sync(0xffffffffu, rows, of), 0, 0, 0, -1};
  if (past) {
    it.head = rest ? at : at / whole;
    const int k = rest ? pieces - 1 : at - it.head * whole;
    it.u0 = k * per_piece;
    it.u1 = k == pieces - 1 ? kToTheEnd : it.u0 + per_piece;
    it.slot = first < 0 ? -1 : first + it.head * pieces + k;
  }
  return it;
}

// One item's rows and keys
struct Work {
  int head, slot, b, s0, rows, row0, u0, u1, kmin, kmax;
};

// Row `key` of a request: element offset in the pages
__device__ __forceinline__ long long page_row(const ChunkProblem& p, const int* table, int key, int head) {
  const int col = page_of(key, p.page, p.page_mul, p.page_shift);
  int id = table[col];
  if ((unsigned)id >= (unsigned)p.n_pages) {
    if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    id = 0;
  }
  return (long long)id * p.sP + (long long)(key - col * p.page) * p.sR + (long long)head * p.sC;
}

// This CTA's item: ROWS threads each take a row's position (-1: none) and its element offset in q.  False: no
// item.
template <int ROWS>
__device__ __forceinline__ bool take_item(const ChunkProblem& p, const Plan& w, Work& k, int* pos,
                                          long long* off, int* lowest, int* highest) {
  __shared__ Item shared_item;
  Item it;
  if (w.small) {
    if (threadIdx.x < 32) {
      it = plan_small(p, w);
      if (threadIdx.x == 0) shared_item = it;
    }
  } else {
    it = w.items[blockIdx.x];  // (read beside the number of them)
    if ((int)blockIdx.x >= w.head[0]) return false;
  }
  if (threadIdx.x == 0) {
    *lowest = 0x7fffffff;
    *highest = -1;
  }
  __syncthreads();
  if (w.small) {
    it = shared_item;
    if (it.u1 == 0) return false;
  }
  const int G = p.H / p.Hk;
  k.head = it.head; k.slot = it.slot; k.b = it.b; k.s0 = it.s0; k.row0 = it.row0; k.rows = it.rows;
  if (threadIdx.x < ROWS) {
    const int r = threadIdx.x;
    int at = -1;
    off[r] = -1;
    if (r < k.rows) {
      const int f = it.row0 + r, token = it.s0 + f / G;
      at = p.positions[token];
      if (at >= p.limit) {
        if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
        at = -1;
      }
      at = max(at, -1);
      off[r] = (long long)token * p.qsT + (long long)(it.head * G + f % G) * p.qsH;
    }
    pos[r] = at;
    const int lo = __reduce_min_sync(0xffffffffu, at < 0 ? 0x7fffffff : at),
              hi = __reduce_max_sync(0xffffffffu, at);
    if ((r & 31) == 0) {
      atomicMin(lowest, lo);
      atomicMax(highest, hi);
    }
  }
  __syncthreads();
  k.kmin = *lowest; k.kmax = *highest;
  const int n = k.kmax < 0 ? 0 : k.kmax / kUnit + 1;
  k.u0 = min(it.u0, n);
  k.u1 = min(it.u1, n);
  return true;
}

// The epilogue's scalars of a row from m (log2), l and its self evidence
struct Mix {
  float g, self, inv_l, logz;
  __device__ __forceinline__ Mix(const ChunkProblem& p, float m, float l, float u_self, int pos) {
    const float S = 1.0f / (1.0f + __expf(-(u_self * p.inv_sqrt_d) / p.tau_s));
    g = 0.f; self = 1.f; inv_l = 0.f; logz = S;  // empty history
    if (!(l == 0.f)) {                           // (a NaN goes on)
      const float A = m * kLn2 + logf(l) - p.lambda * logf((float)(pos + 1));
      g = 1.0f / (1.0f + __expf(S - A));
      self = 1.0f / (1.0f + __expf(A - S));
      const float hi = fmaxf(S, A), lo = fminf(S, A);
      logz = hi + log1pf(__expf(lo - hi)) + 0.f * (A + S);  // (NaN in either)
      inv_l = 1.0f / l;
    }
  }
  __device__ __forceinline__ float y(float z, float v) const { return fmaf(g, z * inv_l, self * v); }
};

// ---------------------------------------------------------------------------------------------------
// bf16
// ---------------------------------------------------------------------------------------------------
constexpr int BM = 128;

// Warps 0-3 scan (thread = row = TMEM lane), warp 4 loads, warp 5 issues the products, as in the forward:
// two CTAs per SM and steps of a unit.
template <int D>
struct Cfg {
  static constexpr int SK = kUnit;
  static constexpr int CTAS = 2;
  static constexpr int TMEM_COLS = 256;
  static constexpr int OCOL = 2 * SK;
  static constexpr int STAGES = D == 64 ? 4 : 2;
  static constexpr int THREADS = 192;
  static constexpr int KB = D / 64;            // 128-byte blocks of a row
  static constexpr int UT = kUnit * D * 2;     // bytes of a unit's keys or values
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = BM * D * 2;
  static constexpr int OFF_V = OFF_K + STAGES * UT;
  static constexpr int OFF_BAR = OFF_V + STAGES * UT;
  static constexpr int OFF_POS = OFF_BAR + 256;
  static constexpr int OFF_ROW = OFF_POS + BM * 4;
  static constexpr int SMEM = OFF_ROW + BM * 8 + 1024;  // + alignment
  static_assert(CTAS * (SMEM + 1024) <= 233472, "CTAs per SM");
  static_assert(OCOL + D <= TMEM_COLS, "TMEM");
};
enum : int { B_KF = 0, B_KE = 4, B_VF = 8, B_VE = 12, B_S = 16, B_P = 18, B_OD = 20, B_O = 22, B_VR = 23, B_Q = 24, N_BAR = 25 };
// How a unit's rows are fetched: element by element, in 16-byte groups, by TMA in boxes of rows of a page
enum : int { kElements = 0, kGroups = 1, kBoxes = 2 };

// 16 bytes, or zeros where !real
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// One arrival of this thread on `bar` when its copies so far have landed
__device__ __forceinline__ void cp_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
// Elements c .. c + 7 of a row of d, zeros past its end
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* row, int c, int d) {
  union {
    uint4 w;
    unsigned short h[8];
  } u;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    u.h[e] = c + e < d ? reinterpret_cast<const unsigned short*>(row)[c + e] : (unsigned short)0;
  return u.w;
}
__device__ __forceinline__ uint32_t unfinite_halves(uint32_t w) {  // 0xffff for each that is
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// TMA boxes have `big` rows of a page or 8; a unit's part of a page is cut into as many big ones as fit (tmK8 and
// tmV8 are empty where these are all)
template <int D, int LOAD>
__global__ void __launch_bounds__(Cfg<D>::THREADS, Cfg<D>::CTAS)
    chunk_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                    const __grid_constant__ CUtensorMap tmK8, const __grid_constant__ CUtensorMap tmV8,
                    const __grid_constant__ ChunkProblem p, const __grid_constant__ Plan w, int big) {
  constexpr bool VEC = LOAD != kElements;
  using C = Cfg<D>;
  using BF = __nv_bfloat16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t sb = smem_u32(smem);
  auto bar = [&](int i) -> uint32_t { return sb + C::OFF_BAR + 8u * (uint32_t)i; };
  static_assert(N_BAR * 8 <= 200, "barrier slots");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_BAR + 200);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_BAR + 204);
  volatile int* special = reinterpret_cast<volatile int*>(smem + C::OFF_BAR + 208);
  int* bounds = reinterpret_cast<int*>(smem + C::OFF_BAR + 212);
  int* pos = reinterpret_cast<int*>(smem + C::OFF_POS);
  long long* row_off = reinterpret_cast<long long*>(smem + C::OFF_ROW);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_wait();
  Work k;
  if (!take_item<BM>(p, w, k, pos, row_off, bounds, bounds + 1)) return;
  const BF* Q = static_cast<const BF*>(p.q);
  const BF* K = static_cast<const BF*>(p.k);
  const BF* V = static_cast<const BF*>(p.v);
  const int* table = p.table + (long long)k.b * p.t_stride;
  const int units = k.u1 - k.u0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(bar(B_KF + s), LOAD == kBoxes ? 1 : 32);
      mbar_init(bar(B_KE + s), 1);
      mbar_init(bar(B_VF + s), LOAD == kBoxes ? 1 : 32);
      mbar_init(bar(B_VE + s), 1);
    }
    mbar_init(bar(B_VR), 1);
    mbar_init(bar(B_Q), 128);
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar(B_S + b), 1);
      mbar_init(bar(B_P + b), 128);
      mbar_init(bar(B_OD + b), 1);
    }
    mbar_init(bar(B_O), 1);
    *abort_flag = 0;
    *special = 0;
    fence_mbar_init();
  }
  if (warp == 5) tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Abort ab{abort_flag, p.dev_status};

  if (warp == 4) {
    // ---------------------------------------------------------------- keys and values, unit by unit
    // Keys that some row does not see have weight 0 there, which an infinite or NaN value would turn into
    // NaN: in the units of such keys (and of rows behind the last key, whatever they hold) these values are
    // taken out of shared memory, and the rows that see them get them at the end.
    auto masked = [&](int j) { return (k.u0 + j) * kUnit + kUnit - 1 >= k.kmin; };
    auto clean = [&](uint32_t at, int j) {
      bool bad = false;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = lane + 32 * half;
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          uint4* x = reinterpret_cast<uint4*>(smem + at + (c >> 3) * (kUnit * 128) + r * 128 +
                                              (((c & 7) ^ (r & 7)) << 4));
          const uint4 v = *x;
          const uint4 f = make_uint4(unfinite_halves(v.x), unfinite_halves(v.y), unfinite_halves(v.z),
                                     unfinite_halves(v.w));
          if (f.x | f.y | f.z | f.w) {
            *x = make_uint4(v.x & ~f.x, v.y & ~f.y, v.z & ~f.z, v.w & ~f.w);
            bad |= (k.u0 + j) * kUnit + r <= k.kmax;
          }
        }
      }
      if (bad) *special = 1;
      fence_async_smem();
      __syncwarp();
    };
    if constexpr (LOAD == kBoxes) {
      // A lane has one box of a unit, of one 64-column block of the keys or the values
      const int mine = lane % 8, kb = lane / 8;  // (at most 8 boxes)
      struct Box {
        int id, row, at, rows, all;  // page (-1: none), row in it, row in the unit, rows; all boxes' rows
      };
      auto box_of = [&](int j) {  // the lane's box of unit j; its page is looked up
        Box x = {-1, 0, 0, 0, 0};
        if (j >= units) return x;
        int key = (k.u0 + j) * kUnit, col = page_of(key, p.page, p.page_mul, p.page_shift), row = key - col * p.page;
        const int end = min(kUnit, k.kmax + 1 - key);
        for (int i = 0, at = 0; at < end; ++i) {
          const int rows = min(p.page - row, kUnit - at) >= big ? big : 8;
          if (i == mine && kb < C::KB) {
            x.id = col;
            x.row = row;
            x.at = at;
            x.rows = rows;
          }
          x.all += rows;
          at += rows;
          row += rows;
          if (row == p.page) {
            row = 0;
            ++col;
          }
        }
        if (x.id >= 0) {
          x.id = table[x.id];
          if ((unsigned)x.id >= (unsigned)p.n_pages) {
            if (p.dev_status) atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
            x.id = 0;
          }
        }
        return x;
      };
      auto fetch = [&](const CUtensorMap* map, const CUtensorMap* map8, uint32_t stage, uint32_t full, const Box& x) {
        if (lane == 0) mbar_arrive_expect_tx(full, x.all * 128 * C::KB);
        __syncwarp();
        if (x.id >= 0)
          tma_load_4d(sb + stage + kb * (kUnit * 128) + x.at * 128, x.rows == big ? map : map8, full, kb * 64, x.row,
                      k.head, x.id);
      };
      // The keys go one unit ahead: their place is free as soon as the scores of two units before are done,
      // the values' only after the products with the weights (keys behind the values: a third of the time
      // of a long prompt's piece was spent waiting for them).
      Box at = box_of(0), last = at;
      int issued = 0, raw = 0;
      for (int j = 0; j <= units; ++j) {
        const int s = j % C::STAGES, u = j / C::STAGES;
        const Box next = box_of(j + 1);  // (the next unit's pages are looked up meanwhile)
        if (j < units) {
          if (u > 0 && !mbar_wait_warp(bar(B_KE + s), (u - 1) & 1, ab)) break;
          fetch(&tmK, &tmK8, C::OFF_K + s * C::UT, bar(B_KF + s), at);
          issued = j + 1;
        }
        if (j > 0) {
          const int v = j - 1, sv = v % C::STAGES, uv = v / C::STAGES;
          if (uv > 0 && !mbar_wait_warp(bar(B_VE + sv), (uv - 1) & 1, ab)) break;
          const uint32_t vs = C::OFF_V + sv * C::UT;
          if (!masked(v)) {
            fetch(&tmV, &tmV8, vs, bar(B_VF + sv), last);
          } else {
            fetch(&tmV, &tmV8, vs, bar(B_VR), last);
            if (!mbar_wait_warp(bar(B_VR), raw & 1, ab)) break;
            ++raw;
            clean(vs, v);
            if (lane == 0) mbar_arrive(bar(B_VF + sv));
          }
        }
        last = at;
        at = next;
      }
      if (ab.raised()) {  // copies in flight land before the CTA gives up its shared memory
        for (int j = max(issued - C::STAGES, 0); j < issued; ++j) {
          tc::drain_wait(bar(B_KF + j % C::STAGES), (j / C::STAGES) & 1);
          tc::drain_wait(bar(B_VF + j % C::STAGES), (j / C::STAGES) & 1);
        }
        tc::drain_wait(bar(B_VR), raw & 1);
      }
    } else {
      auto rows_of = [&](int j, long long& o0, long long& o1) {  // a lane's two rows of unit j, -1: none
        const int key = (k.u0 + j) * kUnit + lane;
        o0 = j < units && key <= k.kmax ? page_row(p, table, key, k.head) : -1;
        o1 = j < units && key + 32 <= k.kmax ? page_row(p, table, key + 32, k.head) : -1;
      };
      auto fetch = [&](const BF* base, uint32_t stage, long long o0, long long o1) {
        constexpr int CH = D / 8, PER = 32 / CH;  // groups of a row, rows at a time
        const int c = lane % CH;
#pragma unroll 8
        for (int i = 0; i < kUnit / PER; ++i) {
          const int r = i * PER + lane / CH;
          const long long off = __shfl_sync(0xffffffffu, i * PER < 32 ? o0 : o1, r & 31);
          const bool real = off >= 0 && 8 * c < p.d;
          const uint32_t dst = stage + (c >> 3) * (kUnit * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
          if (VEC) {
            cp16(sb + dst, real ? base + off + 8 * c : base, real);
          } else {
            *reinterpret_cast<uint4*>(smem + dst) =
                real ? load8(base + off, 8 * c, p.d) : make_uint4(0, 0, 0, 0);
          }
        }
      };
      long long o0, o1, n0, n1, p0 = -1, p1 = -1;
      rows_of(0, o0, o1);
      for (int j = 0; j <= units; ++j) {
        const int s = j % C::STAGES, u = j / C::STAGES;
        rows_of(j + 1, n0, n1);  // (the next unit's pages are looked up meanwhile)
        if (j < units) {
          if (u > 0 && !mbar_wait_warp(bar(B_KE + s), (u - 1) & 1, ab)) break;
          fetch(K, C::OFF_K + s * C::UT, o0, o1);
          if (VEC) {
            cp_arrive(bar(B_KF + s));
          } else {
            fence_async_smem();
            mbar_arrive(bar(B_KF + s));
          }
        }
        if (j > 0) {
          const int v = j - 1, sv = v % C::STAGES, uv = v / C::STAGES;
          if (uv > 0 && !mbar_wait_warp(bar(B_VE + sv), (uv - 1) & 1, ab)) break;
          const uint32_t at = C::OFF_V + sv * C::UT;
          fetch(V, at, p0, p1);
          if (VEC && !masked(v)) {
            cp_arrive(bar(B_VF + sv));
          } else {
            cp_wait_all();
            __syncwarp();
            if (masked(v)) clean(at, v); else fence_async_smem();
            mbar_arrive(bar(B_VF + sv));
          }
        }
        p0 = o0;
        p1 = o1;
        o0 = n0;
        o1 = n1;
      }
      cp_wait_all();
    }
  } else if (warp == 5) {
    // ---------------------------------------------------------------- products (as the forward's)
    constexpr uint32_t idesc_qk = idesc_bf16_f32(BM, C::SK, false, false);
    const int dk = (p.d + 15) / 16;  // 16-column steps; z has as many columns
    const uint32_t idesc_pv = idesc_bf16_f32(BM, 16 * dk, false, true);
    auto issue_u = [&](int s) -> bool {
      const int st = s % C::STAGES, bf = s & 1;
      if (!mbar_wait_warp(bar(B_KF + st), (s / C::STAGES) & 1, ab)) return false;
      if (LOAD != kBoxes) fence_async_smem();  // (cp.async wrote the unit through the generic proxy)
      tc_fence_after();
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        if (kk >= dk) break;
        const uint32_t koff = (kk >> 2) * (BM * 128) + (kk & 3) * 32;
        const uint32_t kkoff = (kk >> 2) * (kUnit * 128) + (kk & 3) * 32;
        const uint64_t a = smem_desc_sw128(sb + C::OFF_Q + koff, 16, 1024);
        const uint64_t bd = smem_desc_sw128(sb + C::OFF_K + st * C::UT + kkoff, 16, 1024);
        mma_ss_w(tmem + bf * C::SK, a, bd, idesc_qk, kk > 0 ? 1u : 0u);
      }
      mma_commit_w(bar(B_S + bf));
      mma_commit_w(bar(B_KE + st));
      return true;
    };
    bool ok = mbar_wait_warp(bar(B_Q), 0, ab);
    for (int s = 0; ok && s < 2 && s < units; ++s) ok = issue_u(s);
    for (int s = 0; ok && s < units; ++s) {
      const int st = s % C::STAGES, bf = s & 1;
      if (!(ok = mbar_wait_warp(bar(B_VF + st), (s / C::STAGES) & 1, ab))) break;
      if (LOAD != kBoxes) fence_async_smem();
      if (!(ok = mbar_wait_warp(bar(B_P + bf), (s / 2) & 1, ab))) break;
      tc_fence_after();
#pragma unroll
      for (int kk = 0; kk < C::SK / 16; ++kk) {
        const uint64_t bd = smem_desc_sw128(sb + C::OFF_V + st * C::UT + kk * 16 * 128, kUnit * 128, 1024);
        mma_ts_w(tmem + C::OCOL, tmem + bf * C::SK + kk * 8, bd, idesc_pv, (s > 0 || kk > 0) ? 1u : 0u);
      }
      mma_commit_w(bar(B_OD + bf));
      mma_commit_w(bar(B_VE + st));
      if (s + 2 < units && !(ok = issue_u(s + 2))) break;
    }
    mma_commit_w(bar(B_O));
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- scan and epilogue
    const int t = threadIdx.x, at = pos[t];
    // the queries, 16-byte groups swizzled within 128 bytes, while the first keys are on their way; zeros for
    // rows and columns that there are not
#pragma unroll 4
    for (int e = t; e < BM * (D / 8); e += 128) {
      const int r = e / (D / 8), c = e % (D / 8);
      const long long off = row_off[r];
      const bool real = off >= 0 && 8 * c < p.d;
      const uint32_t dst = C::OFF_Q + (c >> 3) * (BM * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
      if (VEC) {
        cp16(sb + dst, real ? Q + off + 8 * c : Q, real);
      } else {
        *reinterpret_cast<uint4*>(smem + dst) = real ? load8(Q + off, 8 * c, p.d) : make_uint4(0, 0, 0, 0);
      }
    }
    cp_wait_all();
    fence_async_smem();
    mbar_arrive(bar(B_Q));
    const bool any = __any_sync(0xffffffffu, at >= 0);
    // the first key that some row of the warp does not take as history
    const int first = __reduce_min_sync(0xffffffffu, at < 0 ? 0x7fffffff : at);
    const uint32_t trow = tmem + ((uint32_t)(warp * 32) << 16);
    const float isd = p.inv_sqrt_d, ch = 0.5f * isd, c2k = ch * kLog2e, bk = isd * kLog2e;
    // (the scale's rules are those of the forward)
    float m = -INFINITY, m_next = -INFINITY, l = 0.f, u_self = 0.f;
    bool ok = true;
    auto rescale = [&](bool go, float mn, int s_done) -> bool {
      const float sc = go ? ex2_approx(m - mn) : 1.0f;
      if (!__any_sync(0xffffffffu, go)) return true;
      if (s_done >= 0) {
        if (!mbar_wait_warp(bar(B_OD + (s_done & 1)), (s_done / 2) & 1, ab)) return false;
        tc_fence_after();
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += 32) {
          if (c0 >= p.d) break;
          uint32_t z[32];
          tmem_ld32(trow + C::OCOL + c0, z);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < 32; ++c) z[c] = __float_as_uint(__uint_as_float(z[c]) * sc);
          tmem_st16(trow + C::OCOL + c0, z);
          tmem_st16(trow + C::OCOL + c0 + 16, z + 16);
        }
      }
      l *= sc;
      if (go) m = mn;
      return true;
    };
    for (int s = 0; s < units; ++s) {
      const int bf = s & 1, key0 = k.u0 * kUnit + s * C::SK;
      if (!(ok = mbar_wait_warp(bar(B_S + bf), (s / 2) & 1, ab))) break;
      if (any) {
        tc_fence_after();
        if (!(ok = rescale(m_next > m, m_next, s - 1))) break;
        const uint32_t ucol = trow + bf * C::SK;
        const int tl = at - key0;  // keys before tl are the row's history, tl its own
        const bool diag = key0 + C::SK > first;
        float umax;
        float2 rs;
        uint32_t U[tc::HN];
        tmem_ld32(ucol, U);
        tmem_ld32(ucol + 32, U + 32);
        tmem_ld_wait();
        if (__any_sync(0xffffffffu, m == -INFINITY)) {
          const float um = diag ? tc::row_max<true>(U, tl, u_self) : tc::row_max<false>(U, tl, u_self);
          if (m == -INFINITY && um != -INFINITY) m = fmaxf(um, 0.f) * bk;
        }
        rs = diag ? tc::scan_p<true>(U, tl, ucol, ch, c2k, m == -INFINITY ? 0.f : -m, umax, u_self)
                  : tc::scan_p<false>(U, tl, ucol, ch, c2k, m == -INFINITY ? 0.f : -m, umax, u_self);
        float mt = umax == -INFINITY ? -INFINITY : fmaxf(umax, 0.f) * bk;
        const bool jump = mt > m + tc::kStaleLog2;
        if (__any_sync(0xffffffffu, jump)) {
          if (!(ok = rescale(jump, fmaxf(mt, m_next), s - 1))) break;
          rs = diag ? tc::scan_p<true>(U, tl, ucol, ch, c2k, m == -INFINITY ? 0.f : -m, umax, u_self)
                    : tc::scan_p<false>(U, tl, ucol, ch, c2k, m == -INFINITY ? 0.f : -m, umax, u_self);
        }
        mt = umax == -INFINITY ? -INFINITY : fmaxf(umax, 0.f) * bk;
        if (mt > m + tc::kRescaleLog2) m_next = fmaxf(m_next, mt);
        l += rs.x + rs.y;
        tmem_st_wait();
        tc_fence_before();
      }
      mbar_arrive(bar(B_P + bf));
    }
    // the row's own value, 16 columns ahead of their use
    const bool part = k.slot >= 0, live = at >= 0;
    const BF* own = V + (live && !part ? page_row(p, table, at, k.head) : 0);
    auto own_at = [&](int c) {  // columns c .. c + 7
      if (!live || part || c >= p.d) return make_uint4(0, 0, 0, 0);
      return VEC ? *reinterpret_cast<const uint4*>(own + c) : load8(own, c, p.d);
    };
    uint4 v0 = own_at(0), v1 = own_at(8);
    if (ok) ok = mbar_wait_warp(bar(B_O), 0, ab);
    tc_fence_after();
    if (ok && __any_sync(0xffffffffu, row_off[t] >= 0)) {
      const bool fix = *special != 0;
      // the first unit in which some row does not see every key, in this piece
      const int j0 = max(k.kmin / kUnit, k.u0) * kUnit, j1 = min(at, k.u1 * kUnit);
      const Mix mix(p, m, l, u_self, max(at, 0));
      uint8_t* stage = smem + C::OFF_Q + warp * (32 * D * 2) + lane * 128;
#pragma unroll 1
      for (int c0 = 0; c0 < p.d; c0 += 16) {
        const uint32_t vw[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
        v0 = own_at(c0 + 16);
        v1 = own_at(c0 + 24);
        uint32_t zr[16];
        if (units > 0) {
          tmem_ld16(trow + C::OCOL + c0, zr);
          tmem_ld_wait();
        }
        float z[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) z[c] = units > 0 ? __uint_as_float(zr[c]) : 0.f;
        if (fix && live) {  // rare: the values that were taken out
#pragma unroll 1
          for (int j = j0; j < j1; ++j) {
            const BF* v = V + page_row(p, table, j, k.head);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              const float x = c0 + c < p.d ? (float)v[c0 + c] : 0.f;
              if (!isfinite(x)) z[c] += x;
            }
          }
        }
        if (part) {
          float* dst = w.z + ((long long)k.slot * w.rows + t) * w.width + c0;
          if (live)
#pragma unroll
            for (int c = 0; c < 16; c += 4)
              if (c0 + c < w.width)
                *reinterpret_cast<float4*>(dst + c) = make_float4(z[c], z[c + 1], z[c + 2], z[c + 3]);
        } else {
#pragma unroll
          for (int c = 0; c < 16; c += 8) {
            uint32_t yw[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t w2 = vw[c / 2 + e];
              const float2 vf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w2));
              yw[e] = live ? pack_bf16x2(mix.y(z[c + 2 * e], vf.x), mix.y(z[c + 2 * e + 1], vf.y)) : 0u;
            }
            const int g = ((c0 & 63) + c) >> 3;
            *reinterpret_cast<uint4*>(stage + (c0 >> 6) * (32 * 128) + ((g ^ (lane & 7)) << 4)) =
                make_uint4(yw[0], yw[1], yw[2], yw[3]);
          }
        }
      }
      if (part) {
        if (live)
          w.stats[(long long)k.slot * w.rows + t] =
              make_float4(m, l, u_self, at >= k.u0 * kUnit && at < k.u1 * kUnit ? 1.f : 0.f);
      } else {
        __syncwarp();
        constexpr int CH = D / 8, PER = 32 / CH;
        const int c = lane % CH;
        for (int i = 0; i < 32; i += PER) {
          const int r = i + lane / CH;
          const long long off = row_off[warp * 32 + r];
          if (off < 0 || 8 * c >= p.d) continue;
          const uint4 y = *reinterpret_cast<const uint4*>(smem + C::OFF_Q + warp * (32 * D * 2) + r * 128 +
                                                          (c >> 3) * (32 * 128) + (((c & 7) ^ (r & 7)) << 4));
          BF* dst = static_cast<BF*>(p.out) + off + 8 * c;
          if (VEC) {
            *reinterpret_cast<uint4*>(dst) = y;
          } else {
            const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (8 * c + e < p.d)
                reinterpret_cast<unsigned short*>(dst)[e] = (unsigned short)(yw[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
      // a row without a position is padding: zero, logz -inf (by its tile's first piece)
      if (row_off[t] >= 0 && (!part || !live)) {
        const int f = k.row0 + t, G = p.H / p.Hk;
        const int token = k.s0 + f / G, head = k.head * G + f % G;
        if (!part || k.u0 == 0) {
          p.logz[(long long)token * p.H + head] = live ? mix.logz : -INFINITY;
          if (part)
            for (int c = 0; c < p.d; ++c) static_cast<BF*>(p.out)[row_off[t] + c] = (BF)0.f;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------------------------------
// fp32: 64 rows by 64 keys on 256 threads.  A thread has 4 rows by 4 keys of the scores, then 4 rows by two
// columns of every 32 of the products with the values; the weights pass through the keys' shared memory.
// ---------------------------------------------------------------------------------------------------
constexpr int SM_ROWS = 64, kSimtThreads = 256;

template <int D>
struct SimtSmem {
  float q[SM_ROWS][D + 4];
  union {
    float k[kUnit][D + 4];
    float pr[SM_ROWS][kUnit + 4];
  };
  float v[kUnit][D];
  long long off[SM_ROWS], row[kUnit];
  int pos[SM_ROWS], bounds[2];
  float self[SM_ROWS];
};

template <int D, bool VEC>
__global__ void __launch_bounds__(kSimtThreads, 2)
    chunk_simt_kernel(const __grid_constant__ ChunkProblem p, const __grid_constant__ Plan w) {
  extern __shared__ __align__(16) uint8_t raw[];
  SimtSmem<D>& sm = *reinterpret_cast<SimtSmem<D>*>(raw);
  pdl_wait();
  Work k;
  if (!take_item<SM_ROWS>(p, w, k, sm.pos, sm.off, sm.bounds, sm.bounds + 1)) return;
  const float* Q = static_cast<const float*>(p.q);
  const int* table = p.table + (long long)k.b * p.t_stride;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  // rows of D columns at the offsets `at` (-1: zeros) into shared memory
  auto fetch = [&](const float* base, const long long* at, float* dst, int stride, int rows) {
    for (int e = threadIdx.x; e < rows * (D / 4); e += kSimtThreads) {
      const int r = e / (D / 4), c = 4 * (e % (D / 4));
      const long long off = at[r];
      if (VEC) {
        const bool real = off >= 0 && c < p.d;
        cp16(smem_u32(dst + r * stride + c), real ? base + off + c : base, real);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[r * stride + c + i] = off >= 0 && c + i < p.d ? base[off + c + i] : 0.f;
      }
    }
  };
  fetch(Q, sm.off, &sm.q[0][0], D + 4, SM_ROWS);
  int at[4];
  float m[4], l[4], o[4][D / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at[i] = sm.pos[4 * ty + i];
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
  }
  auto row_of = [&](int u) {  // a key's row, by its thread; the next unit's are looked up meanwhile
    const int key = u * kUnit + (int)threadIdx.x;
    return threadIdx.x < kUnit && u < k.u1 && key <= k.kmax ? page_row(p, table, key, k.head) : -1LL;
  };
  long long next = row_of(k.u0);
  for (int u = k.u0; u < k.u1; ++u) {
    const int key0 = u * kUnit;
    __syncthreads();  // the unit before has been used
    if (threadIdx.x < kUnit) sm.row[threadIdx.x] = next;
    __syncthreads();
    fetch(static_cast<const float*>(p.k), sm.row, &sm.k[0][0], D + 4, kUnit);
    fetch(static_cast<const float*>(p.v), sm.row, &sm.v[0][0], D, kUnit);
    next = row_of(u + 1);
    cp_wait_all();
    __syncthreads();
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float4 a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(&sm.q[4 * ty + i][c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][c]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = fmaf(a[i].x, b[j].x, s[i][j]);
          s[i][j] = fmaf(a[i].y, b[j].y, s[i][j]);
          s[i][j] = fmaf(a[i].z, b[j].z, s[i][j]);
          s[i][j] = fmaf(a[i].w, b[j].w, s[i][j]);
        }
    }
    const bool masked = key0 + kUnit - 1 >= k.kmin;  // some row does not see every key
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = key0 + tx + 16 * j;
        const float x = s[i][j] * p.inv_sqrt_d;
        if (key == at[i]) sm.self[4 * ty + i] = s[i][j];
        // SiLU in units of log 2
        s[i][j] = key < at[i] ? __fdividef(x, 1.0f + ex2_approx(-x * kLog2e)) * kLog2e : -INFINITY;
        mx = fmaxf(mx, s[i][j]);
      }
#pragma unroll
      for (int e = 1; e < 16; e <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, e));
      const float to = fmaxf(m[i], mx), base = to == -INFINITY ? 0.f : to;
      const float f = m[i] == -INFINITY ? 1.f : ex2_approx(m[i] - base);
      m[i] = to;
      l[i] *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = ex2_approx(s[i][j] - base);
        l[i] += s[i][j];
      }
    }
    __syncthreads();  // the keys have been read: the weights take their place
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sm.pr[4 * ty + i][tx + 16 * j] = s[i][j];
    __syncthreads();
    auto add = [&](auto mask) {
#pragma unroll 2
      for (int j = 0; j < kUnit; j += 4) {
        float4 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(&sm.pr[4 * ty + i][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
          for (int e = 0; e < D / 32; ++e) {
            const float2 v = *reinterpret_cast<const float2*>(&sm.v[j + jj][32 * e + 2 * tx]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = jj == 0 ? a[i].x : jj == 1 ? a[i].y : jj == 2 ? a[i].z : a[i].w;
              // (a weight of 0 for a key that the row does not see would turn its infinity into NaN)
              if (decltype(mask)::value && key0 + j + jj >= at[i]) continue;
              o[i][2 * e] = fmaf(x, v.x, o[i][2 * e]);
              o[i][2 * e + 1] = fmaf(x, v.y, o[i][2 * e + 1]);
            }
          }
      }
    };
    if (masked) add(std::true_type()); else add(std::false_type());
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int e = 1; e < 16; e <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], e);
    const int r = 4 * ty + i;
    if (sm.off[r] < 0) continue;
    const bool live = at[i] >= 0, has = at[i] >= k.u0 * kUnit && at[i] < k.u1 * kUnit;
    const float u_self = has ? sm.self[r] : 0.f;
    if (k.slot >= 0 && live) {
      float* dst = w.z + ((long long)k.slot * w.rows + r) * w.width;
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
        if (32 * e + 2 * tx < w.width)
          *reinterpret_cast<float2*>(dst + 32 * e + 2 * tx) = make_float2(o[i][2 * e], o[i][2 * e + 1]);
      if (tx == 0)
        w.stats[(long long)k.slot * w.rows + r] = make_float4(m[i], l[i], u_self, has ? 1.f : 0.f);
      continue;
    }
    if (k.slot >= 0 && k.u0 > 0) continue;  // (padding: by its tile's first piece)
    const Mix mix(p, m[i], l[i], u_self, max(at[i], 0));
    const float* V = static_cast<const float*>(p.v) + (live ? page_row(p, table, at[i], k.head) : 0);
    float* y = static_cast<float*>(p.out) + sm.off[r];
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = 32 * e + 2 * tx + c;
        if (col < p.d) y[col] = live ? mix.y(o[i][2 * e + c], V[col]) : 0.f;
      }
    if (tx == 0) {
      const int f = k.row0 + r, G = p.H / p.Hk;
      p.logz[(long long)(k.s0 + f / G) * p.H + k.head * G + f % G] = live ? mix.logz : -INFINITY;
    }
  }
}

// ---------------------------------------------------------------------------------------------------
// The rows of tiles of several pieces, a warp each, eight rows of a tile and head to a CTA (the first eight of
// all, then the next: tiles of few rows leave nothing behind them); zeros for the tokens of no request.
// ---------------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 256;

template <typename TI>
__global__ void __launch_bounds__(kJoinThreads)
    join_kernel(const __grid_constant__ ChunkProblem p, const __grid_constant__ Plan w) {
  pdl_wait_and_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = p.H / p.Hk;
  const int heads = w.head[1] * p.Hk;  // tiles of several pieces, and heads
  const long long groups = (long long)heads * w.head[2];
  for (long long e = blockIdx.x; e < groups; e += gridDim.x) {
    const int at_head = (int)(e % heads), h = at_head % p.Hk, r = (int)(e / heads) * kJoinRows + warp;
    const Split t = w.split[at_head / p.Hk];
    if (r >= t.rows) continue;
    const int f = t.row0 + r, token = t.s0 + f / G, head = h * G + f % G, at = p.positions[token];
    const long long slot = t.slot + h * t.pieces;
    float4 st = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (lane < t.pieces) st = w.stats[(slot + lane) * w.rows + r];
    if (at < 0 || at >= p.limit) continue;  // (zeros have been written)
    const TI* V = static_cast<const TI*>(p.v) + page_row(p, p.table + (long long)t.b * p.t_stride, at, h);
    float v[4], z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = lane + 32 * c < p.d ? (float)V[lane + 32 * c] : 0.f;
    float m = st.x, l = 0.f, u_self = 0.f;
    for (int k = lane + 32; k < t.pieces; k += 32) m = fmaxf(m, w.stats[(slot + k) * w.rows + r].x);
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    for (int k0 = 0; k0 < t.pieces; k0 += 32) {
      if (k0 > 0) {
        st = make_float4(-INFINITY, 0.f, 0.f, 0.f);
        if (k0 + lane < t.pieces) st = w.stats[(slot + k0 + lane) * w.rows + r];
      }
      // no key seen: 0; m is -inf too where every score is NaN (l NaN): NaN
      const float wt = st.x == -INFINITY ? 0.f * st.y : ex2_approx(st.x - m);
      const unsigned who = __ballot_sync(0xffffffffu, st.w != 0.f);
      if (who) u_self = __shfl_sync(0xffffffffu, st.z, __ffs(who) - 1);
      const int n = min(32, t.pieces - k0);
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float f = __shfl_sync(0xffffffffu, wt, k), lk = __shfl_sync(0xffffffffu, st.y, k);
        if (lk == 0.f) continue;  // (and no z there)
        l = fmaf(f, lk, l);
        const float* src = w.z + ((slot + k0 + k) * w.rows + r) * w.width;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (lane + 32 * c < p.d) z[c] = fmaf(f, src[lane + 32 * c], z[c]);
      }
    }
    const Mix mix(p, m, l, u_self, at);
    TI* y = static_cast<TI*>(p.out) + (long long)token * p.qsT + (long long)head * p.qsH;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (lane + 32 * c < p.d) y[lane + 32 * c] = (TI)mix.y(z[c], v[c]);
    if (lane == 0) p.logz[(long long)token * p.H + head] = mix.logz;
  }
  const long long first = ((long long)blockIdx.x * kJoinThreads + threadIdx.x) >> 5,
                  step = (long long)gridDim.x * (kJoinThreads / 32);
  const int before = min(max(p.starts[0], 0), p.N), after = min(max(p.starts[p.B], before), p.N);
  const long long none = (long long)(before + p.N - after) * p.H;
  for (long long e = first; e < none; e += step) {
    const int i = (int)(e / p.H), head = (int)(e % p.H), token = i < before ? i : after + i - before;
    TI* y = static_cast<TI*>(p.out) + (long long)token * p.qsT + (long long)head * p.qsH;
    for (int c = lane; c < p.d; c += 32) y[c] = (TI)0.f;
    if (lane == 0) p.logz[(long long)token * p.H + head] = -INFINITY;
  }
}

// ---------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------
// The plan's arrays in a workspace; the bytes of it
size_t carve(Plan* w, uint8_t* base, int N, int B, int H, int Hk, int d, int limit, relation_dtype dt) {
  // (as many pieces as CTAs fit the GPU; fp32, whose units take long, twice as many and shorter ones,
  // of one unit at least: 451 tokens of 8 x 72 take 42 us, with two units at least 47)
  w->tile = dt == RELATION_F32 ? SM_ROWS : BM;
  w->target = dt == RELATION_F32 ? 608 : 304;
  w->least = dt == RELATION_F32 ? 1 : 4;
  const long long G = H / Hk, rows = N * G;
  // a request of n rows has ceil(n / tile) tiles, and no more requests than tokens have any
  const long long tiles = (rows + (long long)(B < N ? B : N) * (w->tile - 1)) / w->tile + 1;
  const long long units = ((long long)limit + kUnit - 1) / kUnit;
  const long long most = (units + w->least - 1) / w->least;  // pieces of a tile
  // Pieces are as long as the mean of `target` pieces at least: all tiles have one and `target` more are
  // enough for the rest; a tile of several has them longer than half of that mean.
  const long long items = tiles * Hk + (tiles * Hk * (most - 1) < w->target ? tiles * Hk * (most - 1) : w->target);
  long long slots = 2LL * w->target;
  if (tiles * Hk * most < slots) slots = tiles * Hk * most;
  const long long split = tiles < slots ? tiles : slots;
  w->max_tiles = (int)tiles;
  w->max_items = (int)items;
  w->max_split = (int)split;
  w->small = tiles <= 32 && B <= 32;
  w->slots = most > 1 ? (int)slots : 0;
  w->rows = rows < w->tile ? (int)rows : w->tile;
  w->width = (d + 3) & ~3;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* x = base + at;
    at += (bytes + 15) & ~(size_t)15;
    return x;
  };
  w->head = reinterpret_cast<int*>(take(16));
  w->first = reinterpret_cast<int*>(take((size_t)(B + 1) * 4));
  w->tiles = reinterpret_cast<int4*>(take((size_t)tiles * 16));
  w->upto = reinterpret_cast<int2*>(take((size_t)(tiles + 1) * 8));
  w->split = reinterpret_cast<Split*>(take((size_t)split * sizeof(Split)));
  w->items = reinterpret_cast<Item*>(take((size_t)items * sizeof(Item)));
  w->stats = reinterpret_cast<float4*>(take((size_t)w->slots * w->rows * 16));
  w->z = reinterpret_cast<float*>(take((size_t)w->slots * w->rows * w->width * 4));
  return at;
}

template <typename K, typename... A>
cudaError_t launch_main(K kernel, int threads, int smem, const Plan& w, cudaStream_t s, const A&... args) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(w.max_items), threads, smem, s, 1, args...);
  if (e != cudaSuccess) note_failure("chunk: launch");
  return e;
}

// 4-D map over pages [n_pages][page][Hk][d] of bf16: boxes of 64 columns and `rows` rows of one head and
// page, 128-byte swizzle, zeros past column d
bool make_map(CUtensorMap* m, const void* base, const ChunkProblem& p, int rows) {
  static const PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                                     &q) == cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ok ? ptr : nullptr);
  }();
  if (!encode) return false;
  // (the stride of a dimension of one entry is never used: any that the encoder takes)
  auto bytes = [](long long stride, int n) { return (cuuint64_t)(n > 1 ? stride * 2 : 16); };
  cuuint64_t dims[4] = {(cuuint64_t)p.d, (cuuint64_t)p.page, (cuuint64_t)p.Hk, (cuuint64_t)p.n_pages};
  cuuint64_t strides[3] = {bytes(p.sR, p.page), bytes(p.sC, p.Hk), bytes(p.sP, p.n_pages)};
  cuuint32_t sizes[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, sizes, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch_tc(const ChunkProblem& p, const Plan& w, bool groups, cudaStream_t s) {
  // Boxes as large as pages and units allow: a power of two that divides both, or where that is 8 (whose
  // boxes alone would bound the kernel: 48 requests in pages of 24 rows of 80 bf16 518 us in eights, 390 so) a
  // page, or 32 rows of a large one, and eights for what is left.
  int big = kUnit;
  while (p.page % big) big /= 2;
  if (big == 8) big = p.page < kUnit ? p.page : 32;
  const bool eights = p.page % big != 0 || kUnit % big != 0;  // (boxes of 8 are used beside the big ones)
  CUtensorMap m[4] = {};
  if (groups && p.page % 8 == 0 && make_map(&m[0], p.k, p, big) && make_map(&m[1], p.v, p, big) &&
      (!eights || (make_map(&m[2], p.k, p, 8) && make_map(&m[3], p.v, p, 8))))
    return launch_main(chunk_tc_kernel<D, kBoxes>, Cfg<D>::THREADS, Cfg<D>::SMEM, w, s, m[0], m[1], m[2], m[3], p,
                       w, big);
  if (groups)
    return launch_main(chunk_tc_kernel<D, kGroups>, Cfg<D>::THREADS, Cfg<D>::SMEM, w, s, m[0], m[1], m[2], m[3], p,
                       w, 0);
  return launch_main(chunk_tc_kernel<D, kElements>, Cfg<D>::THREADS, Cfg<D>::SMEM, w, s, m[0], m[1], m[2], m[3], p,
                     w, 0);
}

template <int D>
cudaError_t launch_simt(const ChunkProblem& p, const Plan& w, bool groups, cudaStream_t s) {
  constexpr int smem = (int)sizeof(SimtSmem<D>);
  return groups ? launch_main(chunk_simt_kernel<D, true>, kSimtThreads, smem, w, s, p, w)
                : launch_main(chunk_simt_kernel<D, false>, kSimtThreads, smem, w, s, p, w);
}

}  // namespace chunk

size_t chunk_workspace_bytes(int N, int B, int H, int Hk, int d, int limit, relation_dtype dt) {
  chunk::Plan w;
  return chunk::carve(&w, nullptr, N, B, H, Hk, d, limit, dt);
}

cudaError_t launch_chunk(ChunkProblem p, void* workspace, cudaStream_t s) {
  using namespace chunk;
  page_division(p.page, &p.page_mul, &p.page_shift);
  Plan w;
  carve(&w, static_cast<uint8_t*>(workspace), p.N, p.B, p.H, p.Hk, p.d, p.limit, p.dtype);
  cudaError_t e = cudaSuccess;
  if (!w.small) {
    // as many threads as requests or tiles want, in whole warps
    int threads = 128;
    while (threads < kPlanThreads && (threads < w.max_tiles || threads < p.B)) threads *= 2;
    e = launch_pdl(plan_kernel, dim3(1), (unsigned)threads, 0, s, 1, p, w);
  }
  if (e != cudaSuccess) {
    note_failure("chunk: plan launch");
    return e;
  }
  const int es = p.dtype == RELATION_F32 ? 4 : 2;
  uintptr_t low = 0;
  for (const void* x : {p.q, p.k, p.v, (const void*)p.out}) low |= reinterpret_cast<uintptr_t>(x);
  for (long long x : {p.N > 1 ? p.qsT : 0, p.H > 1 ? p.qsH : 0, p.n_pages > 1 ? p.sP : 0,
                      p.page > 1 ? p.sR : 0, p.Hk > 1 ? p.sC : 0, (long long)p.d})
    low |= (uintptr_t)(x * es);
  const bool groups = low % 16 == 0;
  e = p.dtype == RELATION_BF16 ? (p.d <= 64 ? launch_tc<64>(p, w, groups, s) : launch_tc<128>(p, w, groups, s))
                               : (p.d <= 32   ? launch_simt<32>(p, w, groups, s)
                                  : p.d <= 64 ? launch_simt<64>(p, w, groups, s)
                                  : p.d <= 96 ? launch_simt<96>(p, w, groups, s)
                                              : launch_simt<128>(p, w, groups, s));
  if (e != cudaSuccess) return e;
  e = p.dtype == RELATION_F32 ? launch_pdl(join_kernel<float>, dim3(304), kJoinThreads, 0, s, 1, p, w)
                              : launch_pdl(join_kernel<__nv_bfloat16>, dim3(304), kJoinThreads, 0, s, 1, p, w);
  if (e != cudaSuccess) note_failure("chunk: join launch");
  return e;
}

}  // namespace rel
