// relation_append.cu -- new tokens into a paged key/value cache: the layer's transforms
// (relation_layer.cu) at every token's own position, the results written where they are read from.
//
//   q_t = RoPE(p1_t, m_t),  K[slot_t] = RoPE(p2_t, m_t),  V[slot_t] = Givens(info_t)
// with channel pair c of position m turned by m * base^(-2c/d) and head pairs mixed by theta.  A
// slot names a page and a row in it; a token without a slot (padding) writes no cache row and a
// zero query.
//
// Bound by memory: three reads and three writes of N H d elements.  As in the layer's pass the
// rotations and the mixing are CTAs of their own, the angles of a CTA's tokens are tabulated once
// for all heads, and each thread has two items' loads in flight, the first during the tables.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "layer.cuh"

namespace rel {
namespace append {

using layer::kTurnPositions;
using layer::turn;

constexpr int kThreads = 128;
constexpr int kMaxD = 256;

// The problem and the frequencies base^(-2c/d), in fp64 and as sums of two floats.
struct Args {
  AppendProblem p;
  double w[kMaxD / 2];
  float w_hi[kMaxD / 2], w_lo[kMaxD / 2];
};

// CH consecutive elements as fp32: 8 (16-byte groups, aligned rows), 2 or 1 (any alignment)
template <typename TI, int CH>
struct Group {
  struct Raw {
    TI x[CH];
  };
  static __device__ __forceinline__ Raw load(const TI* p) {
    Raw r;
#pragma unroll
    for (int i = 0; i < CH; ++i) r.x[i] = p[i];
    return r;
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[CH]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) x[i] = (float)r.x[i];
  }
  static __device__ __forceinline__ void store(TI* p, const float (&x)[CH]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) p[i] = (TI)x[i];
  }
};
template <typename TI>
struct Group<TI, 8> : layer::Vec8<TI> {};

// Where a CTA's tokens go: element offset of the cache row, -1 for none.
template <int TOK>
__device__ __forceinline__ void fill_rows(long long (&row)[TOK], const AppendProblem& p, int t0,
                                          bool report) {
  if (threadIdx.x < TOK) {
    const int t = t0 + (int)threadIdx.x;
    const long long slot = t < p.N ? p.slots[t] : -1;
    const bool in = slot >= 0 && slot < (long long)p.n_pages * p.page;
    if (slot >= 0 && !in && report && p.dev_status)
      atomicExch(p.dev_status, (int)RELATION_ERR_INVALID_ARG);
    row[threadIdx.x] = in ? slot / p.page * p.sP + slot % p.page * p.sR : -1;
  }
}

template <typename TI, int CH, int TOK>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ Args ar) {
  using G = Group<TI, CH>;
  __shared__ long long row[TOK];
  const AppendProblem& p = ar.p;
  const int t0 = (int)(blockIdx.x >> 1) * TOK, nt = min(TOK, p.N - t0), nu = p.d / CH;
  pdl_wait_and_launch();
  if (!(blockIdx.x & 1)) {  // q = RoPE(p1), K = RoPE(p2)
    __shared__ float cs[TOK][kMaxD / 2], sn[TOK][kMaxD / 2];
    const int n = nt * p.H * nu;
    struct Item {
      long long in, out;  // element offsets in a token's and in a cache row's tensor
      int tt, u;
    };
    auto item = [&](int e) {  // (clamped: a thread past the end reloads the last item)
      e = min(e, n - 1);
      const int r = e / nu, h = r % p.H, tt = r / p.H, u = e - r * nu;
      return Item{(long long)(t0 + tt) * p.sT + (long long)h * p.sH + CH * u,
                  (long long)h * p.sC + CH * u, tt, u};
    };
    const TI* in1 = reinterpret_cast<const TI*>(p.p1);
    const TI* in2 = reinterpret_cast<const TI*>(p.p2);
    auto put = [&](const Item& i, const typename G::Raw& a, const typename G::Raw& b) {
      float x[CH], y[CH];
      G::unpack(a, x);
      G::unpack(b, y);
      if constexpr (CH > 1) {
        if (p.rope_base > 0.f) {
#pragma unroll
          for (int j = 0; j < CH / 2; ++j) {
            const float c = cs[i.tt][CH / 2 * i.u + j], s = sn[i.tt][CH / 2 * i.u + j];
            const float x0 = x[2 * j], x1 = x[2 * j + 1], y0 = y[2 * j], y1 = y[2 * j + 1];
            x[2 * j] = x0 * c - x1 * s;
            x[2 * j + 1] = x0 * s + x1 * c;
            y[2 * j] = y0 * c - y1 * s;
            y[2 * j + 1] = y0 * s + y1 * c;
          }
        }
      }
      const long long at = row[i.tt];
      if (at < 0) {
#pragma unroll
        for (int j = 0; j < CH; ++j) x[j] = 0.f;
      } else {
        G::store(reinterpret_cast<TI*>(p.k) + at + i.out, y);
      }
      if (p.q) G::store(reinterpret_cast<TI*>(p.q) + i.in, x);
    };
    Item i0 = item(threadIdx.x), i1 = item(threadIdx.x + kThreads);
    // (without queries the keys stand in for them: loaded, not stored)
    if (!p.q) in1 = in2;
    typename G::Raw x0 = G::load(in1 + i0.in), y0 = G::load(in2 + i0.in);
    typename G::Raw x1 = G::load(in1 + i1.in), y1 = G::load(in2 + i1.in);
    fill_rows<TOK>(row, p, t0, true);
    if (p.rope_base > 0.f) {
      const int half = p.d / 2;
      for (int e = threadIdx.x; e < nt * half; e += kThreads) {
        const int tt = e / half, c = e - tt * half, m = p.positions[t0 + tt];
        float r;
        if (m < kTurnPositions && m >= 0 && p.rope_base >= 1.f) {
          r = turn((float)m, ar.w_hi[c], ar.w_lo[c]);
        } else {
          const double a = (double)m * ar.w[c];
          r = (float)fma(-rint(a * 0.15915494309189533576888376337251),
                         6.283185307179586476925286766559, a);
        }
        float s, co;
        sincosf(r, &s, &co);
        cs[tt][c] = co;
        sn[tt][c] = s;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += 2 * kThreads) {
      if (e != (int)threadIdx.x) {
        i0 = item(e);
        i1 = item(e + kThreads);
        x0 = G::load(in1 + i0.in);
        y0 = G::load(in2 + i0.in);
        x1 = G::load(in1 + i1.in);
        y1 = G::load(in2 + i1.in);
      }
      put(i0, x0, y0);
      if (e + kThreads < n) put(i1, x1, y1);
    }
    return;
  }
  // V = Givens(info): (token, head pair, chunk) items; without theta every head by itself
  fill_rows<TOK>(row, p, t0, false);
  __syncthreads();
  const bool mix = p.theta != nullptr;
  const int np = mix ? p.H / 2 : p.H, n = nt * np * nu;
  const TI* in = reinterpret_cast<const TI*>(p.info);
  TI* out = reinterpret_cast<TI*>(p.v);
  for (int e0 = threadIdx.x; e0 < n; e0 += 2 * kThreads) {
    typename G::Raw ra[2], rb[2];
    int ha[2], hb[2], tt[2], col[2];
    float th[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = min(e0 + i * kThreads, n - 1);
      const int r = e / nu, k = r % np;
      tt[i] = r / np;
      col[i] = CH * (e - r * nu);
      ha[i] = !mix ? k : p.pairing == 0 ? 2 * k : 2 * k + 1;
      hb[i] = !mix ? k : p.pairing == 0 ? 2 * k + 1 : (2 * k + 2) % p.H;
      const TI* src = in + (long long)(t0 + tt[i]) * p.sT + col[i];
      ra[i] = G::load(src + (long long)ha[i] * p.sH);
      rb[i] = G::load(src + (long long)hb[i] * p.sH);
      th[i] = mix ? p.theta[k] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (e0 + i * kThreads >= n) break;
      const long long at = row[tt[i]];
      if (at < 0) continue;
      float a[CH], b[CH];
      G::unpack(ra[i], a);
      G::unpack(rb[i], b);
      TI* to = out + at + col[i];
      if (mix) {
        float s, co, va[CH], vb[CH];
        sincosf(th[i], &s, &co);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          va[j] = co * a[j] - s * b[j];
          vb[j] = s * a[j] + co * b[j];
        }
        G::store(to + (long long)ha[i] * p.sC, va);
        G::store(to + (long long)hb[i] * p.sC, vb);
      } else {
        G::store(to + (long long)ha[i] * p.sC, a);
      }
    }
  }
}

template <typename TI, int CH, int TOK>
cudaError_t launch_tok(const Args& ar, cudaStream_t s) {
  const int tiles = ar.p.N / TOK + (ar.p.N % TOK != 0);
  const cudaError_t e =
      launch_pdl(append_kernel<TI, CH, TOK>, dim3(2u * tiles), kThreads, 0, s, 1, ar);
  if (e != cudaSuccess) note_failure("cache append: launch");
  return e;
}

template <typename TI, int CH>
cudaError_t launch_ch(const Args& ar, cudaStream_t s) {
  // Tokens that share a CTA's set-up (row lookups, angles): few where the grid is short, whose time is
  // one CTA's, more where the CTAs come in rounds.  us with 1, 2, 4, 8 tokens, one call after the other
  // in a graph: 262 tokens of 8 x 96 bf16 3.0, 2.8, 3.6, 4.9; 1832 of 12 x 96 8.6, 7.4, 9.0, 10.5;
  // 1821 of 2 x 32 6.5, 4.6, 2.9, 2.8; 11720 of 8 x 48 38, 23, 15, 14; 32768 of 16 x 128 152, 129,
  // 125, 126 (6.4 TB/s).
  const long long items = (long long)ar.p.H * (ar.p.d / CH), want = ar.p.N * items <= 400000 ? 160 : 1024;
  if (items >= want) return launch_tok<TI, CH, 1>(ar, s);
  if (2 * items >= want) return launch_tok<TI, CH, 2>(ar, s);
  if (4 * items >= want) return launch_tok<TI, CH, 4>(ar, s);
  return launch_tok<TI, CH, 8>(ar, s);
}

template <typename TI>
cudaError_t launch_t(const Args& ar, cudaStream_t s) {
  const AppendProblem& p = ar.p;
  uintptr_t low = 0;
  for (const void* x : {p.p1, p.p2, p.info, (const void*)p.q, (const void*)p.k, (const void*)p.v})
    low |= reinterpret_cast<uintptr_t>(x);
  for (long long x : {p.sT, p.sH, p.sP, p.sR, p.sC}) low |= (uintptr_t)(x * (long long)sizeof(TI));
  if (low % 16 == 0 && p.d % 8 == 0) return launch_ch<TI, 8>(ar, s);
  if (p.d % 2 == 0) return launch_ch<TI, 2>(ar, s);
  return launch_ch<TI, 1>(ar, s);
}

}  // namespace append

cudaError_t launch_append(const AppendProblem& p, cudaStream_t s) {
  append::Args ar;
  ar.p = p;
  if (p.rope_base > 0.f) {
    const double step = -2.0 / (double)p.d * log((double)p.rope_base);
    for (int c = 0; c < p.d / 2; ++c) {
      ar.w[c] = exp(step * (double)c);
      ar.w_hi[c] = (float)ar.w[c];
      ar.w_lo[c] = (float)(ar.w[c] - (double)ar.w_hi[c]);
    }
  }
  if (p.dtype == RELATION_F32) return append::launch_t<float>(ar, s);
  return append::launch_t<__nv_bfloat16>(ar, s);
}

}  // namespace rel
