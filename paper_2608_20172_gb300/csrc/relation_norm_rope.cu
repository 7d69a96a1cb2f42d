// relation_norm_rope.cu -- queries and keys normed per head and rotated by their positions, and the
// gradient.
//
// A head's row x of d channels at position m:
//   r = 1 / sqrt(mean x^2 + eps),  n_c = x_c r w_c,
//   the first d_rot channels in pairs (a, b) turned by m f_p and scaled:
//   a' = s (a cos - b sin),  b' = s (a sin + b cos);  the pairs (2p, 2p + 1) or (p, p + d_rot / 2).
// Backward, with u = the transposed turn of dy and x^ = x r:
//   dw_c = sum over the rows of u_c x^_c,  dx = r (w u - x^ mean(x^ w u)).
//
// The angle is kept as a part of a whole turn in 64-bit integers: f / (2 pi) modulo 1 times 2^64, times
// the position, modulo 2^64: no reduction by 2 pi and no fp64.  The step of a position is off by less than 2^-64 of
// a turn, the angle at the last one by 2^-33 of a turn, far below fp32's rounding (a product in fp64 is off by 2^-53
// of f, times the position; its rounding carried along in fp64 too took 1 us more a call).
//
// Bound by memory: a row is read and written once (backward: two reads).  A few lanes share a row, 16
// bytes of two parts of it each, so that both channels of a pair are in one lane in either layout and
// the sums are a few shuffles; a token's turns are taken once for all heads.  Four CTAs of 128 threads an SM
// (three: 134 us in the first case below, five, which leave registers for one row in flight a lane: 141); the
// bf16 gradient spills 40 to 72 bytes for it.  Measured: 32768 tokens of 32 + 8 heads of 128 bf16 118 us, 5.7
// TB/s (16384 fp32 109); the gradient of 16384 tokens of 16 + 16 heads 84 us, 4.8 TB/s (fp32 139); 32 tokens of
// 12 + 12 heads of 64 3.3 us, one chain of position, turn and row.
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace normrope {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kMaxD = 256;
constexpr int kMaxParts = 608;  // CTAs at most (four an SM), each of which leaves a partial sum of dw backward

// GE consecutive elements: 16 bytes of an aligned row, or one element
template <typename TI, int GE>
struct Group {
  struct Raw {
    TI x;
  };
  static __device__ __forceinline__ Raw load(const TI* p) { return Raw{*p}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[1]) { x[0] = (float)r.x; }
  static __device__ __forceinline__ void store(TI* p, const float (&x)[1]) { *p = (TI)x[0]; }
};
template <>
struct Group<__nv_bfloat16, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw load(const __nv_bfloat16* p) {
    return *reinterpret_cast<const uint4*>(p);
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};
template <>
struct Group<float, 4> {
  using Raw = float4;
  static __device__ __forceinline__ Raw load(const float* p) {
    return *reinterpret_cast<const float4*>(p);
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[4]) {
    x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
};

// What a lane holds of a row: IT times two groups, at channels a and b (-1: none), and the first pair
// of each in the table.  ACROSS: pair j is (a + j, b + j); else a group holds whole pairs.
template <int GE, bool ACROSS, int IT>
struct Place {
  int a[IT], b[IT], pa[IT], pb[IT];
  __device__ __forceinline__ Place(int i0, int lanes, int d, int d_rot, bool half) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int i = i0 + it * lanes;
      if (ACROSS) {
        const int n = d_rot / 2 / GE, j = i - n;
        a[it] = j >= 0 ? d_rot + 2 * j * GE : half ? i * GE : 2 * i;
        b[it] = j >= 0 ? a[it] + GE : half ? i * GE + d_rot / 2 : 2 * i + 1;
        pa[it] = pb[it] = j >= 0 ? -1 : i * GE;
      } else {
        const int n = (d / GE + 1) / 2;
        a[it] = i < n ? i * GE : d;
        b[it] = i < n ? (i + n) * GE : d;
        pa[it] = a[it] / 2 < d_rot / 2 ? a[it] / 2 : -1;
        pb[it] = b[it] / 2 < d_rot / 2 ? b[it] / 2 : -1;
      }
      if (a[it] >= d) a[it] = -1;
      if (b[it] >= d) b[it] = -1;
    }
  }
};

__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Two channels at a time: the packed fp32 instructions take the place of two
__device__ __forceinline__ float2 two(float a, float b) { return make_float2(a, b); }
template <int GE, typename F>
__device__ __forceinline__ void each2(F f) {  // f(j) for channels j, j + 1
#pragma unroll
  for (int j = 0; j < GE; j += 2) f(j);
}

// A lane's two groups, at channels a and b, turned (sign 1) or turned back (-1) by their pairs' (cos, sin).
// Channels from d_rot on are left alone: a turn by 0 would multiply an infinite or NaN neighbour by 0.
template <int GE, bool ACROSS>
__device__ __forceinline__ void turned(float (&x)[GE], float (&y)[GE], const float2 (&cs)[GE], float sign, int at,
                                       int bt, int d_rot) {
  const bool is = at < d_rot;
  if constexpr (GE == 1) {
    const float s = cs[0].y * sign, a = x[0], b = y[0];
    x[0] = is ? a * cs[0].x - b * s : a;
    y[0] = is ? a * s + b * cs[0].x : b;
  } else if constexpr (ACROSS) {
    each2<GE>([&](int j) {
      const float2 c = two(cs[j].x, cs[j + 1].x), s = two(cs[j].y * sign, cs[j + 1].y * sign);
      const float2 a = two(x[j], x[j + 1]), b = two(y[j], y[j + 1]);
      const float2 u = __ffma2_rn(two(-b.x, -b.y), s, __fmul2_rn(a, c));
      const float2 v = __ffma2_rn(a, s, __fmul2_rn(b, c));
      x[j] = is ? u.x : a.x; x[j + 1] = is ? u.y : a.y;  // (selected: a branch took 94 us for 89)
      y[j] = is ? v.x : b.x; y[j + 1] = is ? v.y : b.y;
    });
  } else {
#pragma unroll
    for (int j = 0; j < GE; ++j) {
      float(&v)[GE] = j < GE / 2 ? x : y;
      const int e = 2 * (j < GE / 2 ? j : j - GE / 2);
      if ((j < GE / 2 ? at : bt) + e >= d_rot) continue;
      const float s = cs[j].y * sign;
      const float2 u = __ffma2_rn(two(v[e + 1], v[e]), two(-s, s), __fmul2_rn(two(v[e], v[e + 1]), two(cs[j].x, cs[j].x)));
      v[e] = u.x;
      v[e + 1] = u.y;
    }
  }
}

// The parts of a turn that a position adds to the angles of a lane's pairs of a table, 2^-64 each: pairs
// lane, lane + 32, ...
struct Steps {
  unsigned long long s[kMaxD / 64];
  // f / (2 pi) modulo 1: f's 53 bits times 1 / (2 pi) in 128 (after Payne and Hanek), the 64 bits behind the point;
  // off by 2^-64 + f 2^-128 of a turn, frequencies of 2^117 and more count as 0
  static __device__ __forceinline__ unsigned long long part(double f) {
    constexpr unsigned long long C1 = 0x28be60db9391054aull, C0 = 0x7f09d5f47d4d3770ull;
    const unsigned long long bits = (unsigned long long)__double_as_longlong(f);
    const int e = (int)(bits >> 52) & 0x7ff, shift = 1139 - max(e, 1), word = shift >> 6, k = shift & 63;
    const unsigned long long m = (bits & 0xfffffffffffffull) | (e ? 1ull << 52 : 0ull);  // f = m 2^(64 - shift)
    const unsigned long long l1 = m * C1, w0 = m * C0, w1 = __umul64hi(m, C0) + l1,
                             w2 = __umul64hi(m, C1) + (w1 < l1);
    const unsigned long long lo = word == 0 ? w0 : word == 1 ? w1 : word == 2 ? w2 : 0ull;
    const unsigned long long hi = word == 0 ? w1 : word == 1 ? w2 : 0ull;
    const unsigned long long r = k ? lo >> k | hi << (64 - k) : lo;
    return bits >> 63 ? 0ull - r : r;
  }
  __device__ __forceinline__ Steps(const NormRopeProblem& p, int lane) {
#pragma unroll
    for (int i = 0; i < kMaxD / 64; ++i) {
      s[i] = 0;
      if (lane + 32 * i < p.d_rot / 2) s[i] = part(p.freqs[lane + 32 * i]);
    }
  }
};

// The turns (cos, sin) s of one token, by its warp; pairs past the last one of a group that the turned
// part ends in stay as they are.
__device__ __forceinline__ void fill_turns(float2* turn, int pos, const Steps& st, const NormRopeProblem& p,
                                           int lane) {
  const int half = p.d_rot / 2, n = min(p.d / 2, (half + 3) & ~3);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kMaxD / 64; ++i) {
    const int c = lane + 32 * i;
    if (c < n) {
      const unsigned long long at = (unsigned long long)pos * st.s[i];
      float s, co;
      sincospif((float)(int)(at >> 32) * 0x1p-31f, &s, &co);
      turn[c] = c < half ? make_float2(co * p.scale, s * p.scale) : make_float2(1.f, 0.f);
    }
  }
  __syncwarp();
}

// Forward, and with GRAD backward.  A warp takes whole tokens, 32 / lanes of a token's heads at a time, first
// all its tokens' queries, then the keys: a lane's weights stay in registers, its turns for a token's heads,
// and backward its columns' dw.  With few tokens (gridDim.y > 1) a CTA takes one part of its tokens' heads,
// `per` of them: `pq` parts of the queries, then the keys'.
template <typename TI, int GE, bool ACROSS, int IT, bool GRAD>
__global__ void __launch_bounds__(kThreads, 4)
    norm_rope_kernel(const __grid_constant__ NormRopeProblem p, int lanes, int pq, int per) {
  using G = Group<TI, GE>;
  constexpr int U = GRAD ? 1 : 2;  // rows of a lane at a time; the next ones are on their way
  __shared__ __align__(16) float2 turns[kWarps][kMaxD / 2];
  __shared__ float sums[kWarps][GRAD ? kMaxD : 1];
  pdl_wait_and_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int N = p.B * p.T, slots = 32 / lanes, slot = lane / lanes;
  const Place<GE, ACROSS, IT> at(lane % lanes, lanes, p.d, p.d_rot, p.half);
  const Steps steps(p, lane);
  float2* turn = turns[warp];
  const float inv_d = 1.f / (float)p.d;
  struct Rows {
    typename G::Raw x[U][2][IT], y[GRAD ? U : 1][2][IT];
  };
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    int h_lo = 0, h_hi = which ? p.H[1] : p.H[0];  // this CTA's heads
    if (gridDim.y > 1) {
      const int part = (int)blockIdx.y - (which ? pq : 0);
      h_lo = part * per;
      h_hi = part < 0 || (!which && part >= pq) ? h_lo : min(h_hi, h_lo + per);
    }
    const TI* in = static_cast<const TI*>(which ? p.in[1] : p.in[0]);
    const TI* din = static_cast<const TI*>(which ? p.dout[1] : p.dout[0]);
    TI* out = static_cast<TI*>(which ? p.out[1] : p.out[0]);
    const float* wp = which ? p.w[1] : p.w[0];
    const long long sB = which ? p.sB[1] : p.sB[0], sT = which ? p.sT[1] : p.sT[0],
                    sH = which ? p.sH[1] : p.sH[0];
    float w[2][IT][GE], acc[2][IT][GE];
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int j = 0; j < GE; ++j) {
        w[0][it][j] = wp && h_lo < h_hi && at.a[it] >= 0 ? wp[at.a[it] + j] : 1.f;
        w[1][it][j] = wp && h_lo < h_hi && at.b[it] >= 0 ? wp[at.b[it] + j] : 1.f;
        acc[0][it][j] = acc[1][it][j] = 0.f;
      }
    auto fetch = [&](long long base, int h, Rows& r) {  // (zeros for lanes past the last head)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool live = h + u * slots < h_hi;
        const long long off = base + (long long)(h + u * slots) * sH;
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int side = 0; side < 2; ++side) {
            const int c = side ? at.b[it] : at.a[it];
            r.x[u][side][it] = typename G::Raw{};
            if (GRAD) r.y[u][side][it] = typename G::Raw{};
            if (c < 0 || !live) continue;
            r.x[u][side][it] = G::load(in + off + c);
            if (GRAD) r.y[u][side][it] = G::load(din + off + c);
          }
      }
    };
    auto token = [&](int n, long long& base, int& pos) {
      const int b = n / p.T, t = n - b * p.T;
      base = (long long)b * sB + (long long)t * sT;
      pos = p.positions ? p.positions[n] : t;
    };
    Rows now, next;
    const int step = (int)gridDim.x * kWarps;
    long long base = 0, base2 = 0;
    int pos = 0, pos2 = 0, n = h_lo < h_hi ? (int)blockIdx.x * kWarps + warp : N;
    if (n < N) {
      token(n, base, pos);
      fetch(base, h_lo + slot, now);
    }
    for (; n < N; n += step, base = base2, pos = pos2) {
      const bool more = n + step < N;
      if (more) token(n + step, base2, pos2);
      if (pos < 0) {  // padding
        for (int h = h_lo + slot; h < h_hi; h += slots)
#pragma unroll
          for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int side = 0; side < 2; ++side) {
              const int c = side ? at.b[it] : at.a[it];
              const float zero[GE] = {};
              if (c >= 0) G::store(out + base + (long long)h * sH + c, zero);
            }
        if (more) fetch(base2, h_lo + slot, now);
        continue;
      }
      fill_turns(turn, pos, steps, p, lane);
      float2 cs[IT][GE];  // ACROSS: of the pairs (a + j, b + j); else a's pairs, then b's
#pragma unroll
      for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int j = 0; j < GE; ++j) {
          const int first = ACROSS || j < GE / 2 ? at.pa[it] : at.pb[it] - GE / 2;
          const bool is = ACROSS || j < GE / 2 ? at.pa[it] >= 0 : at.pb[it] >= 0;
          cs[it][j] = is ? turn[first + j] : make_float2(1.f, 0.f);
        }
#pragma unroll 1
      for (int h0 = h_lo; h0 < h_hi; h0 += U * slots) {
        if (h0 + U * slots < h_hi) {
          fetch(base, h0 + U * slots + slot, next);
        } else if (more) {
          fetch(base2, h_lo + slot, next);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u * slots + slot;
          float x[2][IT][GE], y[2][IT][GE];
          float2 ss2 = two(0.f, 0.f), dot2 = ss2;
#pragma unroll
          for (int it = 0; it < IT; ++it) {
#pragma unroll
            for (int side = 0; side < 2; ++side) {
              G::unpack(now.x[u][side][it], x[side][it]);
              if (GRAD) G::unpack(now.y[GRAD ? u : 0][side][it], y[side][it]);
            }
            if (GRAD) turned<GE, ACROSS>(y[0][it], y[1][it], cs[it], -1.f, at.a[it], at.b[it], p.d_rot);
            if constexpr (GE == 1) {
              const float2 v = two(x[0][it][0], x[1][it][0]);
              ss2 = __ffma2_rn(v, v, ss2);
              if (GRAD)
                dot2 = __ffma2_rn(__fmul2_rn(v, two(w[0][it][0], w[1][it][0])), two(y[0][it][0], y[1][it][0]), dot2);
            } else {
#pragma unroll
              for (int side = 0; side < 2; ++side)
                each2<GE>([&](int j) {
                  const float2 v = two(x[side][it][j], x[side][it][j + 1]);
                  ss2 = __ffma2_rn(v, v, ss2);
                  if (GRAD)
                    dot2 = __ffma2_rn(__fmul2_rn(v, two(w[side][it][j], w[side][it][j + 1])),
                                      two(y[side][it][j], y[side][it][j + 1]), dot2);
                });
            }
          }
          const bool live = h < h_hi;
          float r = 1.f, mean = 0.f;
          if (p.norm) {
            const float ss = lanes_sum(ss2.x + ss2.y, lanes), dot = GRAD ? lanes_sum(dot2.x + dot2.y, lanes) : 0.f;
            r = rsqrtf(ss * inv_d + p.eps);
            if (GRAD) mean = dot * r * inv_d;  // mean of x^ w u
          }
          // (a lane past the last head adds 0 to dw; r may be infinite there)
          const float ra = GRAD && !live ? 0.f : r;
          TI* dst = out + base + (long long)h * sH;
#pragma unroll
          for (int it = 0; it < IT; ++it) {
#pragma unroll
            for (int side = 0; side < 2; ++side) {
              auto one = [&](float2 v, float2 wt, float2 u_, float2& sum) {
                const float2 xh = __fmul2_rn(v, two(ra, ra));
                if (!GRAD) return __fmul2_rn(xh, wt);
                sum = __ffma2_rn(u_, xh, sum);
                const float2 wu = __fmul2_rn(wt, u_);
                // (without the norm x has no part in dx, not even by 0)
                return p.norm ? __fmul2_rn(__ffma2_rn(xh, two(-mean, -mean), wu), two(ra, ra)) : wu;
              };
              if constexpr (GE == 1) {
                float2 sum = two(acc[side][it][0], 0.f);
                x[side][it][0] = one(two(x[side][it][0], 0.f), two(w[side][it][0], 0.f), two(y[side][it][0], 0.f), sum).x;
                acc[side][it][0] = sum.x;
              } else {
                each2<GE>([&](int j) {
                  float2 sum = two(acc[side][it][j], acc[side][it][j + 1]);
                  const float2 v = one(two(x[side][it][j], x[side][it][j + 1]), two(w[side][it][j], w[side][it][j + 1]),
                                       two(y[side][it][j], y[side][it][j + 1]), sum);
                  x[side][it][j] = v.x; x[side][it][j + 1] = v.y;
                  acc[side][it][j] = sum.x; acc[side][it][j + 1] = sum.y;
                });
              }
            }
            if (!GRAD) turned<GE, ACROSS>(x[0][it], x[1][it], cs[it], 1.f, at.a[it], at.b[it], p.d_rot);
#pragma unroll
            for (int side = 0; side < 2; ++side) {
              const int c = side ? at.b[it] : at.a[it];
              if (live && c >= 0) G::store(dst + c, x[side][it]);
            }
          }
        }
        now = next;
      }
    }
    if constexpr (GRAD) {
      if (!p.part) continue;
      // the CTA's sums: lanes of the same columns by shuffles, then the warps in order
      __syncthreads();
#pragma unroll
      for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          const int c = side ? at.b[it] : at.a[it];
#pragma unroll
          for (int j = 0; j < GE; ++j) {
            float x = acc[side][it][j];
            for (int o = 16; o >= lanes; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (lane < lanes && c >= 0) sums[warp][c + j] = x;
          }
        }
      __syncthreads();
      for (int c = threadIdx.x; c < p.d; c += kThreads) {
        float x = sums[0][c];
#pragma unroll
        for (int i = 1; i < kWarps; ++i) x += sums[i][c];
        p.part[((long long)(blockIdx.y * gridDim.x + blockIdx.x) * 2 + which) * p.d + c] = x;
      }
    }
  }
}

// dw from the CTAs' partial sums: 8 columns a CTA, 32 lots of the sums, in a fixed order (fp32: at most 19
// additions and 5 of pairs)
__global__ void __launch_bounds__(256) dw_kernel(const float* part, int n, int d, float* dw1, float* dw2) {
  constexpr int K = kMaxParts / 32;
  __shared__ float red[8][33];
  pdl_wait_and_launch();
  const int e = blockIdx.x * 8 + (threadIdx.x & 7), lot = threadIdx.x >> 3;
  float x[K], s = 0.f;
#pragma unroll
  for (int i = 0; i < K; ++i)  // (all loads at once)
    x[i] = e < 2 * d && lot + 32 * i < n ? part[(long long)(lot + 32 * i) * 2 * d + e] : 0.f;
#pragma unroll
  for (int i = 0; i < K; ++i) s += x[i];
  red[threadIdx.x & 7][lot] = s;
  __syncthreads();
  const int c = threadIdx.x >> 5, to = blockIdx.x * 8 + c;
  s = red[c][threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0 && to < 2 * d) {
    float* dw = to < d ? dw1 : dw2;
    if (dw) dw[to < d ? to : to - d] = s;
  }
}

template <typename TI, int GE, bool ACROSS, int IT>
cudaError_t launch_t(const NormRopeProblem& p, bool grad, cudaStream_t s) {
  // lanes of a row: its groups in twos (ACROSS: the turned ones and the others apart)
  const int half = p.d_rot / 2 / GE, rest = (p.d - (ACROSS ? p.d_rot : 0) + GE - 1) / GE;
  const int need = ACROSS ? half + (rest + 1) / 2 : (rest + 1) / 2;
  int lanes = 1;
  while (lanes < need && lanes < 32) lanes *= 2;
  // Few tokens: as many CTAs share a token's heads, in whole passes of a warp, as run at once
  const int tiles = (p.B * p.T + kWarps - 1) / kWarps, pass = (grad ? 1 : 2) * (32 / lanes);
  dim3 grid(tiles < kMaxParts ? tiles : kMaxParts);
  int per = 0, pq = 0;
  if (2 * tiles <= kMaxParts)
    for (per = pass;; per *= 2) {
      pq = (p.H[0] + per - 1) / per;
      const int parts = pq + (p.H[1] + per - 1) / per;
      if (parts <= 2 || (long long)tiles * parts <= kMaxParts) {
        grid = dim3(tiles, parts);
        break;
      }
    }
  cudaError_t e;
  if (grad) {
    e = launch_pdl(norm_rope_kernel<TI, GE, ACROSS, IT, true>, grid, kThreads, 0, s, 1, p, lanes, pq, per);
    if (e == cudaSuccess && p.part)
      e = launch_pdl(dw_kernel, dim3((2 * p.d + 7) / 8), 256, 0, s, 1, (const float*)p.part,
                     (int)(grid.x * grid.y), p.d, p.dw[0], p.dw[1]);
  } else {
    e = launch_pdl(norm_rope_kernel<TI, GE, ACROSS, IT, false>, grid, kThreads, 0, s, 1, p, lanes, pq, per);
  }
  if (e != cudaSuccess) note_failure("norm with rotation: launch");
  return e;
}

template <typename TI, int GE>
cudaError_t launch_g(const NormRopeProblem& p, bool grad, cudaStream_t s) {
  uintptr_t low = 0;
  for (int i = 0; i < 2; ++i) {
    if (!p.in[i]) continue;
    for (const void* x : {p.in[i], p.dout[i], (const void*)p.out[i]}) low |= reinterpret_cast<uintptr_t>(x);
    // (the stride of a dimension of one entry is never used)
    for (long long x : {p.B > 1 ? p.sB[i] : 0, p.T > 1 ? p.sT[i] : 0, p.H[i] > 1 ? p.sH[i] : 0})
      low |= (uintptr_t)(x * (long long)sizeof(TI));
  }
  const bool whole = low % 16 == 0 && p.d % GE == 0;
  if (p.half && whole && p.d_rot % (2 * GE) == 0) return launch_t<TI, GE, true, 1>(p, grad, s);
  if (!p.half && whole) return launch_t<TI, GE, false, 1>(p, grad, s);
  return launch_t<TI, 1, true, 4>(p, grad, s);
}

}  // namespace normrope

size_t norm_rope_grad_workspace_bytes(int d) {
  return (size_t)normrope::kMaxParts * 2 * d * sizeof(float);
}

cudaError_t launch_norm_rope(const NormRopeProblem& p, bool grad, cudaStream_t s) {
  if (p.dtype == RELATION_F32) return normrope::launch_g<float, 4>(p, grad, s);
  return normrope::launch_g<__nv_bfloat16, 8>(p, grad, s);
}

}  // namespace rel
