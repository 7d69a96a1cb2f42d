// scan.cuh -- the Exchange scan of a step's evidence in registers, shared by the forward
// (relation_tc_fwd.cu) and the chunk over a paged cache (relation_chunk.cu): a row's maximum, and
// P = e^{E - m} as bf16 pairs.
#pragma once

#include "common.cuh"

namespace rel {
namespace tc {

constexpr int HN = 64;         // keys of the scan's longer step
constexpr float kRescaleLog2 = 8.0f;  // rescale z only when the max grows by > 2^8
constexpr float kStaleLog2 = 32.0f;   // a step's P may reach 2^32 at the previous scale

// Bounded wait used while draining at teardown: never raises, just gives up.
__device__ __forceinline__ void drain_wait(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = globaltimer_ns();
  while (!mbar_try_wait(bar, parity)) {
    if (globaltimer_ns() - t0 > 20ull * 1000ull * 1000ull) return;  // 20 ms
  }
}

__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Maximum of the raw evidence U over the row's history in one step; on the diagonal tile
// only the keys before the row's own (t, relative to the step's first key) count, and U at
// key t (the Self evidence U_ii) is returned in u_self.
template <bool DIAG>
__device__ __forceinline__ float row_max(const uint32_t (&U)[HN], int t, float& u_self) {
  if (!DIAG) {
    float m0 = __uint_as_float(U[0]), m1 = __uint_as_float(U[1]);
    float m2 = __uint_as_float(U[2]), m3 = __uint_as_float(U[3]);
#pragma unroll
    for (int c = 4; c + 8 <= HN; c += 8) {
      m0 = fmax3(m0, __uint_as_float(U[c]), __uint_as_float(U[c + 1]));
      m1 = fmax3(m1, __uint_as_float(U[c + 2]), __uint_as_float(U[c + 3]));
      m2 = fmax3(m2, __uint_as_float(U[c + 4]), __uint_as_float(U[c + 5]));
      m3 = fmax3(m3, __uint_as_float(U[c + 6]), __uint_as_float(U[c + 7]));
    }
    // the last four keys (the loop covers keys 4 .. HN - 5)
    m0 = fmax3(m0, __uint_as_float(U[HN - 4]), __uint_as_float(U[HN - 3]));
    m1 = fmax3(m1, __uint_as_float(U[HN - 2]), __uint_as_float(U[HN - 1]));
    return fmaxf(fmax3(m0, m1, m2), m3);
  }
  float m = -INFINITY;
#pragma unroll
  for (int c = 0; c < HN; ++c) {
    const float x = __uint_as_float(U[c]);
    m = c < t ? fmaxf(m, x) : m;
    u_self = c == t ? x : u_self;
  }
  return m;
}

// P = 2^(U c2k (1 + tanh(U ch)) - m) for the 64 keys of a step (0 off the history on the
// diagonal tile), written to TMEM columns pcol.. as bf16 pairs; returns the row sum as two
// halves, and on the way the maximum of the raw evidence over the row's history in the
// step (umax) and, on the diagonal tile, U_ii (u_self).
template <bool DIAG>
__device__ __forceinline__ float2 scan_p(const uint32_t (&U)[HN], int t, uint32_t pcol, float ch,
                                         float c2k, float negm, float& umax, float& u_self) {
  const float2 ch2 = make_float2(ch, ch), c2k2 = make_float2(c2k, c2k);
  const float2 nm2 = make_float2(negm, negm);
  float2 sum = make_float2(0.f, 0.f);
  float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
  for (int c0 = 0; c0 < HN; c0 += 32) {
    uint32_t pk[16];
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      const float2 x = make_float2(__uint_as_float(U[c0 + c]), __uint_as_float(U[c0 + c + 1]));
      const float2 h = __fmul2_rn(x, ch2);
      const float2 th = make_float2(tanh_approx(h.x), tanh_approx(h.y));
      const float2 w = __ffma2_rn(th, c2k2, c2k2);  // log2(e) sigma(u) / sqrt(d), times 2
      const float2 e = __ffma2_rn(x, w, nm2);
      float2 pv = make_float2(ex2_approx(e.x), ex2_approx(e.y));
      if (DIAG) {
        const bool in0 = c0 + c < t, in1 = c0 + c + 1 < t;
        pv.x = in0 ? pv.x : 0.f;
        pv.y = in1 ? pv.y : 0.f;
        mx0 = fmax3(mx0, in0 ? x.x : -INFINITY, in1 ? x.y : -INFINITY);
        u_self = c0 + c == t ? x.x : (c0 + c + 1 == t ? x.y : u_self);
      } else {
        (c & 2 ? mx1 : mx0) = fmax3(c & 2 ? mx1 : mx0, x.x, x.y);
      }
      sum = __fadd2_rn(sum, pv);
      pk[c >> 1] = pack_bf16x2(pv.x, pv.y);
    }
    tmem_st16(pcol + (c0 >> 1), pk);
  }
  umax = fmaxf(mx0, mx1);
  return sum;
}

// The four-CTA layout's scan works on 32 keys at a time (registers): the maximum of the
// raw evidence over the history among them (keys before t, relative to their first key,
// on a masked step), and U at key t in u_self.
template <bool DIAG>
__device__ __forceinline__ float row_max32(const uint32_t (&U)[32], int t, float& u_self) {
  if (!DIAG) {
    float m0 = __uint_as_float(U[0]), m1 = __uint_as_float(U[1]);
    float m2 = __uint_as_float(U[2]), m3 = __uint_as_float(U[3]);
#pragma unroll
    for (int c = 4; c + 8 <= 32; c += 8) {
      m0 = fmax3(m0, __uint_as_float(U[c]), __uint_as_float(U[c + 1]));
      m1 = fmax3(m1, __uint_as_float(U[c + 2]), __uint_as_float(U[c + 3]));
      m2 = fmax3(m2, __uint_as_float(U[c + 4]), __uint_as_float(U[c + 5]));
      m3 = fmax3(m3, __uint_as_float(U[c + 6]), __uint_as_float(U[c + 7]));
    }
    m0 = fmax3(m0, __uint_as_float(U[28]), __uint_as_float(U[29]));
    m1 = fmax3(m1, __uint_as_float(U[30]), __uint_as_float(U[31]));
    return fmaxf(fmax3(m0, m1, m2), m3);
  }
  float m = -INFINITY;
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const float x = __uint_as_float(U[c]);
    m = c < t ? fmaxf(m, x) : m;
    u_self = c == t ? x : u_self;
  }
  return m;
}

// P of 32 keys as 16 bf16 pairs (not stored), their row sum, and on the way the maximum
// of their raw evidence over the history and U_ii (as scan_p).
template <bool DIAG>
__device__ __forceinline__ float2 scan_p32(const uint32_t (&U)[32], int t, float ch, float c2k,
                                           float negm, float& umax, float& u_self,
                                           uint32_t (&pk)[16]) {
  const float2 ch2 = make_float2(ch, ch), c2k2 = make_float2(c2k, c2k);
  const float2 nm2 = make_float2(negm, negm);
  float2 sum = make_float2(0.f, 0.f);
  float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
  for (int c = 0; c < 32; c += 2) {
    const float2 x = make_float2(__uint_as_float(U[c]), __uint_as_float(U[c + 1]));
    const float2 h = __fmul2_rn(x, ch2);
    const float2 th = make_float2(tanh_approx(h.x), tanh_approx(h.y));
    const float2 w = __ffma2_rn(th, c2k2, c2k2);
    const float2 e = __ffma2_rn(x, w, nm2);
    float2 pv = make_float2(ex2_approx(e.x), ex2_approx(e.y));
    if (DIAG) {
      const bool in0 = c < t, in1 = c + 1 < t;
      pv.x = in0 ? pv.x : 0.f;
      pv.y = in1 ? pv.y : 0.f;
      mx0 = fmax3(mx0, in0 ? x.x : -INFINITY, in1 ? x.y : -INFINITY);
      u_self = c == t ? x.x : (c + 1 == t ? x.y : u_self);
    } else {
      (c & 2 ? mx1 : mx0) = fmax3(c & 2 ? mx1 : mx0, x.x, x.y);
    }
    sum = __fadd2_rn(sum, pv);
    pk[c >> 1] = pack_bf16x2(pv.x, pv.y);
  }
  umax = fmaxf(mx0, mx1);
  return sum;
}

}  // namespace tc
}  // namespace rel
