// layer.cuh -- pieces that the layer's transforms (relation_layer.cu) and the cache's write
// (relation_append.cu) share: 8-element vectors and the rotation's angles.
#pragma once

#include "common.cuh"

namespace rel {
namespace layer {

template <typename TI>
struct Vec8;
template <>
struct Vec8<__nv_bfloat16> {
  using Raw = uint4;
  __device__ static Raw load(const __nv_bfloat16* p) { return *reinterpret_cast<const uint4*>(p); }
  __device__ static void unpack(const Raw& w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  __device__ static void store(void* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};
template <>
struct Vec8<float> {
  struct Raw {
    float4 a, b;
  };
  __device__ static Raw load(const float* p) {
    return {reinterpret_cast<const float4*>(p)[0], reinterpret_cast<const float4*>(p)[1]};
  }
  __device__ static void unpack(const Raw& w, float (&x)[8]) {
    x[0] = w.a.x; x[1] = w.a.y; x[2] = w.a.z; x[3] = w.a.w;
    x[4] = w.b.x; x[5] = w.b.y; x[6] = w.b.z; x[7] = w.b.w;
  }
  __device__ static void store(void* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// Positions whose angles come from turn: up to there they are as exact as fp64's, both being
// rounded to fp32 in the end (against 64 bits over d 48 to 256, bases 1 to 5e5: rms 4.66e-8 rad with
// either, at most 1.193e-7 against 1.192e-7 below 2^15 positions; 1.20e-7 at 2^17, 1.49e-7 at 2^22).
constexpr int kTurnPositions = 1 << 15;

// m * w modulo 2 pi (|r| <= pi + rounding) for a position m and w = w_hi + w_lo <= 1: the product
// and n 2 pi are kept as rounded value and exact remainder (two-product by fma; their leading
// parts are close, so that their difference is exact), 2 pi as a sum of two floats (48 bits).
// The _rn forms: a product that was contracted into the difference would have its remainder
// counted twice.
__device__ __forceinline__ float turn(float m, float w_hi, float w_lo) {
  constexpr float kTwoPiHi = 6.28318530717958647692f;
  constexpr float kTwoPiLo = (float)(6.28318530717958647692 - (double)kTwoPiHi);
  const float a = __fmul_rn(m, w_hi);
  const float a_lo = fmaf(m, w_lo, fmaf(m, w_hi, -a));
  const float n = rintf(__fmul_rn(a, 0.15915494309189533577f));
  const float q = __fmul_rn(n, kTwoPiHi);
  const float q_lo = fmaf(n, kTwoPiLo, fmaf(n, kTwoPiHi, -q));
  return __fadd_rn(__fsub_rn(a, q), __fsub_rn(a_lo, q_lo));
}

}  // namespace layer
}  // namespace rel
