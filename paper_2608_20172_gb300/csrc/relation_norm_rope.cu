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
// the position, modulo 2^64 -- exact at every position, no reduction by 2 pi, and no fp64 but one
// product a frequency (fp64 angles cost four times the table's other work on this GPU).
//
// Bound by memory: a row is read and written once (backward: two reads).  A few lanes share a row, 16
// bytes of two parts of it each, so that both channels of a pair are in one lane in either layout and
// the sums are a few shuffles; the turns of a CTA's tokens are tabulated once for all heads.
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace rel {
namespace normrope {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kMaxD = 256;
constexpr int kMaxParts = 1216;  // CTAs that leave a partial sum of dw

// GE consecutive elements: 16 bytes of an aligned row, or one element
template <typename TI, int GE>
struct Group {
  struct Raw {
    TI x;
  };
  static __device__ __forceinline__ Raw load(const TI* p) { return {*p}; }
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

// The turns (cos, sin) s of a CTA's tokens; pairs past the last one of a group that the turned part
// ends in stay as they are.
template <int TOK>
__device__ __forceinline__ void fill_turns(float2 (&turn)[TOK][kMaxD / 2], const int (&pos)[TOK],
                                           const NormRopeProblem& p, int nt) {
  const int half = p.d_rot / 2, n = min(p.d / 2, (half + 3) & ~3);
  for (int c = threadIdx.x; c < n; c += kThreads) {
    if (c >= half) {
      for (int tt = 0; tt < nt; ++tt) turn[tt][c] = make_float2(1.f, 0.f);
      continue;
    }
    const double t = p.freqs[c] * 0.15915494309189533576888376337251;  // turns a position
    const unsigned long long step =
        (unsigned long long)__double2ll_rn((t - rint(t)) * 9223372036854775808.0) << 1;
    for (int tt = 0; tt < nt; ++tt) {
      const unsigned long long at = (unsigned long long)max(pos[tt], 0) * step;
      float s, co;
      sincospif((float)(int)(at >> 32) * 0x1p-31f, &s, &co);
      turn[tt][c] = make_float2(co * p.scale, s * p.scale);
    }
  }
}

__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// A lane's two groups turned (SIGN 1) or turned back (-1)
template <int GE, bool ACROSS>
__device__ __forceinline__ void turned(float (&x)[GE], float (&y)[GE], const float2* t, int pa, int pb,
                                       float sign) {
  if constexpr (ACROSS) {
    if (pa < 0) return;
#pragma unroll
    for (int j = 0; j < GE; ++j) {
      const float2 cs = t[pa + j];
      const float s = cs.y * sign, a = x[j], b = y[j];
      x[j] = a * cs.x - b * s;
      y[j] = a * s + b * cs.x;
    }
  } else {
#pragma unroll
    for (int j = 0; j < GE / 2; ++j) {
      if (pa >= 0) {
        const float2 cs = t[pa + j];
        const float s = cs.y * sign, a = x[2 * j], b = x[2 * j + 1];
        x[2 * j] = a * cs.x - b * s;
        x[2 * j + 1] = a * s + b * cs.x;
      }
      if (pb >= 0) {
        const float2 cs = t[pb + j];
        const float s = cs.y * sign, a = y[2 * j], b = y[2 * j + 1];
        y[2 * j] = a * cs.x - b * s;
        y[2 * j + 1] = a * s + b * cs.x;
      }
    }
  }
}

// Element offset of token n, in the tensors of the queries (which 0) or keys (1)
__device__ __forceinline__ long long token_at(const NormRopeProblem& p, int which, int n) {
  const int b = n / p.T, t = n - b * p.T;
  return (long long)b * p.sB[which] + (long long)t * p.sT[which];
}

template <int TOK>
__device__ __forceinline__ void fill_positions(int (&pos)[TOK], const NormRopeProblem& p, int t0) {
  if (threadIdx.x < TOK) {
    const int n = min(t0 + (int)threadIdx.x, p.B * p.T - 1);
    pos[threadIdx.x] = p.positions ? p.positions[n] : n % p.T;
  }
}
__device__ __forceinline__ void fill_weights(float (&w)[2][kMaxD], const NormRopeProblem& p) {
  for (int e = threadIdx.x; e < 2 * p.d; e += kThreads) {
    const int which = e >= p.d, c = e - which * p.d;
    w[which][c] = p.w[which] ? p.w[which][c] : 1.f;
  }
}

template <typename TI, int GE, bool ACROSS, int IT, int TOK>
__global__ void __launch_bounds__(kThreads)
    norm_rope_kernel(const __grid_constant__ NormRopeProblem p, int lanes) {
  using G = Group<TI, GE>;
  __shared__ __align__(16) float2 turn[TOK][kMaxD / 2];
  __shared__ __align__(16) float w[2][kMaxD];
  __shared__ int pos[TOK];
  pdl_wait_and_launch();
  const int N = p.B * p.T, t0 = (int)blockIdx.x * TOK, nt = min(TOK, N - t0);
  const int per = p.H[0] + p.H[1], rows = nt * per, step = kThreads / lanes;
  const Place<GE, ACROSS, IT> at(threadIdx.x % lanes, lanes, p.d, p.d_rot, p.half);
  struct Row {
    int which, tt;
    long long off;
    typename G::Raw a[IT], b[IT];
  };
  auto fetch = [&](int r, Row& row) {  // (clamped: a group of lanes past the end takes the last row)
    r = min(r, rows - 1);
    row.tt = r / per;
    const int h = r - row.tt * per;
    row.which = h >= p.H[0];
    row.off = token_at(p, row.which, t0 + row.tt) + (long long)(h - row.which * p.H[0]) * p.sH[row.which];
    const TI* src = static_cast<const TI*>(p.in[row.which]) + row.off;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if (at.a[it] >= 0) row.a[it] = G::load(src + at.a[it]);
      if (at.b[it] >= 0) row.b[it] = G::load(src + at.b[it]);
    }
  };
  auto finish = [&](const Row& row, bool live) {
    float x[IT][GE], y[IT][GE], ss = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
#pragma unroll
      for (int j = 0; j < GE; ++j) x[it][j] = y[it][j] = 0.f;
      if (at.a[it] >= 0) G::unpack(row.a[it], x[it]);
      if (at.b[it] >= 0) G::unpack(row.b[it], y[it]);
#pragma unroll
      for (int j = 0; j < GE; ++j) ss = fmaf(x[it][j], x[it][j], fmaf(y[it][j], y[it][j], ss));
    }
    ss = lanes_sum(ss, lanes);
    const float r = p.norm ? rsqrtf(ss / (float)p.d + p.eps) : 1.f;
    const bool none = pos[row.tt] < 0;
    TI* dst = static_cast<TI*>(p.out[row.which]) + row.off;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
#pragma unroll
      for (int j = 0; j < GE; ++j) {
        x[it][j] *= r * w[row.which][max(at.a[it], 0) + j];
        y[it][j] *= r * w[row.which][max(at.b[it], 0) + j];
      }
      turned<GE, ACROSS>(x[it], y[it], turn[row.tt], at.pa[it], at.pb[it], 1.f);
#pragma unroll
      for (int j = 0; j < GE; ++j) {
        x[it][j] = none ? 0.f : x[it][j];
        y[it][j] = none ? 0.f : y[it][j];
      }
      if (live && at.a[it] >= 0) G::store(dst + at.a[it], x[it]);
      if (live && at.b[it] >= 0) G::store(dst + at.b[it], y[it]);
    }
  };
  Row r0, r1;
  const int first = threadIdx.x / lanes;
  fetch(first, r0);
  fetch(first + step, r1);
  fill_positions<TOK>(pos, p, t0);
  fill_weights(w, p);
  __syncthreads();
  fill_turns<TOK>(turn, pos, p, nt);
  __syncthreads();
  // (whole warps: the sums are shuffles)
  for (int r = first; r - first < rows; r += 2 * step) {
    if (r != first) {
      fetch(r, r0);
      fetch(r + step, r1);
    }
    finish(r0, r < rows);
    finish(r1, r + step < rows);
  }
}

// Backward.  CTAs walk the tokens in steps of the grid and keep their columns' dw; the sums over a
// CTA's rows are in a fixed order, and dw_kernel adds the CTAs' up.
template <typename TI, int GE, bool ACROSS, int IT, int TOK>
__global__ void __launch_bounds__(kThreads)
    norm_rope_grad_kernel(const __grid_constant__ NormRopeProblem p, int lanes) {
  using G = Group<TI, GE>;
  __shared__ __align__(16) float2 turn[TOK][kMaxD / 2];
  __shared__ __align__(16) float w[2][kMaxD];
  __shared__ float sums[kWarps][kMaxD];
  __shared__ int pos[TOK];
  pdl_wait_and_launch();
  const int N = p.B * p.T, tiles = (N + TOK - 1) / TOK, step = kThreads / lanes;
  const Place<GE, ACROSS, IT> at(threadIdx.x % lanes, lanes, p.d, p.d_rot, p.half);
  float acc[2][2][IT][GE];
#pragma unroll
  for (int e = 0; e < 4 * IT * GE; ++e) (&acc[0][0][0][0])[e] = 0.f;
  fill_weights(w, p);
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int t0 = tile * TOK, nt = min(TOK, N - t0);
    __syncthreads();
    fill_positions<TOK>(pos, p, t0);
    __syncthreads();
    fill_turns<TOK>(turn, pos, p, nt);
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int H = p.H[which], rows = nt * H;
      for (int r0 = 0; r0 < rows; r0 += step) {
        const int r = r0 + (int)threadIdx.x / lanes;
        const int tt = min(r, rows - 1) / H, h = min(r, rows - 1) - tt * H;
        const bool live = r < rows;
        const long long off = token_at(p, which, t0 + tt) + (long long)h * p.sH[which];
        const TI* sx = static_cast<const TI*>(p.in[which]) + off;
        const TI* sy = static_cast<const TI*>(p.dout[which]) + off;
        float x[2][IT][GE], u[2][IT][GE], ss = 0.f, dot = 0.f;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
#pragma unroll
          for (int j = 0; j < GE; ++j) x[0][it][j] = x[1][it][j] = u[0][it][j] = u[1][it][j] = 0.f;
          if (at.a[it] >= 0) {
            G::unpack(G::load(sx + at.a[it]), x[0][it]);
            G::unpack(G::load(sy + at.a[it]), u[0][it]);
          }
          if (at.b[it] >= 0) {
            G::unpack(G::load(sx + at.b[it]), x[1][it]);
            G::unpack(G::load(sy + at.b[it]), u[1][it]);
          }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          turned<GE, ACROSS>(u[0][it], u[1][it], turn[tt], at.pa[it], at.pb[it], -1.f);
#pragma unroll
          for (int j = 0; j < GE; ++j) {
            ss = fmaf(x[0][it][j], x[0][it][j], fmaf(x[1][it][j], x[1][it][j], ss));
            const float wa = w[which][max(at.a[it], 0) + j], wb = w[which][max(at.b[it], 0) + j];
            dot = fmaf(x[0][it][j] * wa, u[0][it][j], fmaf(x[1][it][j] * wb, u[1][it][j], dot));
          }
        }
        const bool none = pos[tt] < 0;
        float rn = 1.f, mean = 0.f;
        if (p.norm) {
          ss = lanes_sum(ss, lanes);
          dot = lanes_sum(dot, lanes);
          rn = rsqrtf(ss / (float)p.d + p.eps);
          mean = dot * rn / (float)p.d;  // mean of x^ w u
        }
        TI* dst = static_cast<TI*>(p.out[which]) + off;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
#pragma unroll
          for (int side = 0; side < 2; ++side) {
            const int c = side ? at.b[it] : at.a[it];
            float dx[GE];
#pragma unroll
            for (int j = 0; j < GE; ++j) {
              const float xh = x[side][it][j] * rn;
              dx[j] = none ? 0.f : rn * (w[which][max(c, 0) + j] * u[side][it][j] - xh * mean);
              if (live && !none) acc[which][side][it][j] = fmaf(u[side][it][j], xh, acc[which][side][it][j]);
            }
            if (live && c >= 0) G::store(dst + c, dx);
          }
        }
      }
    }
  }
  if (!p.part) return;
  // the CTA's sums: lanes of the same columns by shuffles, then the warps in order
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const int c = side ? at.b[it] : at.a[it];
#pragma unroll
        for (int j = 0; j < GE; ++j) {
          float x = acc[which][side][it][j];
          for (int o = 16; o >= lanes; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
          if ((threadIdx.x & 31) < lanes && c >= 0) sums[threadIdx.x >> 5][c + j] = x;
        }
      }
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += kThreads) {
      float x = sums[0][c];
#pragma unroll
      for (int i = 1; i < kWarps; ++i) x += sums[i][c];
      p.part[((long long)blockIdx.x * 2 + which) * p.d + c] = x;
    }
  }
}

// dw from the CTAs' partial sums, in fp64: 8 columns a CTA, 32 lots of the partial sums
__global__ void __launch_bounds__(256) dw_kernel(const float* part, int n, int d, float* dw1, float* dw2) {
  __shared__ double red[32][8];
  pdl_wait_and_launch();
  const int e = blockIdx.x * 8 + (threadIdx.x & 7), lot = threadIdx.x >> 3;
  double s = 0.0;
  if (e < 2 * d)
    for (int i = lot; i < n; i += 32) s += (double)part[(long long)i * 2 * d + e];
  red[lot][threadIdx.x & 7] = s;
  __syncthreads();
  if (lot == 0 && e < 2 * d) {
    for (int i = 1; i < 32; ++i) s += red[i][threadIdx.x & 7];
    float* dw = e < d ? dw1 : dw2;
    if (dw) dw[e < d ? e : e - d] = (float)s;
  }
}

constexpr int kGradTok = 4;

template <typename TI, int GE, bool ACROSS, int IT>
cudaError_t launch_t(const NormRopeProblem& p, bool grad, cudaStream_t s) {
  // lanes of a row: its groups in twos (ACROSS: the turned ones and the others apart)
  const int half = p.d_rot / 2 / GE, rest = (p.d - (ACROSS ? p.d_rot : 0) + GE - 1) / GE;
  int need = ACROSS ? half + (rest + 1) / 2 : (rest + 1) / 2, lanes = 1;
  while (lanes < need && lanes < 32) lanes *= 2;
  const int N = p.B * p.T;
  cudaError_t e;
  if (grad) {
    const int tiles = (N + kGradTok - 1) / kGradTok, grid = tiles < kMaxParts ? tiles : kMaxParts;
    e = launch_pdl(norm_rope_grad_kernel<TI, GE, ACROSS, IT, kGradTok>, dim3(grid), kThreads, 0, s, 1, p, lanes);
    if (e == cudaSuccess && p.part)
      e = launch_pdl(dw_kernel, dim3((2 * p.d + 7) / 8), 256, 0, s, 1, (const float*)p.part, grid, p.d,
                     p.dw[0], p.dw[1]);
  } else {
    e = launch_pdl(norm_rope_kernel<TI, GE, ACROSS, IT, 2>, dim3((N + 1) / 2), kThreads, 0, s, 1, p, lanes);
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
    for (long long x : {p.sB[i], p.sT[i], p.sH[i]}) low |= (uintptr_t)(x * (long long)sizeof(TI));
  }
  const bool whole = low % 16 == 0 && p.d % GE == 0;
  if (p.half && whole && p.d_rot % (2 * GE) == 0) return launch_t<TI, GE, true, 1>(p, grad, s);
  if (!p.half && whole) return launch_t<TI, GE, false, 1>(p, grad, s);
  return launch_t<TI, 1, true, 4>(p, grad, s);
}

}  // namespace normrope

size_t norm_rope_grad_workspace_bytes(int tokens, int d) {
  const int tiles = (tokens + normrope::kGradTok - 1) / normrope::kGradTok;
  return (size_t)(tiles < normrope::kMaxParts ? tiles : normrope::kMaxParts) * 2 * d * sizeof(float);
}

cudaError_t launch_norm_rope(const NormRopeProblem& p, bool grad, cudaStream_t s) {
  if (p.dtype == RELATION_F32) return normrope::launch_g<float, 4>(p, grad, s);
  return normrope::launch_g<__nv_bfloat16, 8>(p, grad, s);
}

}  // namespace rel
