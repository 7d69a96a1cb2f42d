// relation_api.cu -- the C ABI of librelation (declared in include/relation.h).
//
// Host code only: argument validation (nothing is launched on an error), selection of
// the kernel family, workspace carving and launches on the caller's stream.  The
// library allocates no device memory.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "kernels.h"
#include "relation.h"

namespace {

using rel::Problem;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

size_t elem_size(relation_dtype dt) { return dt == RELATION_F32 ? 4 : 2; }

relation_status check_shape(const relation_shape& s, relation_dtype dt) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (s.B < 1 || s.T < 1 || s.H < 1 || s.d_h < 1) return RELATION_ERR_INVALID_ARG;
  if ((long long)s.B * s.H > 65535) return RELATION_ERR_UNSUPPORTED;  // grid.y limit
  if (s.sB < 1 || s.sT < 1 || s.sH < 1) return RELATION_ERR_INVALID_ARG;
  if (!rel::simt::supports(dt, s.d_h) && !rel::tc::supports(dt, s.d_h))
    return RELATION_ERR_UNSUPPORTED;
  const long long vec = 16 / (long long)elem_size(dt);
  if (s.sB % vec || s.sT % vec || s.sH % vec) return RELATION_ERR_ALIGNMENT;
  return RELATION_OK;
}

relation_status check_scalars(float lambda, float tau_s) {
  if (!isfinite(lambda) || !isfinite(tau_s) || !(tau_s > 0.0f)) return RELATION_ERR_INVALID_ARG;
  return RELATION_OK;
}

relation_status check_ptrs(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!p) return RELATION_ERR_INVALID_ARG;
  for (const void* p : ptrs)
    if (!aligned16(p)) return RELATION_ERR_ALIGNMENT;
  return RELATION_OK;
}

// Family that will run: 1 = SIMT, 2 = tcgen05; 0 when the request cannot be served.
int pick_family(relation_kernel kernel, relation_dtype dt, int d, bool backward) {
  const bool tc = backward ? rel::tc::supports_bwd(dt, d) : rel::tc::supports(dt, d);
  const bool simt = rel::simt::supports(dt, d);
  switch (kernel) {
    case RELATION_KERNEL_AUTO: return tc ? 2 : (simt ? 1 : 0);
    case RELATION_KERNEL_SIMT: return simt ? 1 : 0;
    case RELATION_KERNEL_TCGEN05: return tc ? 2 : 0;
  }
  return 0;
}

Problem make_problem(relation_shape s, relation_dtype dt, float lambda, float tau_s,
                     int* dev_status) {
  Problem p{};
  p.lambda = lambda;
  p.tau_s = tau_s;
  p.inv_sqrt_d = 1.0f / sqrtf((float)s.d_h);
  p.B = s.B; p.T = s.T; p.H = s.H; p.d = s.d_h;
  p.sB = s.sB; p.sT = s.sT; p.sH = s.sH;
  p.dtype = dt;
  p.dev_status = dev_status;
  return p;
}

thread_local cudaError_t g_last_cuda_error = cudaSuccess;
thread_local const char* g_last_where = "";
thread_local char g_last_message[256];

relation_status from_cuda(cudaError_t e) {
  if (e == cudaSuccess) return RELATION_OK;
  if (e == cudaErrorInvalidValue && !g_last_where[0]) g_last_where = "launch";
  g_last_cuda_error = e;
  return RELATION_ERR_CUDA;
}

}  // namespace

namespace rel {
void note_failure(const char* where) { g_last_where = where; }
}  // namespace rel

extern "C" {

relation_status relation_fwd_flow(const void* q, const void* k, const void* v, void* o,
                                  float* logz, float* self_flow, float lambda, float tau_s,
                                  relation_shape shp, relation_dtype dt, relation_kernel kernel,
                                  int* dev_status, relation_stream_t stream) {
  relation_status st;
  if ((st = check_shape(shp, dt)) != RELATION_OK) return st;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if ((st = check_ptrs({q, k, v, o, logz})) != RELATION_OK) return st;
  if (self_flow && (st = check_ptrs({self_flow})) != RELATION_OK) return st;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  const int fam = pick_family(kernel, dt, shp.d_h, false);
  if (fam == 0) return RELATION_ERR_UNSUPPORTED;
  Problem p = make_problem(shp, dt, lambda, tau_s, dev_status);
  p.q = q; p.k = k; p.v = v; p.out = o; p.logz = logz; p.fself = self_flow;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return from_cuda(fam == 2 ? rel::tc::launch_fwd(p, s) : rel::simt::launch_fwd(p, s));
}

relation_status relation_fwd_ex(const void* q, const void* k, const void* v, void* o, float* logz,
                                float lambda, float tau_s, relation_shape shp, relation_dtype dt,
                                relation_kernel kernel, int* dev_status, relation_stream_t stream) {
  return relation_fwd_flow(q, k, v, o, logz, nullptr, lambda, tau_s, shp, dt, kernel, dev_status,
                           stream);
}

relation_status relation_fwd(const void* q, const void* k, const void* v, void* o, float* logz,
                             float lambda, float tau_s, relation_shape shp, relation_dtype dt,
                             int* dev_status, relation_stream_t stream) {
  return relation_fwd_ex(q, k, v, o, logz, lambda, tau_s, shp, dt, RELATION_KERNEL_AUTO,
                         dev_status, stream);
}

relation_status relation_fwd_state(const void* q, const void* k, const void* v, float* m,
                                   float* l, float* z, relation_shape shp_q,
                                   relation_shape shp_kv, int causal, relation_dtype dt,
                                   int* dev_status, relation_stream_t stream) {
  relation_status st;
  if ((st = check_shape(shp_q, dt)) != RELATION_OK) return st;
  if ((st = check_shape(shp_kv, dt)) != RELATION_OK) return st;
  if (causal != 0 && causal != 1) return RELATION_ERR_INVALID_ARG;
  if (shp_kv.B != shp_q.B || shp_kv.H != shp_q.H || shp_kv.d_h != shp_q.d_h)
    return RELATION_ERR_INVALID_ARG;
  if (causal && shp_kv.T != shp_q.T) return RELATION_ERR_INVALID_ARG;
  if (!rel::tc::supports(dt, shp_q.d_h)) return RELATION_ERR_UNSUPPORTED;  // bf16 tiles
  if ((long long)((shp_q.T + 127) / 128) * shp_q.B * shp_q.H > 0x7fffffffLL)
    return RELATION_ERR_UNSUPPORTED;
  if ((st = check_ptrs({q, k, v, m, l, z})) != RELATION_OK) return st;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  Problem p = make_problem(shp_q, dt, 0.0f, 1.0f, dev_status);
  p.q = q; p.k = k; p.v = v;
  rel::StateArgs sa{};
  sa.causal = causal;
  sa.Tk = shp_kv.T;
  sa.k_sB = shp_kv.sB; sa.k_sT = shp_kv.sT; sa.k_sH = shp_kv.sH;
  sa.m = m; sa.l = l; sa.z = z;
  return from_cuda(rel::tc::launch_fwd_state(p, sa, reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_state_merge(float* m, float* l, float* z, const float* m2,
                                     const float* l2, const float* z2, relation_shape shp,
                                     relation_stream_t stream) {
  if (shp.B < 1 || shp.T < 1 || shp.H < 1) return RELATION_ERR_INVALID_ARG;
  if (shp.d_h < 4 || shp.d_h > 128 || shp.d_h % 4) return RELATION_ERR_UNSUPPORTED;
  relation_status st;
  if ((st = check_ptrs({m, l, z, m2, l2, z2})) != RELATION_OK) return st;
  const long long rows = (long long)shp.B * shp.H * shp.T;
  return from_cuda(rel::launch_state_merge(m, l, z, m2, l2, z2, rows, shp.d_h,
                                           reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_state_finish(const void* q, const void* k, const void* v,
                                      const float* m, const float* l, const float* z, void* o,
                                      float* logz, float* self_flow, float lambda, float tau_s,
                                      long long pos0, relation_shape shp, relation_dtype dt,
                                      relation_stream_t stream) {
  relation_status st;
  if ((st = check_shape(shp, dt)) != RELATION_OK) return st;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if (pos0 < 0) return RELATION_ERR_INVALID_ARG;
  if (shp.d_h < 4 || shp.d_h > 128 || shp.d_h % 4) return RELATION_ERR_UNSUPPORTED;
  if ((st = check_ptrs({q, k, v, m, l, z, o, logz})) != RELATION_OK) return st;
  if (self_flow && (st = check_ptrs({self_flow})) != RELATION_OK) return st;
  Problem p = make_problem(shp, dt, lambda, tau_s, nullptr);
  p.q = q; p.k = k; p.v = v; p.out = o; p.logz = logz; p.fself = self_flow;
  return from_cuda(rel::launch_state_finish(p, m, l, z, pos0,
                                            reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_linear_fwd(const void* p1, const void* p2, const void* v,
                                   const float* alpha, void* y, float tau_s, relation_shape shp,
                                   relation_dtype dt, int* dev_status, relation_stream_t stream) {
  return relation_linear_fwd_ex(p1, p2, v, alpha, y, tau_s, shp, dt, RELATION_KERNEL_AUTO,
                                dev_status, stream);
}

relation_status relation_linear_fwd_ex(const void* p1, const void* p2, const void* v,
                                      const float* alpha, void* y, float tau_s,
                                      relation_shape shp, relation_dtype dt,
                                      relation_kernel kernel, int* dev_status,
                                      relation_stream_t stream) {
  relation_status st;
  if (kernel != RELATION_KERNEL_AUTO && kernel != RELATION_KERNEL_SIMT &&
      kernel != RELATION_KERNEL_TCGEN05)
    return RELATION_ERR_INVALID_ARG;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (shp.B < 1 || shp.T < 1 || shp.H < 1 || shp.d_h < 1) return RELATION_ERR_INVALID_ARG;
  if (shp.sB < 1 || shp.sT < 1 || shp.sH < 1) return RELATION_ERR_INVALID_ARG;
  if (!rel::linear_supports(dt, shp.d_h)) return RELATION_ERR_UNSUPPORTED;
  // grid: up to 8 column splits per head
  if ((long long)shp.B * shp.H * 8 > 0x7fffffffLL) return RELATION_ERR_UNSUPPORTED;
  // 4-element vector loads of every token row (alpha is fp32 with the same strides)
  if (shp.sB % 4 || shp.sT % 4 || shp.sH % 4) return RELATION_ERR_ALIGNMENT;
  if (!isfinite(tau_s) || !(tau_s > 0.0f)) return RELATION_ERR_INVALID_ARG;
  if ((st = check_ptrs({p1, p2, v, alpha, y})) != RELATION_OK) return st;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  rel::LinearProblem p{};
  p.p1 = p1; p.p2 = p2; p.v = v; p.alpha = alpha; p.y = y; p.dev_status = dev_status;
  p.tau_s = tau_s; p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  const bool tc = rel::linear_tc_supports(p);
  if (kernel == RELATION_KERNEL_TCGEN05 && !tc)
    return (dt == RELATION_BF16 && (shp.d_h == 64 || shp.d_h == 128)) ? RELATION_ERR_ALIGNMENT
                                                                     : RELATION_ERR_UNSUPPORTED;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (tc && kernel != RELATION_KERNEL_SIMT)
    return from_cuda(rel::launch_linear_tc_fwd(p, nullptr, s));
  return from_cuda(rel::launch_linear_fwd(p, s));
}

size_t relation_linear_fwd_workspace_size(relation_shape shp, relation_dtype dt) {
  if (dt != RELATION_BF16 || shp.B < 1 || shp.T < 1 || shp.H < 1) return 0;
  rel::LinearProblem p{};
  p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  return rel::linear_tc_workspace_bytes(p);
}

relation_status relation_linear_fwd_ws(const void* p1, const void* p2, const void* v,
                                      const float* alpha, void* y, float tau_s,
                                      relation_shape shp, relation_dtype dt, void* workspace,
                                      size_t ws_bytes, int* dev_status,
                                      relation_stream_t stream) {
  const size_t need = relation_linear_fwd_workspace_size(shp, dt);
  if (need == 0)  // no chunked kernel for this request: the regular entry point decides
    return relation_linear_fwd_ex(p1, p2, v, alpha, y, tau_s, shp, dt, RELATION_KERNEL_AUTO,
                                  dev_status, stream);
  if (!workspace || ws_bytes < need) return RELATION_ERR_WORKSPACE;
  if (!aligned16(workspace)) return RELATION_ERR_ALIGNMENT;
  int dev = 0, nsm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return RELATION_ERR_CUDA;
  const long long ctas = (long long)shp.B * shp.H * (shp.d_h / 64);
  const long long nb = (shp.T + 127) / 128, waves = nsm > 0 ? (ctas + nsm - 1) / nsm : 0;
  // The sequential walk takes `waves` rounds of the SMs, one (head, column) pair each, however
  // full the last one is; the chunk-parallel passes share out the blocks evenly, at 1.52 times a
  // round's time per block of all SMs (d_h = 128: 1.61) and 1.75 (2.0) blocks' time for the
  // launches and the scan.  us, chunk-parallel and sequential, d_h = 64: 12 pairs, T 8192 44 / 262;
  // 84 pairs, T 2048 66 / 74; 96 76 / 74; 144 108 / 78; 156 112 / 139; 216 152 / 142; 60 pairs,
  // T 640 22 / 26; 72 28 / 26.  d_h = 128, T 2048: 80 132 / 144; 96 157 / 147; 160 249 / 277.
  const long long per_block = shp.d_h == 64 ? 152 : 161, fixed = shp.d_h == 64 ? 175 : 200;
  // A stride below 1 (one entry along it: 0 is as good as any) is refused by the sequential entry
  // point and taken by the passes: there the choice goes by the number of pairs alone, as it did
  // before it went by cost, so that the same calls are refused.
  const bool strided = shp.sB >= 1 && shp.sT >= 1 && shp.sH >= 1;
  if (strided ? 100 * waves * nb * nsm <= fixed * nsm + per_block * ctas * nb : 2 * ctas >= nsm)
    return relation_linear_fwd_ex(p1, p2, v, alpha, y, tau_s, shp, dt, RELATION_KERNEL_TCGEN05,
                                  dev_status, stream);
  relation_status st;
  if ((st = check_ptrs({p1, p2, v, alpha, y})) != RELATION_OK) return st;
  if (!isfinite(tau_s) || !(tau_s > 0.0f)) return RELATION_ERR_INVALID_ARG;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  if ((long long)ctas * ((shp.T + 127) / 128) > 0x7fffffffLL) return RELATION_ERR_UNSUPPORTED;
  rel::LinearProblem p{};
  p.p1 = p1; p.p2 = p2; p.v = v; p.alpha = alpha; p.y = y; p.dev_status = dev_status;
  p.tau_s = tau_s; p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  return from_cuda(rel::launch_linear_tc_fwd(p, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

namespace {

// The kernel family a backward request runs on (SIMT or TCGEN05), or -1 when the request
// is not served: the arguments' shapes and dtypes only, no pointers.
int linear_bwd_family(const relation_shape& shp, relation_dtype dt, relation_kernel kernel,
                      relation_status* why) {
  *why = RELATION_OK;
  if (kernel != RELATION_KERNEL_AUTO && kernel != RELATION_KERNEL_SIMT &&
      kernel != RELATION_KERNEL_TCGEN05) { *why = RELATION_ERR_INVALID_ARG; return -1; }
  if (dt != RELATION_F32 && dt != RELATION_BF16) { *why = RELATION_ERR_INVALID_ARG; return -1; }
  if (shp.B < 1 || shp.T < 1 || shp.H < 1 || shp.d_h < 1) { *why = RELATION_ERR_INVALID_ARG; return -1; }
  if (shp.sB < 1 || shp.sT < 1 || shp.sH < 1) { *why = RELATION_ERR_INVALID_ARG; return -1; }
  if (!rel::linear_supports(dt, shp.d_h)) { *why = RELATION_ERR_UNSUPPORTED; return -1; }
  // grid: up to 8 column splits per head
  if ((long long)shp.B * shp.H * 8 > 0x7fffffffLL) { *why = RELATION_ERR_UNSUPPORTED; return -1; }
  // 4-element vector loads of every token row (alpha is fp32 with the same strides)
  if (shp.sB % 4 || shp.sT % 4 || shp.sH % 4) { *why = RELATION_ERR_ALIGNMENT; return -1; }
  rel::LinearProblem p{};
  p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  const bool tc = rel::linear_tc_bwd_supports(p) &&
                  (long long)shp.B * shp.H * ((shp.T + 127) / 128) <= 0x7fffffffLL;
  if (kernel == RELATION_KERNEL_TCGEN05 && !tc) {
    *why = (dt == RELATION_BF16 && shp.d_h == 64 && (shp.sB % 8 || shp.sT % 8 || shp.sH % 8))
               ? RELATION_ERR_ALIGNMENT : RELATION_ERR_UNSUPPORTED;
    return -1;
  }
  return (tc && kernel != RELATION_KERNEL_SIMT) ? (int)RELATION_KERNEL_TCGEN05
                                                : (int)RELATION_KERNEL_SIMT;
}

size_t linear_bwd_bytes(const relation_shape& shp, relation_dtype dt, int family) {
  if (family == (int)RELATION_KERNEL_SIMT)
    return rel::linear_bwd_workspace_bytes(shp.B, shp.H, shp.T, shp.d_h);
  rel::LinearProblem p{};
  p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  return rel::linear_tc_bwd_workspace_bytes(p);
}

}  // namespace

size_t relation_linear_bwd_ex_workspace_size(relation_shape shp, relation_dtype dt,
                                             relation_kernel kernel) {
  relation_status why;
  const int fam = linear_bwd_family(shp, dt, kernel, &why);
  return fam < 0 ? 0 : linear_bwd_bytes(shp, dt, fam);
}

size_t relation_linear_bwd_workspace_size(relation_shape shp, relation_dtype dt) {
  return relation_linear_bwd_ex_workspace_size(shp, dt, RELATION_KERNEL_AUTO);
}

relation_status relation_linear_bwd(const void* p1, const void* p2, const void* v,
                                   const float* alpha, const void* dy, void* dp1, void* dp2,
                                   void* dv, float* dalpha, float tau_s, relation_shape shp,
                                   relation_dtype dt, void* workspace, size_t ws_bytes,
                                   int* dev_status, relation_stream_t stream) {
  return relation_linear_bwd_ex(p1, p2, v, alpha, dy, dp1, dp2, dv, dalpha, tau_s, shp, dt,
                                RELATION_KERNEL_AUTO, workspace, ws_bytes, dev_status, stream);
}

relation_status relation_linear_bwd_ex(const void* p1, const void* p2, const void* v,
                                      const float* alpha, const void* dy, void* dp1, void* dp2,
                                      void* dv, float* dalpha, float tau_s, relation_shape shp,
                                      relation_dtype dt, relation_kernel kernel, void* workspace,
                                      size_t ws_bytes, int* dev_status,
                                      relation_stream_t stream) {
  relation_status st;
  const int fam = linear_bwd_family(shp, dt, kernel, &st);
  if (fam < 0) return st;
  if (!isfinite(tau_s) || !(tau_s > 0.0f)) return RELATION_ERR_INVALID_ARG;
  if ((st = check_ptrs({p1, p2, v, alpha, dy, dp1, dp2, dv, dalpha, workspace})) != RELATION_OK)
    return st;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  if (ws_bytes < linear_bwd_bytes(shp, dt, fam)) return RELATION_ERR_WORKSPACE;
  if (!aligned16(workspace)) return RELATION_ERR_ALIGNMENT;
  rel::LinearProblem p{};
  p.p1 = p1; p.p2 = p2; p.v = v; p.alpha = alpha; p.dy = dy;
  p.dp1 = dp1; p.dp2 = dp2; p.dv = dv; p.dalpha = dalpha; p.workspace = workspace;
  p.dev_status = dev_status; p.tau_s = tau_s;
  p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (fam == (int)RELATION_KERNEL_TCGEN05) return from_cuda(rel::launch_linear_tc_bwd(p, s));
  return from_cuda(rel::launch_linear_bwd(p, s));
}

namespace {

relation_status check_layer(const relation_shape& shp, relation_dtype dt, int pairing,
                            float rope_base) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (shp.B < 1 || shp.T < 1 || shp.H < 1 || shp.d_h < 1) return RELATION_ERR_INVALID_ARG;
  if (shp.sB < 1 || shp.sT < 1 || shp.sH < 1) return RELATION_ERR_INVALID_ARG;
  if (pairing != 0 && pairing != 1) return RELATION_ERR_INVALID_ARG;
  if (!isfinite(rope_base) || !(rope_base > 0.0f)) return RELATION_ERR_INVALID_ARG;
  if (!rel::layer_supports(dt, shp.d_h, shp.H)) return RELATION_ERR_UNSUPPORTED;
  if ((long long)shp.B * ((shp.T + 15) / 16) > 0x7fffffffLL) return RELATION_ERR_UNSUPPORTED;
  const long long vec = 16 / (long long)elem_size(dt);
  if (shp.sB % vec || shp.sT % vec || shp.sH % vec) return RELATION_ERR_ALIGNMENT;
  return RELATION_OK;
}

rel::LayerProblem layer_problem(const relation_shape& shp, relation_dtype dt, int pairing,
                                float rope_base, const float* theta) {
  rel::LayerProblem p{};
  p.theta = theta; p.pairing = pairing; p.rope_base = rope_base;
  p.B = shp.B; p.T = shp.T; p.H = shp.H; p.d = shp.d_h;
  p.sB = shp.sB; p.sT = shp.sT; p.sH = shp.sH; p.dtype = dt;
  return p;
}

}  // namespace

relation_status relation_layer_prep(const void* p1, const void* p2, const void* info,
                                    const float* theta, int pairing, float rope_base, void* q,
                                    void* k, void* v, relation_shape shp, relation_dtype dt,
                                    relation_stream_t stream) {
  relation_status st;
  if ((st = check_layer(shp, dt, pairing, rope_base)) != RELATION_OK) return st;
  if ((st = check_ptrs({p1, p2, info, q, k, v})) != RELATION_OK) return st;
  if (!theta || (reinterpret_cast<uintptr_t>(theta) & 3u)) return RELATION_ERR_INVALID_ARG;
  rel::LayerProblem p = layer_problem(shp, dt, pairing, rope_base, theta);
  p.in1 = p1; p.in2 = p2; p.in3 = info; p.out1 = q; p.out2 = k; p.out3 = v;
  return from_cuda(rel::launch_layer_prep(p, reinterpret_cast<cudaStream_t>(stream)));
}

size_t relation_layer_grad_workspace_size(relation_shape shp, relation_dtype dt) {
  if (check_layer(shp, dt, 0, 1.0f) != RELATION_OK) return 0;
  return rel::layer_grad_workspace_bytes(shp.B, shp.T, shp.H);
}

relation_status relation_layer_grad(const void* dq, const void* dk, const void* dv,
                                    const void* info, const float* theta, int pairing,
                                    float rope_base, void* dp1, void* dp2, void* dinfo,
                                    float* dtheta, relation_shape shp, relation_dtype dt,
                                    void* workspace, size_t ws_bytes, relation_stream_t stream) {
  relation_status st;
  if ((st = check_layer(shp, dt, pairing, rope_base)) != RELATION_OK) return st;
  if ((st = check_ptrs({dq, dk, dv, info, dp1, dp2, dinfo, workspace})) != RELATION_OK) return st;
  if (!theta || (reinterpret_cast<uintptr_t>(theta) & 3u)) return RELATION_ERR_INVALID_ARG;
  if (!dtheta || (reinterpret_cast<uintptr_t>(dtheta) & 3u)) return RELATION_ERR_INVALID_ARG;
  if (ws_bytes < rel::layer_grad_workspace_bytes(shp.B, shp.T, shp.H)) return RELATION_ERR_WORKSPACE;
  rel::LayerProblem p = layer_problem(shp, dt, pairing, rope_base, theta);
  p.in1 = dq; p.in2 = dk; p.in3 = dv; p.in4 = info;
  p.out1 = dp1; p.out2 = dp2; p.out3 = dinfo;
  p.dtheta = dtheta; p.dtheta_part = reinterpret_cast<float*>(workspace);
  return from_cuda(rel::launch_layer_grad(p, reinterpret_cast<cudaStream_t>(stream)));
}

size_t relation_decode_workspace_size(relation_shape cache, relation_dtype dt) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return 0;
  if (cache.B < 1 || cache.T < 1 || cache.H < 1 || cache.d_h < 1 || cache.d_h > 128) return 0;
  return rel::decode_workspace_bytes(cache.B, cache.H, cache.T);
}

relation_status relation_decode(const void* q, const void* k_cache, const void* v_cache,
                                const int* lengths, void* o, float* logz, float lambda,
                                float tau_s, relation_shape cache, long long q_sB, long long q_sH,
                                relation_dtype dt, void* workspace, size_t ws_bytes,
                                int* dev_status, relation_stream_t stream) {
  relation_status st;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (cache.B < 1 || cache.T < 1 || cache.H < 1 || cache.d_h < 1) return RELATION_ERR_INVALID_ARG;
  if (cache.d_h > 128) return RELATION_ERR_UNSUPPORTED;
  if ((long long)cache.B * cache.H > 0x7fffffffLL) return RELATION_ERR_UNSUPPORTED;
  if (cache.sB < 1 || cache.sT < 1 || cache.sH < 1 || q_sB < 1 || q_sH < 1)
    return RELATION_ERR_INVALID_ARG;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if ((st = check_ptrs({q, k_cache, v_cache, lengths, o, logz, workspace})) != RELATION_OK)
    return st;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  if (ws_bytes < rel::decode_workspace_bytes(cache.B, cache.H, cache.T))
    return RELATION_ERR_WORKSPACE;
  rel::DecodeProblem p{};
  p.q = q; p.k = k_cache; p.v = v_cache; p.lengths = lengths; p.out = o; p.logz = logz;
  p.dev_status = dev_status;
  p.lambda = lambda; p.tau_s = tau_s; p.inv_sqrt_d = 1.0f / sqrtf((float)cache.d_h);
  p.B = cache.B; p.T = cache.T; p.H = cache.H; p.d = cache.d_h;
  p.sB = cache.sB; p.sT = cache.sT; p.sH = cache.sH; p.qsB = q_sB; p.qsH = q_sH;
  p.dtype = dt;
  if (rel::decode_chunks(cache.T) > 65535) return RELATION_ERR_UNSUPPORTED;  // grid.y limit
  return from_cuda(rel::launch_decode(p, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_page_plan(const int* lengths, const int* counts, int B, int page_size,
                                   int* block_table, int cols, long long table_stride,
                                   int* free_pages, int n_pages, const int* free_state,
                                   int* free_state_out, int* lengths_out, int* starts,
                                   long long* slots, int* positions, int n_tokens,
                                   int* dev_status, relation_stream_t stream) {
  if (B < 1 || page_size < 1 || cols < 1 || n_pages < 1 || n_tokens < 1 || table_stride < cols)
    return RELATION_ERR_INVALID_ARG;
  if ((long long)cols * page_size > 0x7fffffffLL || (long long)B * cols > 0x7fffffffLL)
    return RELATION_ERR_UNSUPPORTED;
  for (const void* x : {(const void*)lengths, (const void*)counts, (const void*)block_table,
                        (const void*)free_pages, (const void*)free_state,
                        (const void*)free_state_out, (const void*)lengths_out,
                        (const void*)starts, (const void*)slots, (const void*)positions}) {
    if (!x) return RELATION_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x) & (x == slots ? 7u : 3u)) return RELATION_ERR_ALIGNMENT;
  }
  if (lengths_out == lengths || lengths_out == counts || free_state_out == free_state)
    return RELATION_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(dev_status) & 3u) return RELATION_ERR_ALIGNMENT;
  rel::PlanProblem p{};
  p.lengths = lengths; p.counts = counts; p.table = block_table; p.ring = free_pages;
  p.state = free_state; p.state_out = free_state_out; p.lengths_out = lengths_out;
  p.starts = starts; p.slots = slots; p.positions = positions; p.dev_status = dev_status;
  p.t_stride = table_stride; p.B = B; p.page = page_size; p.cols = cols; p.n_pages = n_pages;
  p.n_tokens = n_tokens;
  return from_cuda(rel::launch_plan(p, reinterpret_cast<cudaStream_t>(stream)));
}

namespace {

relation_status check_pages(const relation_pages& c, relation_dtype dt) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (c.n_pages < 1 || c.page_size < 1 || c.H < 1 || c.d_h < 1) return RELATION_ERR_INVALID_ARG;
  if (c.sP < 1 || c.sR < 1 || c.sH < 1) return RELATION_ERR_INVALID_ARG;
  return RELATION_OK;
}

// Null or not a multiple of the element size
relation_status check_elements(std::initializer_list<const void*> ptrs, size_t size) {
  for (const void* p : ptrs) {
    if (!p) return RELATION_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p) % size) return RELATION_ERR_ALIGNMENT;
  }
  return RELATION_OK;
}

}  // namespace

relation_status relation_cache_append(const void* p1, const void* p2, const void* info,
                                      const float* theta, int pairing, float rope_base,
                                      const int* positions, const long long* slots, void* q,
                                      int N, long long sT, long long sH, void* k_pages,
                                      void* v_pages, relation_pages cache, relation_dtype dt,
                                      int* dev_status, relation_stream_t stream) {
  relation_status st;
  if ((st = check_pages(cache, dt)) != RELATION_OK) return st;
  if (N < 1 || sT < 1 || sH < 1 || (pairing != 0 && pairing != 1)) return RELATION_ERR_INVALID_ARG;
  if (!isfinite(rope_base) || rope_base < 0.0f) return RELATION_ERR_INVALID_ARG;
  if ((p1 == nullptr) != (q == nullptr)) return RELATION_ERR_INVALID_ARG;
  if (rope_base > 0.0f && !positions) return RELATION_ERR_INVALID_ARG;
  if ((st = check_elements({p2, info, k_pages, v_pages}, elem_size(dt))) != RELATION_OK) return st;
  if (p1 && (st = check_elements({p1, q}, elem_size(dt))) != RELATION_OK) return st;
  if ((st = check_elements({slots}, 8)) != RELATION_OK) return st;
  for (const void* x : {(const void*)theta, (const void*)positions, (const void*)dev_status})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  if (cache.d_h > 256 || (rope_base > 0.0f && cache.d_h % 2) || (theta && cache.H % 2))
    return RELATION_ERR_UNSUPPORTED;
  if (N > 0x3fffffff || (long long)cache.H * cache.d_h > (1 << 24)) return RELATION_ERR_UNSUPPORTED;
  rel::AppendProblem p{};
  p.p1 = p1; p.p2 = p2; p.info = info; p.theta = theta; p.positions = positions; p.slots = slots;
  p.q = q; p.k = k_pages; p.v = v_pages; p.dev_status = dev_status;
  p.pairing = pairing; p.rope_base = rope_base;
  p.N = N; p.H = cache.H; p.d = cache.d_h; p.n_pages = cache.n_pages; p.page = cache.page_size;
  p.sT = sT; p.sH = sH; p.sP = cache.sP; p.sR = cache.sR; p.sC = cache.sH;
  p.dtype = dt;
  return from_cuda(rel::launch_append(p, reinterpret_cast<cudaStream_t>(stream)));
}

size_t relation_paged_decode_workspace_size(int H, relation_pages cache, relation_dtype dt) {
  if (check_pages(cache, dt) != RELATION_OK || cache.d_h > 128 || H < 1 || H % cache.H) return 0;
  return rel::paged_workspace_bytes(H, cache.H);
}

relation_status relation_paged_decode(const void* q, const void* k_pages, const void* v_pages,
                                      const int* block_table, int cols, long long table_stride,
                                      const int* lengths, void* o, float* logz, float lambda,
                                      float tau_s, int B, int H, relation_pages cache,
                                      long long q_sB, long long q_sH, relation_dtype dt,
                                      void* workspace, size_t ws_bytes, int* dev_status,
                                      relation_stream_t stream) {
  relation_status st;
  if ((st = check_pages(cache, dt)) != RELATION_OK) return st;
  if (B < 1 || H < 1 || H % cache.H || cols < 1 || table_stride < cols || q_sB < 1 || q_sH < 1)
    return RELATION_ERR_INVALID_ARG;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if (cache.d_h > 128) return RELATION_ERR_UNSUPPORTED;
  // (row numbers a few tiles past the last one fit in 32 bits)
  if ((long long)B * H > 0x7fff0000LL || (long long)cols * cache.page_size > 0x7fffe000LL)
    return RELATION_ERR_UNSUPPORTED;
  if ((st = check_elements({q, k_pages, v_pages, o}, elem_size(dt))) != RELATION_OK) return st;
  if ((st = check_elements({block_table, lengths, logz}, 4)) != RELATION_OK) return st;
  if (reinterpret_cast<uintptr_t>(dev_status) & 3u) return RELATION_ERR_ALIGNMENT;
  if (!workspace || ws_bytes < rel::paged_workspace_bytes(H, cache.H)) return RELATION_ERR_WORKSPACE;
  if (!aligned16(workspace)) return RELATION_ERR_ALIGNMENT;
  rel::PagedProblem p{};
  p.q = q; p.k = k_pages; p.v = v_pages; p.table = block_table; p.lengths = lengths;
  p.out = o; p.logz = logz; p.dev_status = dev_status;
  p.lambda = lambda; p.tau_s = tau_s; p.inv_sqrt_d = 1.0f / sqrtf((float)cache.d_h);
  p.B = B; p.H = H; p.Hk = cache.H; p.d = cache.d_h; p.cols = cols; p.n_pages = cache.n_pages;
  p.page = cache.page_size; p.t_stride = table_stride; p.sP = cache.sP; p.sR = cache.sR;
  p.sC = cache.sH; p.qsB = q_sB; p.qsH = q_sH; p.dtype = dt;
  return from_cuda(rel::launch_paged(p, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

namespace {

// The sizes of a relation_paged_chunk call
relation_status check_chunk(int N, int B, int H, int cols, const relation_pages& cache, relation_dtype dt) {
  relation_status st;
  if ((st = check_pages(cache, dt)) != RELATION_OK) return st;
  if (N < 1 || B < 1 || H < 1 || H % cache.H || cols < 1) return RELATION_ERR_INVALID_ARG;
  if (cache.d_h > 128) return RELATION_ERR_UNSUPPORTED;
  // (row numbers a few units past the last one, and tiles and their heads, fit in 32 bits)
  if ((long long)cols * cache.page_size > 0x7fffe000LL || (long long)N * H > 0x7fff0000LL ||
      ((long long)N + B) * H > 0x7fff0000LL)
    return RELATION_ERR_UNSUPPORTED;
  return RELATION_OK;
}

}  // namespace

size_t relation_paged_chunk_workspace_size(int N, int B, int H, int cols, relation_pages cache,
                                           relation_dtype dt) {
  if (check_chunk(N, B, H, cols, cache, dt) != RELATION_OK) return 0;
  return rel::chunk_workspace_bytes(N, B, H, cache.H, cache.d_h, cols * cache.page_size, dt);
}

relation_status relation_paged_chunk(const void* q, const void* k_pages, const void* v_pages,
                                     const int* block_table, int cols, long long table_stride,
                                     const int* starts, const int* positions, void* o, float* logz,
                                     float lambda, float tau_s, int N, int B, int H,
                                     relation_pages cache, long long q_sT, long long q_sH,
                                     relation_dtype dt, void* workspace, size_t ws_bytes,
                                     int* dev_status, relation_stream_t stream) {
  relation_status st;
  if ((st = check_chunk(N, B, H, cols, cache, dt)) != RELATION_OK) return st;
  if (table_stride < cols || q_sT < 1 || q_sH < 1) return RELATION_ERR_INVALID_ARG;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if ((st = check_elements({q, k_pages, v_pages, o}, elem_size(dt))) != RELATION_OK) return st;
  if ((st = check_elements({block_table, starts, positions, logz}, 4)) != RELATION_OK) return st;
  if (reinterpret_cast<uintptr_t>(dev_status) & 3u) return RELATION_ERR_ALIGNMENT;
  const int limit = cols * cache.page_size;
  if (!workspace || ws_bytes < rel::chunk_workspace_bytes(N, B, H, cache.H, cache.d_h, limit, dt))
    return RELATION_ERR_WORKSPACE;
  if (!aligned16(workspace)) return RELATION_ERR_ALIGNMENT;
  rel::ChunkProblem p{};
  p.q = q; p.k = k_pages; p.v = v_pages; p.table = block_table; p.starts = starts;
  p.positions = positions; p.out = o; p.logz = logz; p.dev_status = dev_status;
  p.lambda = lambda; p.tau_s = tau_s; p.inv_sqrt_d = 1.0f / sqrtf((float)cache.d_h);
  p.N = N; p.B = B; p.H = H; p.Hk = cache.H; p.d = cache.d_h; p.limit = limit;
  p.n_pages = cache.n_pages; p.page = cache.page_size; p.t_stride = table_stride; p.sP = cache.sP;
  p.sR = cache.sR; p.sC = cache.sH; p.qsT = q_sT; p.qsH = q_sH; p.dtype = dt;
  return from_cuda(rel::launch_chunk(p, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_sample(const void* logits, int R, int V, long long s_row,
                                relation_dtype dt, const float* u, const float* temperature,
                                const int* top_k, const float* top_p, const float* min_p,
                                int* token, float* logprob, float* logz, int* dev_status,
                                relation_stream_t stream) {
  relation_status st;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (R < 1 || V < 1 || (R > 1 && s_row < V)) return RELATION_ERR_INVALID_ARG;
  if ((st = check_elements({logits}, elem_size(dt))) != RELATION_OK) return st;
  if ((st = check_elements({u, token, logprob, logz}, 4)) != RELATION_OK) return st;
  for (const void* x : {(const void*)temperature, (const void*)top_k, (const void*)top_p,
                        (const void*)min_p, (const void*)dev_status})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  if (V > rel::sample_max_vocabulary() || R > (1 << 27)) return RELATION_ERR_UNSUPPORTED;
  rel::SampleProblem p{};
  p.logits = logits; p.u = u; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p;
  p.min_p = min_p; p.token = token; p.logprob = logprob; p.logz = logz; p.dev_status = dev_status;
  p.R = R; p.V = V; p.s_row = s_row; p.dtype = dt;
  return from_cuda(rel::launch_sample(p, reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_logprobs(const void* logits, int R, int V, long long s_row,
                                  relation_dtype dt, const int* targets, const float* temperature,
                                  float* logprob, float* entropy, float* logz, int top,
                                  int* top_tokens, float* top_logprobs, int* dev_status,
                                  relation_stream_t stream) {
  relation_status st;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (R < 1 || V < 1 || (R > 1 && s_row < V) || top < 0) return RELATION_ERR_INVALID_ARG;
  if ((st = check_elements({logits}, elem_size(dt))) != RELATION_OK) return st;
  if ((st = check_elements({targets, logprob, entropy, logz}, 4)) != RELATION_OK) return st;
  if (top > 0 && (st = check_elements({top_tokens, top_logprobs}, 4)) != RELATION_OK) return st;
  for (const void* x : {(const void*)temperature, (const void*)dev_status})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  if (top > rel::logprobs_max_top() || V > (1 << 30) || R > (1 << 27)) return RELATION_ERR_UNSUPPORTED;
  rel::LogprobsProblem p{};
  p.logits = logits; p.targets = targets; p.temperature = temperature; p.logprob = logprob;
  p.entropy = entropy; p.logz = logz; p.top_tokens = top_tokens; p.top_logprobs = top_logprobs;
  p.dev_status = dev_status; p.R = R; p.V = V; p.top = top; p.s_row = s_row; p.dtype = dt;
  return from_cuda(rel::launch_logprobs(p, reinterpret_cast<cudaStream_t>(stream)));
}

relation_status relation_logprobs_grad(const void* logits, int R, int V, long long s_row,
                                       relation_dtype dt, const int* targets,
                                       const float* temperature, const float* logz,
                                       const float* entropy, const float* dlogprob,
                                       const float* dentropy, const float* dlogz, void* dlogits,
                                       long long s_out, relation_stream_t stream) {
  relation_status st;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if (R < 1 || V < 1 || (R > 1 && (s_row < V || s_out < V))) return RELATION_ERR_INVALID_ARG;
  if ((st = check_elements({logits, dlogits}, elem_size(dt))) != RELATION_OK) return st;
  if (dlogits == logits && R > 1 && s_out != s_row) return RELATION_ERR_INVALID_ARG;
  if ((st = check_elements({targets, logz, entropy}, 4)) != RELATION_OK) return st;
  for (const void* x : {(const void*)temperature, (const void*)dlogprob, (const void*)dentropy,
                        (const void*)dlogz})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  // (a CTA takes at least 4096 elements of a row)
  if (V > (1 << 30) || (long long)R * (V / 4096 + 2) > 0x7fffffffLL) return RELATION_ERR_UNSUPPORTED;
  rel::LogprobsGradProblem p{};
  p.logits = logits; p.targets = targets; p.temperature = temperature; p.logz = logz;
  p.entropy = entropy; p.dlogprob = dlogprob; p.dentropy = dentropy; p.dlogz = dlogz;
  p.dlogits = dlogits; p.R = R; p.V = V; p.s_row = s_row; p.s_out = s_out; p.dtype = dt;
  return from_cuda(rel::launch_logprobs_grad(p, reinterpret_cast<cudaStream_t>(stream)));
}

namespace {

// The arguments that relation_norm_rope and its gradient share; p is filled from them
relation_status norm_rope_problem(const void* p1, const void* p2, const float* w1, const float* w2, int norm,
                                  float eps, const relation_rotary& rot, const int* positions,
                                  const relation_shape& sq, const relation_shape& sk, relation_dtype dt,
                                  rel::NormRopeProblem* p) {
  relation_status st;
  if (dt != RELATION_F32 && dt != RELATION_BF16) return RELATION_ERR_INVALID_ARG;
  if ((norm != 0 && norm != 1) || (rot.layout != 0 && rot.layout != 1)) return RELATION_ERR_INVALID_ARG;
  if (!isfinite(eps) || eps < 0.0f || !isfinite(rot.scale)) return RELATION_ERR_INVALID_ARG;
  if (sq.B < 1 || sq.T < 1 || sq.H < 1 || sq.d_h < 1 || sq.sB < 1 || sq.sT < 1 || sq.sH < 1)
    return RELATION_ERR_INVALID_ARG;
  if (p2 && (sk.B != sq.B || sk.T != sq.T || sk.d_h != sq.d_h || sk.H < 1 || sk.sB < 1 || sk.sT < 1 ||
             sk.sH < 1))
    return RELATION_ERR_INVALID_ARG;
  if (rot.d_rot < 0 || rot.d_rot > sq.d_h || rot.d_rot % 2) return RELATION_ERR_INVALID_ARG;
  if (rot.d_rot > 0 && (st = check_elements({rot.freqs}, 8)) != RELATION_OK) return st;
  if ((st = check_elements({p1}, elem_size(dt))) != RELATION_OK) return st;
  for (const void* x : {(const void*)w1, (const void*)w2, (const void*)positions})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  if (sq.d_h > 256 || (long long)sq.B * sq.T > (1 << 30)) return RELATION_ERR_UNSUPPORTED;
  // (a CTA's rows are counted in 32 bits)
  if ((long long)sq.H + (p2 ? sk.H : 0) > (1 << 24)) return RELATION_ERR_UNSUPPORTED;
  p->in[0] = p1; p->in[1] = p2; p->w[0] = w1; p->w[1] = w2;
  p->freqs = rot.freqs; p->d_rot = rot.d_rot; p->half = rot.layout; p->scale = rot.scale;
  p->positions = positions; p->eps = eps; p->norm = norm;
  p->B = sq.B; p->T = sq.T; p->d = sq.d_h; p->dtype = dt;
  p->H[0] = sq.H; p->sB[0] = sq.sB; p->sT[0] = sq.sT; p->sH[0] = sq.sH;
  if (p2) {
    p->H[1] = sk.H; p->sB[1] = sk.sB; p->sT[1] = sk.sT; p->sH[1] = sk.sH;
  }
  return RELATION_OK;
}

}  // namespace

relation_status relation_norm_rope(const void* p1, const void* p2, const float* w1, const float* w2,
                                   int norm, float eps, relation_rotary rotary,
                                   const int* positions, void* q, void* k, relation_shape shp_q,
                                   relation_shape shp_k, relation_dtype dt,
                                   relation_stream_t stream) {
  relation_status st;
  rel::NormRopeProblem p{};
  if ((p2 == nullptr) != (k == nullptr)) return RELATION_ERR_INVALID_ARG;
  if ((st = norm_rope_problem(p1, p2, w1, w2, norm, eps, rotary, positions, shp_q, shp_k, dt, &p)) != RELATION_OK)
    return st;
  if ((st = check_elements({q}, elem_size(dt))) != RELATION_OK) return st;
  if (p2 && (st = check_elements({p2, k}, elem_size(dt))) != RELATION_OK) return st;
  p.out[0] = q; p.out[1] = k;
  return from_cuda(rel::launch_norm_rope(p, false, reinterpret_cast<cudaStream_t>(stream)));
}

size_t relation_norm_rope_grad_workspace_size(relation_shape shp, relation_dtype dt) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return 0;
  if (shp.B < 1 || shp.T < 1 || shp.d_h < 1 || shp.d_h > 256 || (long long)shp.B * shp.T > (1 << 30)) return 0;
  return rel::norm_rope_grad_workspace_bytes(shp.d_h);
}

relation_status relation_norm_rope_grad(const void* dq, const void* dk, const void* p1,
                                        const void* p2, const float* w1, const float* w2, int norm,
                                        float eps, relation_rotary rotary, const int* positions,
                                        void* dp1, void* dp2, float* dw1, float* dw2,
                                        relation_shape shp_q, relation_shape shp_k,
                                        relation_dtype dt, void* workspace, size_t ws_bytes,
                                        relation_stream_t stream) {
  relation_status st;
  rel::NormRopeProblem p{};
  if ((p2 == nullptr) != (dk == nullptr) || (p2 == nullptr) != (dp2 == nullptr) || (!p2 && dw2))
    return RELATION_ERR_INVALID_ARG;
  if ((st = norm_rope_problem(p1, p2, w1, w2, norm, eps, rotary, positions, shp_q, shp_k, dt, &p)) != RELATION_OK)
    return st;
  if ((st = check_elements({dq, dp1}, elem_size(dt))) != RELATION_OK) return st;
  if (p2 && (st = check_elements({dk, p2, dp2}, elem_size(dt))) != RELATION_OK) return st;
  for (const void* x : {(const void*)dw1, (const void*)dw2})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return RELATION_ERR_ALIGNMENT;
  if (dw1 || dw2) {
    if (!workspace || ws_bytes < rel::norm_rope_grad_workspace_bytes(p.d))
      return RELATION_ERR_WORKSPACE;
    if (!aligned16(workspace)) return RELATION_ERR_ALIGNMENT;
    p.part = static_cast<float*>(workspace);
  }
  p.dout[0] = dq; p.dout[1] = dk; p.out[0] = dp1; p.out[1] = dp2; p.dw[0] = dw1; p.dw[1] = dw2;
  return from_cuda(rel::launch_norm_rope(p, true, reinterpret_cast<cudaStream_t>(stream)));
}

size_t relation_bwd_workspace_size(relation_shape shp, relation_dtype dt) {
  if (check_shape(shp, dt) != RELATION_OK) return 0;
  return rel::bwd_workspace_bytes(shp.B, shp.H, shp.T, shp.d_h);
}

relation_status relation_bwd_stages(const void* q, const void* k, const void* v, const void* o,
                                    const void* dout, const float* logz, void* dq, void* dk,
                                    void* dv, float* dlambda, float lambda, float tau_s,
                                    relation_shape shp, relation_dtype dt, void* workspace,
                                    size_t ws_bytes, relation_kernel kernel, unsigned stages,
                                    int* dev_status, relation_stream_t stream) {
  relation_status st;
  if (stages == 0 || (stages & ~7u)) return RELATION_ERR_INVALID_ARG;
  if ((st = check_shape(shp, dt)) != RELATION_OK) return st;
  if ((st = check_scalars(lambda, tau_s)) != RELATION_OK) return st;
  if ((st = check_ptrs({q, k, v, o, dout, logz, dq, dk, dv})) != RELATION_OK) return st;
  if (!dlambda) return RELATION_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(dlambda) & 3u) return RELATION_ERR_ALIGNMENT;
  if (dev_status && (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return RELATION_ERR_ALIGNMENT;
  const size_t need = rel::bwd_workspace_bytes(shp.B, shp.H, shp.T, shp.d_h);
  if (!workspace || ws_bytes < need) return RELATION_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return RELATION_ERR_ALIGNMENT;
  const int fam = pick_family(kernel, dt, shp.d_h, true);
  if (fam == 0) return RELATION_ERR_UNSUPPORTED;

  Problem p = make_problem(shp, dt, lambda, tau_s, dev_status);
  p.q = q; p.k = k; p.v = v; p.o = o; p.dout = dout; p.logz_in = logz;
  p.dq = dq; p.dk = dk; p.dv = dv; p.dlambda = dlambda;
  rel::BwdWorkspace ws = rel::carve_workspace(workspace, shp.B, shp.H, shp.T, shp.d_h);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (fam == 2) return from_cuda(rel::tc::launch_bwd(p, ws, stages, s));
  cudaError_t e = cudaSuccess;
  if ((stages & 1) && (e = rel::bwd_common::launch_pre(p, ws, s)) != cudaSuccess) return from_cuda(e);
  if ((stages & 2) && (e = rel::simt::launch_bwd(p, ws, s)) != cudaSuccess) return from_cuda(e);
  if (stages & 4) e = rel::bwd_common::launch_dlambda(p, ws, rel::simt::main_partials(ws),
                                                   rel::simt::main_ctas(p), s);
  return from_cuda(e);
}

relation_status relation_bwd_ex(const void* q, const void* k, const void* v, const void* o,
                                const void* dout, const float* logz, void* dq, void* dk, void* dv,
                                float* dlambda, float lambda, float tau_s, relation_shape shp,
                                relation_dtype dt, void* workspace, size_t ws_bytes,
                                relation_kernel kernel, int* dev_status, relation_stream_t stream) {
  return relation_bwd_stages(q, k, v, o, dout, logz, dq, dk, dv, dlambda, lambda, tau_s, shp, dt,
                             workspace, ws_bytes, kernel, RELATION_BWD_ALL, dev_status, stream);
}

relation_status relation_bwd(const void* q, const void* k, const void* v, const void* o,
                             const void* dout, const float* logz, void* dq, void* dk, void* dv,
                             float* dlambda, float lambda, float tau_s, relation_shape shp,
                             relation_dtype dt, void* workspace, size_t ws_bytes,
                             int* dev_status, relation_stream_t stream) {
  return relation_bwd_ex(q, k, v, o, dout, logz, dq, dk, dv, dlambda, lambda, tau_s, shp, dt,
                         workspace, ws_bytes, RELATION_KERNEL_AUTO, dev_status, stream);
}

const char* relation_status_string(relation_status s) {
  switch (s) {
    case RELATION_OK: return "RELATION_OK";
    case RELATION_ERR_INVALID_ARG: return "RELATION_ERR_INVALID_ARG";
    case RELATION_ERR_UNSUPPORTED: return "RELATION_ERR_UNSUPPORTED";
    case RELATION_ERR_ALIGNMENT: return "RELATION_ERR_ALIGNMENT";
    case RELATION_ERR_WORKSPACE: return "RELATION_ERR_WORKSPACE";
    case RELATION_ERR_CUDA: return "RELATION_ERR_CUDA";
    case RELATION_ERR_TIMEOUT: return "RELATION_ERR_TIMEOUT";
    case RELATION_ERR_CAPACITY: return "RELATION_ERR_CAPACITY";
  }
  return "RELATION_ERR_UNKNOWN";
}

const char* relation_last_cuda_error(void) {
  snprintf(g_last_message, sizeof(g_last_message), "%s%s%s", g_last_where,
           g_last_where[0] ? ": " : "", cudaGetErrorString(g_last_cuda_error));
  return g_last_message;
}

int relation_version(void) { return (1 << 16) | 0; }

int relation_launch_count(relation_dtype dt, int d_h, relation_kernel kernel, int backward) {
  if (dt != RELATION_F32 && dt != RELATION_BF16) return 0;
  const int fam = pick_family(kernel, dt, d_h, backward != 0);
  if (fam == 0) return 0;
  if (!backward) return 1;
  // SIMT: row pre-pass, tile kernel (dK/dV and dQ CTAs), dlambda reduction;
  // tcgen05: row pass, tile kernel, finalisation (dQ conversion + dlambda reduction)
  return fam == 2 ? rel::tc::bwd_launches() : 3;
}

relation_status relation_selftest_wait_timeout(int* dev_status, int timeout_us,
                                               relation_stream_t stream) {
  if (!dev_status || timeout_us < 1 || timeout_us > 100000) return RELATION_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(dev_status) & 3u) return RELATION_ERR_ALIGNMENT;
  return from_cuda(
      rel::launch_selftest_wait(dev_status, timeout_us, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
