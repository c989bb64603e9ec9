// The C ABI of the conditioning operators (include/ultratex.h): argument
// validation on the host, then the launches.  Nothing here allocates, frees
// or synchronises.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ultratex.h"
#include "gnorm.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "xattn.cuh"

namespace ut {

static bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static bool at4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

static ut_status status_of(cudaError_t e) { return e == cudaSuccess ? UT_OK : UT_ERR_CUDA; }

// ------------------------------------------------------------ cross attention
static ut_status xattn_problem(const ut_xattn_shape* s, bool backward, XattnParams* p) {
  if (!s) return UT_ERR_INVALID_ARG;
  if (s->n_q < 0 || s->n_k < 0 || s->n_seg < 1 || s->n_heads < 1 || s->n_kv_heads < 1 || s->head_dim < 1)
    return UT_ERR_INVALID_ARG;
  if (s->dtype != UT_BF16 && s->dtype != UT_F32) return UT_ERR_INVALID_ARG;
  if (s->n_heads % s->n_kv_heads != 0) return UT_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return UT_ERR_UNSUPPORTED;
  if (s->n_heads / s->n_kv_heads > 64 || s->n_kv_heads > 65535) return UT_ERR_UNSUPPORTED;
  if (s->n_q > INT32_MAX / 2 || s->n_k > INT32_MAX / 2 || s->n_seg > INT32_MAX / 4) return UT_ERR_UNSUPPORTED;
  const int64_t esz = s->dtype == UT_BF16 ? 2 : 4, qw = (int64_t)s->n_heads * s->head_dim,
                kw = (int64_t)s->n_kv_heads * s->head_dim;
  const int64_t strides[8] = {s->q_stride, s->o_stride, s->do_stride, s->dq_stride,
                              s->k_stride, s->v_stride, s->dk_stride, s->dv_stride};
  const bool fwd_too[8] = {true, true, false, false, true, true, false, false};
  for (int i = 0; i < 8; ++i) {
    if (!backward && !fwd_too[i]) continue;
    if (strides[i] < (i < 4 ? qw : kw) || (strides[i] * esz) % 16 != 0 || strides[i] > ((int64_t)1 << 38) / esz)
      return UT_ERR_INVALID_ARG;
  }
  *p = XattnParams{};
  p->nq = s->n_q;
  p->nk = s->n_k;
  p->B = s->n_seg;
  p->H = s->n_heads;
  p->Hk = s->n_kv_heads;
  p->G = s->n_heads / s->n_kv_heads;
  p->d = s->head_dim;
  p->qs = s->q_stride;
  p->ks = s->k_stride;
  p->vs = s->v_stride;
  p->os = s->o_stride;
  p->dos = s->do_stride;
  p->dqs = s->dq_stride;
  p->dks = s->dk_stride;
  p->dvs = s->dv_stride;
  p->sms = device_sms();
  const bool bf16 = s->dtype == UT_BF16;
  if (xattn_items(*p, bf16, backward) > INT32_MAX / 2) return UT_ERR_UNSUPPORTED;
  p->nsplit = xattn_splits(*p, bf16, backward);
  return UT_OK;
}

static size_t xattn_fwd_ws(const XattnParams& p) {
  if (p.nsplit == 1) return 0;
  const size_t rows = (size_t)p.nsplit * p.nq * p.H;
  return up256(rows * p.d * sizeof(float)) + up256(rows * sizeof(float2));
}

// D, then partial dK and dV
static size_t xattn_bwd_ws(const XattnParams& p, bool bf16) {
  const size_t part = up256((size_t)p.nsplit * p.nk * p.Hk * p.d * sizeof(float));
  return up256((size_t)p.H * p.nq * sizeof(float)) + (bf16 ? xattn_bwd_tc_ws(p) : 2 * part);
}

static ut_status xattn_pointers(const ut_xattn_shape* s, const XattnParams& p) {
  if ((p.cu_q == nullptr) != (p.cu_k == nullptr) || (!p.cu_q && s->n_seg != 1)) return UT_ERR_INVALID_ARG;
  if (!at4(p.cu_q) || !at4(p.cu_k) || !at4(p.status)) return UT_ERR_INVALID_ARG;
  if (!(p.scale > 0.f) || !isfinite(p.scale)) return UT_ERR_INVALID_ARG;
  if (p.nq > 0 && (!p.q || !p.o || !p.lse)) return UT_ERR_INVALID_ARG;
  if (p.nk > 0 && (!p.k || !p.v)) return UT_ERR_INVALID_ARG;
  if (!at16(p.q) || !at16(p.k) || !at16(p.v) || !at16(p.o) || !at4(p.lse)) return UT_ERR_INVALID_ARG;
  return UT_OK;
}

// ----------------------------------------------------------------- group norm
static ut_status gnorm_problem(const ut_gnorm_shape* s, bool backward, GnormParams* p) {
  if (!s) return UT_ERR_INVALID_ARG;
  if (s->n_rows < 0 || s->n_seg < 1 || s->channels < 1 || s->groups < 1 || s->channels % s->groups != 0)
    return UT_ERR_INVALID_ARG;
  if (s->dtype != UT_BF16 && s->dtype != UT_F32) return UT_ERR_INVALID_ARG;
  if (s->act != UT_ACT_NONE && s->act != UT_ACT_SILU) return UT_ERR_INVALID_ARG;
  if (!(s->eps > 0.f) || !isfinite(s->eps)) return UT_ERR_INVALID_ARG;
  const int64_t esz = s->dtype == UT_BF16 ? 2 : 4;
  if ((s->channels * esz) % 16 != 0) return UT_ERR_INVALID_ARG;
  const int64_t strides[4] = {s->x_stride, s->y_stride, s->dy_stride, s->dx_stride};
  for (int i = 0; i < 4; ++i) {
    if (i == 1 ? backward : (i > 1 && !backward)) continue;
    if (strides[i] < s->channels || (strides[i] * esz) % 16 != 0 || strides[i] > ((int64_t)1 << 38) / esz)
      return UT_ERR_INVALID_ARG;
  }
  if (s->channels > kGnMaxChannels || s->channels + s->groups > kGnMaxBoth) return UT_ERR_UNSUPPORTED;
  if (s->n_rows > INT32_MAX / 2 || s->n_seg > INT32_MAX / 4) return UT_ERR_UNSUPPORTED;
  *p = GnormParams{};
  p->n = s->n_rows;
  p->xs = s->x_stride;
  p->ys = s->y_stride;
  p->dys = s->dy_stride;
  p->dxs = s->dx_stride;
  p->B = s->n_seg;
  p->C = s->channels;
  p->G = s->groups;
  p->act = s->act;
  p->eps = s->eps;
  p->sms = device_sms();
  p->timeout_ns = wait_timeout_ns();
  return UT_OK;
}

}  // namespace ut

using namespace ut;

extern "C" {

size_t ut_xattn_fwd_workspace_size(const ut_xattn_shape* shape) {
  XattnParams p;
  return xattn_problem(shape, false, &p) == UT_OK ? xattn_fwd_ws(p) : 0;
}

ut_status ut_xattn_fwd(const ut_xattn_shape* shape, const void* q, const void* k, const void* v,
                       const int32_t* cu_q, const int32_t* cu_k, const uint8_t* key_mask, float softmax_scale,
                       void* o, float* lse, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  XattnParams p;
  ut_status st = xattn_problem(shape, false, &p);
  if (st != UT_OK) return st;
  p.q = q;
  p.k = k;
  p.v = v;
  p.o = o;
  p.lse = lse;
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  p.mask = key_mask;
  p.scale = softmax_scale;
  p.status = dev_status;
  p.timeout_ns = wait_timeout_ns();
  st = xattn_pointers(shape, p);
  if (st != UT_OK) return st;
  if (p.nq == 0) return UT_OK;
  const size_t need = xattn_fwd_ws(p);
  if (need > 0) {
    if (!ws || ws_bytes < need || !at16(ws)) return UT_ERR_INVALID_ARG;
    p.part_o = static_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) +
                                          up256((size_t)p.nsplit * p.nq * p.H * p.d * sizeof(float)));
  }
  const bool bf16 = shape->dtype == UT_BF16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = bf16 ? launch_xattn_fwd_tc(p, s) : launch_xattn_fwd_simt(p, s);
  if (e == cudaSuccess && p.nsplit > 1) e = launch_xattn_join(p, bf16, s);
  return status_of(e);
}

size_t ut_xattn_bwd_workspace_size(const ut_xattn_shape* shape) {
  XattnParams p;
  return xattn_problem(shape, true, &p) == UT_OK ? xattn_bwd_ws(p, shape->dtype == UT_BF16) : 0;
}

ut_status ut_xattn_bwd(const ut_xattn_shape* shape, const void* q, const void* k, const void* v,
                       const int32_t* cu_q, const int32_t* cu_k, const uint8_t* key_mask, float softmax_scale,
                       const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv, void* ws,
                       size_t ws_bytes, int32_t* dev_status, void* stream) {
  XattnParams p;
  ut_status st = xattn_problem(shape, true, &p);
  if (st != UT_OK) return st;
  p.q = q;
  p.k = k;
  p.v = v;
  p.o = const_cast<void*>(o);
  p.lse = const_cast<float*>(lse);
  p.dout = dout;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  p.mask = key_mask;
  p.scale = softmax_scale;
  p.status = dev_status;
  p.timeout_ns = wait_timeout_ns();
  st = xattn_pointers(shape, p);
  if (st != UT_OK) return st;
  if ((p.nq > 0 && (!dout || !dq)) || (p.nk > 0 && (!dk || !dv))) return UT_ERR_INVALID_ARG;
  if (!at16(dout) || !at16(dq) || !at16(dk) || !at16(dv)) return UT_ERR_INVALID_ARG;
  if (p.nq == 0 && p.nk == 0) return UT_OK;
  const bool bf16 = shape->dtype == UT_BF16;
  const size_t need = xattn_bwd_ws(p, bf16);  // 0 for bf16 without queries
  if (need > 0 && (!ws || ws_bytes < need || !at16(ws))) return UT_ERR_INVALID_ARG;
  char* w = static_cast<char*>(ws);
  p.dsum = reinterpret_cast<float*>(w);
  w += up256((size_t)p.H * p.nq * sizeof(float));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (bf16) return status_of(launch_xattn_bwd_tc(p, w, s));
  p.part_dk = reinterpret_cast<float*>(w);
  p.part_dv = reinterpret_cast<float*>(w + up256((size_t)p.nsplit * p.nk * p.Hk * p.d * sizeof(float)));
  return status_of(launch_xattn_bwd_simt(p, s));
}

size_t ut_group_norm_fwd_workspace_size(const ut_gnorm_shape* shape) {
  GnormParams p;
  return gnorm_problem(shape, false, &p) == UT_OK ? gnorm_ws(p, false) : 0;
}

ut_status ut_group_norm_fwd(const ut_gnorm_shape* shape, const void* x, const int32_t* cu, const float* gamma,
                            const float* beta, void* y, float* mean, float* rstd, void* ws, size_t ws_bytes,
                            int32_t* dev_status, void* stream) {
  GnormParams p;
  ut_status st = gnorm_problem(shape, false, &p);
  if (st != UT_OK) return st;
  if ((!cu && p.B != 1) || !mean || !rstd || (p.n > 0 && (!x || !y))) return UT_ERR_INVALID_ARG;
  if (!at16(x) || !at16(y) || !at4(cu) || !at4(gamma) || !at4(beta) || !at4(mean) || !at4(rstd) || !at4(dev_status))
    return UT_ERR_INVALID_ARG;
  if (!ws || ws_bytes < gnorm_ws(p, false) || !at16(ws)) return UT_ERR_INVALID_ARG;
  p.x = x;
  p.y = y;
  p.cu = cu;
  p.gamma = gamma;
  p.beta = beta;
  p.mean = mean;
  p.rstd = rstd;
  p.status = dev_status;
  p.ws = ws;
  return status_of(launch_gnorm_fwd(p, shape->dtype == UT_BF16, static_cast<cudaStream_t>(stream)));
}

size_t ut_group_norm_bwd_workspace_size(const ut_gnorm_shape* shape) {
  GnormParams p;
  return gnorm_problem(shape, true, &p) == UT_OK ? gnorm_ws(p, true) : 0;
}

ut_status ut_group_norm_bwd(const ut_gnorm_shape* shape, const void* x, const void* dy, const int32_t* cu,
                            const float* gamma, const float* beta, const float* mean, const float* rstd, void* dx,
                            float* dgamma, float* dbeta, void* ws, size_t ws_bytes, int32_t* dev_status,
                            void* stream) {
  GnormParams p;
  ut_status st = gnorm_problem(shape, true, &p);
  if (st != UT_OK) return st;
  if ((!cu && p.B != 1) || !mean || !rstd || (p.n > 0 && (!x || !dy || !dx))) return UT_ERR_INVALID_ARG;
  if (!at16(x) || !at16(dy) || !at16(dx) || !at4(cu) || !at4(gamma) || !at4(beta) || !at4(mean) || !at4(rstd) ||
      !at4(dgamma) || !at4(dbeta) || !at4(dev_status))
    return UT_ERR_INVALID_ARG;
  if (!ws || ws_bytes < gnorm_ws(p, true) || !at16(ws)) return UT_ERR_INVALID_ARG;
  p.x = x;
  p.dy = dy;
  p.dx = dx;
  p.cu = cu;
  p.gamma = gamma;
  p.beta = beta;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.dgamma = dgamma;
  p.dbeta = dbeta;
  p.status = dev_status;
  p.ws = ws;
  return status_of(launch_gnorm_bwd(p, shape->dtype == UT_BF16, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
