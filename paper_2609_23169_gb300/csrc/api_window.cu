// The C ABI of the windowed-attention operators (include/ultratex.h): argument
// validation on the host, then the launches.  Nothing here allocates, frees or
// synchronises.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ultratex.h"
#include "checks.h"
#include "kernels.h"
#include "qknorm.cuh"
#include "wattn.cuh"

namespace ut {

// --------------------------------------------------- norms of queries and keys
static bool row_ok(int64_t stride, int64_t width, int64_t esz) {
  return stride >= width && (stride * esz) % 16 == 0 && stride <= ((int64_t)1 << 38) / esz;
}

static ut_status qknorm_problem(const ut_qknorm_shape* s, const ut_rope* rope, bool backward, QkNormParams* p) {
  if (!s || !rope) return UT_ERR_INVALID_ARG;
  if (s->n_rows < 0 || s->n_heads < 1 || s->n_kv_heads < 1 || s->head_dim < 1) return UT_ERR_INVALID_ARG;
  if (s->dtype != UT_BF16 && s->dtype != UT_F32) return UT_ERR_INVALID_ARG;
  if (!(s->eps > 0.f) || !isfinite(s->eps)) return UT_ERR_INVALID_ARG;
  if (rope->side < 1 || rope->prefix < 0 || !(rope->theta > 0.f) || !isfinite(rope->theta)) return UT_ERR_INVALID_ARG;
  int64_t dims = 0;
  for (int a = 0; a < 3; ++a) {
    if (rope->axes[a] < 0 || rope->axes[a] % 2) return UT_ERR_INVALID_ARG;
    dims += rope->axes[a];
  }
  if (dims != s->head_dim) return UT_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return UT_ERR_UNSUPPORTED;
  if (s->n_rows > INT32_MAX / 2 || s->n_heads > 65535 || s->n_kv_heads > 65535) return UT_ERR_UNSUPPORTED;
  const int64_t esz = s->dtype == UT_BF16 ? 2 : 4, qw = (int64_t)s->n_heads * s->head_dim,
                kw = (int64_t)s->n_kv_heads * s->head_dim;
  if (!row_ok(s->q_stride, qw, esz) || !row_ok(s->k_stride, kw, esz)) return UT_ERR_INVALID_ARG;
  if (!row_ok(s->qo_stride, qw, esz) || !row_ok(s->ko_stride, kw, esz)) return UT_ERR_INVALID_ARG;
  if (backward && (!row_ok(s->dqo_stride, qw, esz) || !row_ok(s->dko_stride, kw, esz))) return UT_ERR_INVALID_ARG;
  *p = QkNormParams{};
  p->n = s->n_rows;
  p->H = s->n_heads;
  p->Hk = s->n_kv_heads;
  p->d = s->head_dim;
  p->qs = s->q_stride;
  p->ks = s->k_stride;
  p->vs = s->v_stride;
  p->qos = s->qo_stride;
  p->kos = s->ko_stride;
  p->vos = s->vo_stride;
  p->dqos = s->dqo_stride;
  p->dkos = s->dko_stride;
  p->cache_rows = s->cache_rows;
  p->eps = s->eps;
  p->side = (uint32_t)rope->side;
  const uint64_t area = (uint64_t)rope->side * rope->side;
  p->area = area > 0x80000000ull ? 0x80000000u : (uint32_t)area;
  p->prefix = rope->prefix;
  int at = 0;
  for (int a = 0; a < 3; ++a)
    for (int j = 0; j < rope->axes[a] / 2; ++j, ++at) {
      // whole turns a token make no difference
      const double t = fmod(pow((double)rope->theta, -2.0 * j / rope->axes[a]) / 6.283185307179586476925287, 1.0);
      p->turn[at] = (uint64_t)ldexp(t, 64);
      p->axis[at] = (uint8_t)a;
    }
  p->sms = device_sms();
  return UT_OK;
}

static size_t qknorm_ws(const QkNormParams& p) {
  return (size_t)qknorm_bwd_blocks(p.n, p.sms) * 2 * p.d * sizeof(float);
}

// ---------------------------------------------------------- windowed attention
static ut_status window_problem(const ut_xattn_shape* s, const ut_window* win, bool backward, WinParams* w) {
  *w = WinParams{};
  const ut_status st = xattn_shape(s, backward, &w->x);
  if (st != UT_OK) return st;
  if (!win || win->left < 0 || win->right < 0 || win->sinks < 0) return UT_ERR_INVALID_ARG;
  w->left = win->left < kWinMost ? win->left : kWinMost;
  w->right = win->right < kWinMost ? win->right : kWinMost;
  w->sinks = win->sinks < kWinMost ? win->sinks : kWinMost;
  if (s->n_q > kWinMost || s->n_k > kWinMost) return UT_ERR_UNSUPPORTED;
  const bool tc = s->dtype == UT_BF16;
  const int64_t items = !tc ? wattn_simt_items(*w, backward) : (backward ? wattn_bwd_tc_items(*w) : wattn_fwd_tc_items(*w));
  if (items > INT32_MAX / 2) return UT_ERR_UNSUPPORTED;
  w->x.nsplit = backward ? 1 : (tc ? wattn_fwd_tc_splits(*w) : wattn_simt_splits(*w));
  if (!tc && backward) wattn_simt_parts(*w);
  return UT_OK;
}

static size_t window_fwd_ws(const XattnParams& p) {
  if (p.nsplit == 1) return 0;
  const size_t rows = (size_t)p.nsplit * p.nq * p.H;
  return up256(rows * p.d * sizeof(float)) + up256(rows * sizeof(float2));
}

// D, then partial dK and dV
static size_t window_bwd_ws(const WinParams& w, bool bf16) {
  const XattnParams& p = w.x;
  return up256((size_t)p.H * p.nq * sizeof(float)) +
         (bf16 ? wattn_bwd_tc_ws(w) : 2 * up256(wattn_simt_part_rows(w) * p.Hk * p.d * sizeof(float)));
}

}  // namespace ut

using namespace ut;

extern "C" {

ut_status ut_qk_norm_rope_fwd(const ut_qknorm_shape* shape, const ut_rope* rope, const int32_t* pos, const void* q,
                              const void* k, const void* v, const float* wq, const float* wk, const int32_t* rows,
                              void* q_out, void* k_out, void* v_out, int32_t* dev_status, void* stream) {
  QkNormParams p;
  const ut_status st = qknorm_problem(shape, rope, false, &p);
  if (st != UT_OK) return st;
  const int64_t esz = shape->dtype == UT_BF16 ? 2 : 4, kw = (int64_t)p.Hk * p.d;
  if (p.n > 0 && (v == nullptr) != (v_out == nullptr)) return UT_ERR_INVALID_ARG;  // (no rows have no address)
  if (v && (!row_ok(shape->v_stride, kw, esz) || !row_ok(shape->vo_stride, kw, esz))) return UT_ERR_INVALID_ARG;
  if (rows && (shape->cache_rows < 0 || shape->cache_rows > INT32_MAX / 2)) return UT_ERR_INVALID_ARG;
  if (!at16(q) || !at16(k) || !at16(v) || !at16(q_out) || !at16(k_out) || !at16(v_out)) return UT_ERR_INVALID_ARG;
  if (!at4(pos) || !at4(wq) || !at4(wk) || !at4(rows) || !at4(dev_status)) return UT_ERR_INVALID_ARG;
  if (p.n == 0) return UT_OK;
  if (!q || !k || !q_out || !k_out) return UT_ERR_INVALID_ARG;
  p.q = q;
  p.k = k;
  p.v = v;
  p.wq = wq;
  p.wk = wk;
  p.pos = pos;
  p.rows = rows;
  p.qo = q_out;
  p.ko = k_out;
  p.vo = v_out;
  p.status = dev_status;
  return status_of(launch_qknorm_fwd(p, shape->dtype == UT_BF16, static_cast<cudaStream_t>(stream)));
}

size_t ut_qk_norm_rope_bwd_workspace_size(const ut_qknorm_shape* shape, const ut_rope* rope) {
  QkNormParams p;
  return qknorm_problem(shape, rope, true, &p) == UT_OK ? qknorm_ws(p) : 0;
}

ut_status ut_qk_norm_rope_bwd(const ut_qknorm_shape* shape, const ut_rope* rope, const int32_t* pos, const void* q,
                              const void* k, const float* wq, const float* wk, const void* dqo, const void* dko,
                              void* dq, void* dk, float* dwq, float* dwk, void* ws, size_t ws_bytes, void* stream) {
  QkNormParams p;
  const ut_status st = qknorm_problem(shape, rope, true, &p);
  if (st != UT_OK) return st;
  if (!at16(q) || !at16(k) || !at16(dqo) || !at16(dko) || !at16(dq) || !at16(dk)) return UT_ERR_INVALID_ARG;
  if (!at4(pos) || !at4(wq) || !at4(wk) || !at4(dwq) || !at4(dwk)) return UT_ERR_INVALID_ARG;
  if (p.n > 0 && (!q || !k || !dqo || !dko || !dq || !dk)) return UT_ERR_INVALID_ARG;
  if (p.n > 0 && (!ws || ws_bytes < qknorm_ws(p) || !at16(ws))) return UT_ERR_INVALID_ARG;
  p.q = q;
  p.k = k;
  p.wq = wq;
  p.wk = wk;
  p.pos = pos;
  p.dqo = dqo;
  p.dko = dko;
  p.qo = dq;
  p.ko = dk;
  p.dwq = dwq;
  p.dwk = dwk;
  p.part = static_cast<float*>(ws);
  return status_of(launch_qknorm_bwd(p, shape->dtype == UT_BF16, static_cast<cudaStream_t>(stream)));
}

size_t ut_window_attn_fwd_workspace_size(const ut_xattn_shape* shape, const ut_window* window) {
  WinParams w;
  return window_problem(shape, window, false, &w) == UT_OK ? window_fwd_ws(w.x) : 0;
}

ut_status ut_window_attn_fwd(const ut_xattn_shape* shape, const ut_window* window, const void* q, const void* k,
                             const void* v, const int32_t* cu_q, const int32_t* cu_k, const int32_t* k_len,
                             const uint8_t* key_mask, float softmax_scale, void* o, float* lse, void* ws,
                             size_t ws_bytes, int32_t* dev_status, void* stream) {
  WinParams w;
  ut_status st = window_problem(shape, window, false, &w);
  if (st != UT_OK) return st;
  XattnParams& p = w.x;
  p.q = q;
  p.k = k;
  p.v = v;
  p.o = o;
  p.lse = lse;
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  w.k_len = k_len;
  p.mask = key_mask;
  p.scale = softmax_scale;
  p.status = dev_status;
  p.timeout_ns = wait_timeout_ns();
  st = xattn_pointers(shape, p);
  if (st != UT_OK) return st;
  if (!at4(k_len)) return UT_ERR_INVALID_ARG;
  if (p.nq == 0) return UT_OK;
  const size_t need = window_fwd_ws(p);
  if (need > 0) {
    if (!ws || ws_bytes < need || !at16(ws)) return UT_ERR_INVALID_ARG;
    p.part_o = static_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) +
                                          up256((size_t)p.nsplit * p.nq * p.H * p.d * sizeof(float)));
  }
  const bool bf16 = shape->dtype == UT_BF16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = bf16 ? launch_wattn_fwd_tc(w, s) : launch_wattn_fwd_simt(w, s);
  if (e == cudaSuccess && p.nsplit > 1) e = launch_xattn_join(p, bf16, s);
  return status_of(e);
}

size_t ut_window_attn_bwd_workspace_size(const ut_xattn_shape* shape, const ut_window* window) {
  WinParams w;
  return window_problem(shape, window, true, &w) == UT_OK ? window_bwd_ws(w, shape->dtype == UT_BF16) : 0;
}

ut_status ut_window_attn_bwd(const ut_xattn_shape* shape, const ut_window* window, const void* q, const void* k,
                             const void* v, const int32_t* cu_q, const int32_t* cu_k, const int32_t* k_len,
                             const uint8_t* key_mask, float softmax_scale, const void* o, const float* lse,
                             const void* dout, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                             int32_t* dev_status, void* stream) {
  WinParams w;
  ut_status st = window_problem(shape, window, true, &w);
  if (st != UT_OK) return st;
  XattnParams& p = w.x;
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
  w.k_len = k_len;
  p.mask = key_mask;
  p.scale = softmax_scale;
  p.status = dev_status;
  p.timeout_ns = wait_timeout_ns();
  st = xattn_pointers(shape, p);
  if (st != UT_OK) return st;
  if ((p.nq > 0 && (!dout || !dq)) || (p.nk > 0 && (!dk || !dv))) return UT_ERR_INVALID_ARG;
  if (!at16(dout) || !at16(dq) || !at16(dk) || !at16(dv) || !at4(k_len)) return UT_ERR_INVALID_ARG;
  if (p.nq == 0 && p.nk == 0) return UT_OK;
  const bool bf16 = shape->dtype == UT_BF16;
  const size_t need = window_bwd_ws(w, bf16);
  if (need > 0 && (!ws || ws_bytes < need || !at16(ws))) return UT_ERR_INVALID_ARG;
  char* at = static_cast<char*>(ws);
  p.dsum = reinterpret_cast<float*>(at);
  at += up256((size_t)p.H * p.nq * sizeof(float));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (bf16) return status_of(launch_wattn_bwd_tc(w, at, s));
  p.part_dk = reinterpret_cast<float*>(at);
  p.part_dv = reinterpret_cast<float*>(at + up256(wattn_simt_part_rows(w) * p.Hk * p.d * sizeof(float)));
  return status_of(launch_wattn_bwd_simt(w, s));
}

}  // extern "C"
