// Windowed attention with visible first keys on the CUDA cores, in fp32
// arithmetic.  Per segment, query head h and its kv head h' = h / G, over the
// keys j that query i sees (wattn.cuh) and whose mask is set:
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
//   D_i = dO_i . O_i,  P = exp(S - LSE),  dS = P o (dO V^T - D)
//   dQ = scale dS K,  dK = scale sum dS^T Q,  dV = sum P^T dO
//
// Tiles of 64 rows (the G heads of a kv head of 64 / G tokens) and 64 keys, as
// cross attention has them (xattn_simt.cuh).  A query tile goes over the blocks
// of its two key ranges, a key tile over the query tiles that see some of its
// keys, so work grows with rows times window.  Rows and keys that do not exist,
// and masked keys, are staged as zeros and never enter a product; inside a
// block a row's own limits are applied to its scores.
// Bound by latency of the staged rows and of the shared-memory reads, two
// blocks an SM.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "wattn.cuh"
#include "xattn_simt.cuh"

namespace ut {

namespace {

// Which keys of a block a thread's four rows see.
struct Limits {
  int pos[4];  // positions of the rows' tokens
  int left, right, sinks;
  UT_DEV Limits(const WinParams& w, int p0, int G) : left(w.left), right(w.right), sinks(w.sinks) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pos[i] = p0 + ((threadIdx.x >> 4) * 4 + i) / G;
  }
  UT_DEV bool sees(int i, int key) const {
    return key <= pos[i] + right && (key >= pos[i] - left || key < sinks);
  }
};

UT_DEV void check_lens(const WinParams& w) {
  check_cu(w.x.cu_q, w.x.B, w.x.nq, w.x.status);
  check_cu(w.x.cu_k, w.x.B, w.x.nk, w.x.status);
  check_lens_of(w.x, w.k_len);
}

// grid (q slots, kv heads, key splits)
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads) wattn_fwd_simt_kernel(const WinParams w) {
  const XattnParams& p = w.x;
  extern __shared__ float sm[];
  float* qs = sm;
  float* ks = qs + kXs * (D + 4);
  float* vs = ks + kXs * (D + 4);
  float* ps = vs + kXs * (D + 4);
  float* on = ps + kXs * kXsLdP;
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) check_lens(w);
  const int tpt = kXs / p.G;
  const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, tpt, blockIdx.x);
  if (g.tile * tpt >= g.n) return;
  const int hk = blockIdx.y, split = blockIdx.z, t0 = (int)g.tile * tpt, ntok = (int)min((int64_t)tpt, g.n - t0);
  XsTile t{g.row + t0, ntok * p.G, hk * p.G, p.G};
  int64_t k0, kn;
  win_keys(w, g.s, k0, kn);
  const int p0 = (int)(kn - g.n) + t0;
  const Limits lim(w, p0, p.G);
  const WinRange rg = win_range(p0, p0 + ntok - 1, (int)kn, w.left, w.right, w.sinks);
  const int nblk = win_blocks<kXs>(rg), per = (nblk + p.nsplit - 1) / p.nsplit;
  const int b0 = min(nblk, per * split), b1 = min(nblk, b0 + per);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  stage_q<T, D>(qs, p.q, t, p.qs);
  float m[4], l[4];
  float4 o[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) o[i][c] = make_float4(0, 0, 0, 0);
  }
  for (int b = b0; b < b1; ++b) {
    int x, e;
    win_block<kXs>(rg, b, x, e);
    __syncthreads();
    if (!stage_mask(on, p.mask, k0 + x, e - x)) continue;  // no key of the tile is left
    stage_k<T, D>(ks, p.k, k0 + x, on, hk, p.ks);
    stage_k<T, D>(vs, p.v, k0 + x, on, hk, p.vs);
    __syncthreads();
    float s[4][4];
    product_nt<D>(qs, ks, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = on[tx + 16 * j] != 0.f && lim.sees(i, x + tx + 16 * j) ? s[i][j] * p.scale : -INFINITY;
        mx = fmaxf(mx, s[i][j]);
      }
      mx = fmaxf(m[i], half_warp_max(mx));
      const float ref = mx == -INFINITY ? 0.f : mx;  // a row that saw no key yet
      const float alpha = expf(m[i] - ref);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float y = expf(s[i][j] - ref);
        sum += y;
        ps[(ty * 4 + i) * kXsLdP + tx + 16 * j] = y;
      }
      l[i] = l[i] * alpha + half_warp_sum(sum);
      m[i] = mx;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        o[i][c].x *= alpha;
        o[i][c].y *= alpha;
        o[i][c].z *= alpha;
        o[i][c].w *= alpha;
      }
    }
    __syncthreads();
    product_nn<D>(ps, vs, o);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i;
    if (r >= t.rows) continue;
    const int64_t tok = t.tok0 + r / p.G;
    const int h = t.head0 + r % p.G;
    if (p.nsplit == 1) {
      const float inv = l[i] > 0.f ? 1.f / l[i] : (l[i] == 0.f ? 0.f : l[i]);
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        st4(static_cast<T*>(p.o) + t.off(r, p.os, D) + tx * 4 + 64 * c,
            make_float4(o[i][c].x * inv, o[i][c].y * inv, o[i][c].z * inv, o[i][c].w * inv));
      if (tx == 0) p.lse[(int64_t)h * p.nq + tok] = m[i] + logf(l[i]);
    } else {
      const int64_t row = ((int64_t)split * p.nq + tok) * p.H + h;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) st4(p.part_o + row * D + tx * 4 + 64 * c, o[i][c]);
      if (tx == 0) p.part_ml[row] = make_float2(m[i] * kLog2e, l[i]);
    }
  }
}

// P and dS of one 64 x 64 pair of tiles; s, dp are its products
UT_DEV void probabilities(const XattnParams& p, const Limits& lim, int x, const float* on, const float* lse,
                          const float* dsum, float (&s)[4][4], float (&dp)[4][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float le = lse[ty * 4 + i], ds = dsum[ty * 4 + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool is = on[tx + 16 * j] != 0.f && le != -INFINITY && lim.sees(i, x + tx + 16 * j);
      s[i][j] = is ? expf(s[i][j] * p.scale - le) : 0.f;
      dp[i][j] = is ? s[i][j] * (dp[i][j] - ds) : 0.f;
    }
  }
}

// dQ of a query tile over its keys
template <typename T, int D>
UT_DEV void dq_tile(const WinParams& w, float* sm, int64_t slot, int hk) {
  const XattnParams& p = w.x;
  float* qs = sm;
  float* dos = qs + kXs * (D + 4);
  float* ks = dos + kXs * (D + 4);
  float* vs = ks + kXs * (D + 4);
  float* dss = vs + kXs * (D + 4);
  float* on = dss + kXs * kXsLdP;
  float* lse = on + kXs;
  float* dsum = lse + kXs;
  const int tpt = kXs / p.G;
  const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, tpt, slot);
  if (g.tile * tpt >= g.n) return;
  const int t0 = (int)g.tile * tpt, ntok = (int)min((int64_t)tpt, g.n - t0);
  XsTile t{g.row + t0, ntok * p.G, hk * p.G, p.G};
  int64_t k0, kn;
  win_keys(w, g.s, k0, kn);
  const int p0 = (int)(kn - g.n) + t0;
  const Limits lim(w, p0, p.G);
  const WinRange rg = win_range(p0, p0 + ntok - 1, (int)kn, w.left, w.right, w.sinks);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  stage_q<T, D>(qs, p.q, t, p.qs);
  stage_q<T, D>(dos, p.dout, t, p.dos);
  stage_rows(lse, dsum, p, t);
  float4 acc[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) acc[i][c] = make_float4(0, 0, 0, 0);
  for (int b = 0; b < win_blocks<kXs>(rg); ++b) {
    int x, e;
    win_block<kXs>(rg, b, x, e);
    __syncthreads();
    if (!stage_mask(on, p.mask, k0 + x, e - x)) continue;  // no key of the tile is left
    stage_k<T, D>(ks, p.k, k0 + x, on, hk, p.ks);
    stage_k<T, D>(vs, p.v, k0 + x, on, hk, p.vs);
    __syncthreads();
    float s[4][4], dp[4][4];
    product_nt<D>(qs, ks, s);
    product_nt<D>(dos, vs, dp);
    probabilities(p, lim, x, on, lse, dsum, s, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) dss[(ty * 4 + i) * kXsLdP + tx + 16 * j] = dp[i][j];
    __syncthreads();
    product_nn<D>(dss, ks, acc);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i;
    if (r >= t.rows) continue;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
      st4(static_cast<T*>(p.dq) + t.off(r, p.dqs, D) + tx * 4 + 64 * c,
          make_float4(acc[i][c].x * p.scale, acc[i][c].y * p.scale, acc[i][c].z * p.scale, acc[i][c].w * p.scale));
  }
}

// Partial dK, dV of a key tile over a part of the query tiles that see it
template <typename T, int D>
UT_DEV void dkdv_tile(const WinParams& w, float* sm, int64_t slot, int hk, int split) {
  const XattnParams& p = w.x;
  float* qs = sm;
  float* dos = qs + kXs * (D + 4);
  float* ks = dos + kXs * (D + 4);
  float* vs = ks + kXs * (D + 4);
  float* ps = vs + kXs * (D + 4);
  float* dss = ps + kXs * kXsLdP;
  float* on = dss + kXs * kXsLdP;
  float* lse = on + kXs;
  float* dsum = lse + kXs;
  const Segment g = segment_of_slot(p.cu_k, p.B, p.nk, kXs, slot);
  if (g.tile * kXs >= g.n) return;
  int64_t q0, qn, k0, kn;
  segment_rows(p.cu_q, g.s, p.nq, q0, qn);
  win_keys(w, g.s, k0, kn);
  const int x0 = (int)g.tile * kXs, rows = (int)min((int64_t)kXs, g.n - x0);  // rows of dK, dV; keys may be fewer
  const int tpt = kXs / p.G;
  int a = 0, b = 0;  // tokens, then tiles
  if (x0 < kn) win_tokens(x0, min(x0 + kXs, (int)kn), (int)kn, (int)qn, w.left, w.right, w.sinks, a, b);
  b = (b + tpt - 1) / tpt;
  a = min(a / tpt, b);
  const int per = (b - a + p.nsplit - 1) / p.nsplit, first = min(b, a + per * split), last = min(b, first + per);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const bool any = stage_mask(on, p.mask, k0 + x0, kn - x0);
  stage_k<T, D>(ks, p.k, k0 + x0, on, hk, p.ks);
  stage_k<T, D>(vs, p.v, k0 + x0, on, hk, p.vs);
  float4 dk[4][D / 64], dv[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) dk[i][c] = dv[i][c] = make_float4(0, 0, 0, 0);
  for (int tt = first; any && tt < last; ++tt) {
    XsTile t{q0 + tt * tpt, (int)min((int64_t)tpt, qn - tt * tpt) * p.G, hk * p.G, p.G};
    const Limits lim(w, (int)(kn - qn) + tt * tpt, p.G);
    __syncthreads();
    stage_q<T, D>(qs, p.q, t, p.qs);
    stage_q<T, D>(dos, p.dout, t, p.dos);
    stage_rows(lse, dsum, p, t);
    __syncthreads();
    float s[4][4], dp[4][4];
    product_nt<D>(qs, ks, s);
    product_nt<D>(dos, vs, dp);
    probabilities(p, lim, x0, on, lse, dsum, s, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ps[(ty * 4 + i) * kXsLdP + tx + 16 * j] = s[i][j];
        dss[(ty * 4 + i) * kXsLdP + tx + 16 * j] = dp[i][j];
      }
    __syncthreads();
    product_tn<D>(ps, dos, dv);
    product_tn<D>(dss, qs, dk);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i;
    if (r >= rows) continue;
    const int64_t row = ((int64_t)split * p.nk + k0 + x0 + r) * p.Hk + hk;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      st4(p.part_dk + row * D + tx * 4 + 64 * c, dk[i][c]);
      st4(p.part_dv + row * D + tx * 4 + 64 * c, dv[i][c]);
    }
  }
}

// One launch for both: n_kv blocks of dK, dV (k slots fastest, then kv heads,
// splits), then dQ (q slots, kv heads).
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads) wattn_bwd_simt_kernel(const WinParams w, uint32_t n_kv, uint32_t kslots,
                                                                    uint32_t qslots) {
  extern __shared__ float sm[];
  grid_wait();
  const uint32_t x = blockIdx.x;
  if (x == 0) check_lens_of(w.x, w.k_len);
  if (x < n_kv) {
    const uint32_t y = x / kslots;
    dkdv_tile<T, D>(w, sm, x - y * kslots, (int)(y % w.x.Hk), (int)(y / w.x.Hk));
  } else {
    const uint32_t y = (x - n_kv) / qslots;
    dq_tile<T, D>(w, sm, x - n_kv - y * qslots, (int)y);
  }
}

template <typename T, int D>
cudaError_t fwd(const WinParams& w, cudaStream_t s) {
  const XattnParams& p = w.x;
  const size_t smem = sizeof(float) * (3 * kXs * (D + 4) + kXs * kXsLdP + kXs);
  cudaError_t e = cudaFuncSetAttribute(wattn_fwd_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  wattn_fwd_simt_kernel<T, D>
      <<<dim3((unsigned)segment_slots(p.nq, p.B, kXs / p.G), p.Hk, p.nsplit), kXsThreads, smem, s>>>(w);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t bwd(const WinParams& w, cudaStream_t s) {
  const XattnParams& p = w.x;
  cudaError_t e = launch_xattn_dsum(p, sizeof(T) == 2, s);
  if (e != cudaSuccess) return e;
  const size_t smem = sizeof(float) * (4 * kXs * (D + 4) + 2 * kXs * kXsLdP + 3 * kXs);
  const uint32_t kslots = (uint32_t)segment_slots(p.nk, p.B, kXs), qslots = (uint32_t)segment_slots(p.nq, p.B, kXs / p.G);
  const int64_t n_kv = p.nk > 0 ? (int64_t)kslots * p.Hk * p.nsplit : 0, n_q = p.nq > 0 ? (int64_t)qslots * p.Hk : 0;
  if (n_kv + n_q > INT32_MAX) return cudaErrorInvalidValue;
  e = cudaFuncSetAttribute(wattn_bwd_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess)
    e = launch_next(wattn_bwd_simt_kernel<T, D>, dim3((unsigned)(n_kv + n_q)), dim3(kXsThreads), smem, s, w,
                    (uint32_t)n_kv, kslots, qslots);
  if (e == cudaSuccess && p.nk > 0) e = launch_xattn_dkdv_join(p, s);
  return e;
}

}  // namespace

int64_t wattn_simt_items(const WinParams& w, bool backward) {
  const XattnParams& p = w.x;
  return (backward ? segment_slots(p.nk, p.B, kXs) : segment_slots(p.nq, p.B, kXs / p.G)) * p.Hk;
}

// Enough parts for two blocks an SM (four backward), none shorter than two
// blocks of a mean segment (one tile backward).  Of the keys a tile sees, and
// of the tiles that see a key tile: all of a segment's for the first keys.
int wattn_simt_splits(const WinParams& w, bool backward) {
  const XattnParams& p = w.x;
  const int64_t tpt = kXs / p.G, items = wattn_simt_items(w, backward);
  const int64_t want = ((backward ? 4 : 2) * (int64_t)p.sms + items - 1) / items;
  const int64_t near = (int64_t)w.left + w.right + (backward ? kXs : w.sinks + tpt), rows = (backward ? p.nq : p.nk) / p.B;
  const int64_t seen = near < rows && !(backward && w.sinks > 0) ? near : rows;
  const int64_t most = backward ? (seen + tpt - 1) / tpt : (seen + kXs - 1) / kXs / 2;
  const int64_t n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

cudaError_t launch_wattn_fwd_simt(const WinParams& w, cudaStream_t s) {
  return w.x.d == 64 ? fwd<float, 64>(w, s) : fwd<float, 128>(w, s);
}
cudaError_t launch_wattn_bwd_simt(const WinParams& w, cudaStream_t s) {
  return w.x.d == 64 ? bwd<float, 64>(w, s) : bwd<float, 128>(w, s);
}

}  // namespace ut
