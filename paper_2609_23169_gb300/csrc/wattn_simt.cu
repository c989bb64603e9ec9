// Windowed attention with visible first keys on the CUDA cores, in fp32
// arithmetic.  Per segment, query head h and its kv head h' = h / G, over the
// keys j that query i sees (wattn.cuh) and whose mask is set:
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
//   D_i = dO_i . O_i,  P = exp(S - LSE),  dS = P o (dO V^T - D)
//   dQ = scale dS K,  dK = scale sum dS^T Q,  dV = sum P^T dO
//
// Tiles of 64 rows (the G heads of a kv head of 64 / G tokens) and 64 keys, as
// cross attention has them (xattn_simt.cuh).  A query tile goes over the keys of
// its two ranges one after the other, 64 at a time (a block may hold first keys
// and window keys), a key tile over the query tiles that see some of its keys,
// so work grows with rows times window.  Rows and keys that do not exist, and
// masked keys, are staged as zeros and never enter a product; inside a block a
// row's own limits are applied to its scores.  A key tile that many tokens see
// (first keys) is split over them and joined.
// Bound by latency of the staged rows and of the shared-memory reads: 2,501 rows
// in 3 segments, 8 / 4 heads of 64, 100 keys before, 28 behind, 7 first ones,
// masked: forward 50 us, D 6, gradient 142 (44% of the issue slots), join 15;
// 8,000 rows, 500 before, 8 heads of 64: 29 TFLOP/s forward, the shared-memory
// path 70% busy.  (Eight rows a thread read a quarter less from it, but leave half
// the warps: 291 -> 303 us at that step.)
#include <math.h>

#include <algorithm>

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

// Parts that the `tiles` query tiles of a key tile are split into
UT_DEV int parts_of(const WinParams& w, int tiles, int most) { return max(1, min(most, (tiles + w.run - 1) / w.run)); }

// Key i of a tile's two ranges (of the segment), and how many there are
UT_DEV int key_of(const WinRange& r, int i) { return i < r.first ? i : i + (r.lo - r.first); }
UT_DEV int keys_of(const WinRange& r) { return r.first + r.hi - r.lo; }

// on[64] <- 1 where key i0 + r exists and is not masked; whether any is.  Synchronises the block.
UT_DEV bool stage_window_mask(float* on, const WinRange& rg, const uint8_t* mask, int64_t k0, int i0) {
  const int r = threadIdx.x;
  const bool is = r < kXs && i0 + r < keys_of(rg) && (!mask || mask[k0 + key_of(rg, i0 + r)]);
  if (r < kXs) on[r] = is ? 1.f : 0.f;
  return __syncthreads_or(is);
}
// ks, vs [64][D + 4] <- keys i0 .. of kv head hk (zeros where `on` is 0)
template <typename T, int D>
UT_DEV void stage_window(float* ks, float* vs, const XattnParams& p, const WinRange& rg, int64_t k0, int i0, const float* on,
                         int hk) {
#pragma unroll 2
  for (int e = threadIdx.x; e < kXs * (D / 4); e += kXsThreads) {
    const int r = e / (D / 4), c = (e % (D / 4)) * 4;
    float4 k = make_float4(0, 0, 0, 0), v = k;
    if (on[r] != 0.f) {
      const int64_t row = k0 + key_of(rg, i0 + r);
      k = ld4(static_cast<const T*>(p.k) + row * p.ks + (int64_t)hk * D + c);
      v = ld4(static_cast<const T*>(p.v) + row * p.vs + (int64_t)hk * D + c);
    }
    st4(ks + r * (D + 4) + c, k);
    st4(vs + r * (D + 4) + c, v);
  }
}

UT_DEV void check_lens(const WinParams& w) {
  check_cu(w.x.cu_q, w.x.B, w.x.nq, w.x.status);
  check_cu(w.x.cu_k, w.x.B, w.x.nk, w.x.status);
  check_lens_of(w.x, w.k_len);
}

// grid (q slots, kv heads, key splits)
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads, D == 64 ? 2 : 1) wattn_fwd_simt_kernel(const WinParams w) {
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
  const int nblk = (keys_of(rg) + kXs - 1) / kXs, per = (nblk + p.nsplit - 1) / p.nsplit;
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
    __syncthreads();
    if (!stage_window_mask(on, rg, p.mask, k0, b * kXs)) continue;  // no key of the tile is left
    stage_window<T, D>(ks, vs, p, rg, k0, b * kXs, on, hk);
    __syncthreads();
    int key[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) key[j] = key_of(rg, b * kXs + tx + 16 * j);
    float s[4][4];
    product_nt<D>(qs, ks, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = on[tx + 16 * j] != 0.f && lim.sees(i, key[j]) ? s[i][j] * p.scale : -INFINITY;
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
UT_DEV void probabilities(const XattnParams& p, const Limits& lim, const int (&key)[4], const float* on, const float* lse,
                          const float* dsum, float (&s)[4][4], float (&dp)[4][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float le = lse[ty * 4 + i], ds = dsum[ty * 4 + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool is = on[tx + 16 * j] != 0.f && le != -INFINITY && lim.sees(i, key[j]);
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
  for (int i0 = 0; i0 < keys_of(rg); i0 += kXs) {
    __syncthreads();
    if (!stage_window_mask(on, rg, p.mask, k0, i0)) continue;  // no key of the tile is left
    stage_window<T, D>(ks, vs, p, rg, k0, i0, on, hk);
    __syncthreads();
    int key[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) key[j] = key_of(rg, i0 + tx + 16 * j);
    float s[4][4], dp[4][4];
    product_nt<D>(qs, ks, s);
    product_nt<D>(dos, vs, dp);
    probabilities(p, lim, key, on, lse, dsum, s, dp);
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

// The query tiles [a, b) that see keys of key tile x0 of a segment of n_k keys and n_q queries
UT_DEV void tiles_of(const WinParams& w, int x0, int n_k, int n_q, int& a, int& b) {
  const int tpt = kXs / w.x.G;
  a = b = 0;
  if (x0 < n_k) win_tokens(x0, min(x0 + kXs, n_k), n_k, n_q, w.left, w.right, w.sinks, a, b);
  b = (b + tpt - 1) / tpt;
  a = min(a / tpt, b);
}

// Row r of part i of a key tile: [parts, nk, Hk, d], and behind them those of the
// tiles with first keys where they have more parts, [B, sb, first_parts, 64, Hk, d]
struct KeyParts {
  int parts;       // of this key tile
  int64_t at, step;  // its row 0 of part 0, rows from part to part
};
UT_DEV KeyParts key_parts(const WinParams& w, const Segment& g, int64_t k0, int tiles) {
  const int64_t x0 = g.tile * kXs;
  const bool first = x0 < w.sinks && w.first_parts > w.parts;
  KeyParts k;
  k.parts = parts_of(w, tiles, first ? w.first_parts : w.parts);
  k.step = first ? kXs : w.x.nk;
  k.at = first ? w.parts * w.x.nk + ((int64_t)g.s * w.sb + g.tile) * w.first_parts * kXs : k0 + x0;
  return k;
}

// Partial dK, dV of a key tile over a part of the query tiles that see it
template <typename T, int D>
UT_DEV void dkdv_tile(const WinParams& w, float* sm, const Segment& g, int hk, int split) {
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
  if (g.tile * kXs >= g.n) return;
  int64_t q0, qn, k0, kn;
  segment_rows(p.cu_q, g.s, p.nq, q0, qn);
  win_keys(w, g.s, k0, kn);
  const int x0 = (int)g.tile * kXs, rows = (int)min((int64_t)kXs, g.n - x0);  // rows of dK, dV; keys may be fewer
  const int tpt = kXs / p.G;
  int a, b;
  tiles_of(w, x0, (int)kn, (int)qn, a, b);
  const KeyParts kp = key_parts(w, g, k0, b - a);
  if (split >= kp.parts) return;
  const int per = (b - a + kp.parts - 1) / kp.parts, first = min(b, a + per * split), last = min(b, first + per);
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
    const int key[4] = {x0 + tx, x0 + tx + 16, x0 + tx + 32, x0 + tx + 48};
    probabilities(p, lim, key, on, lse, dsum, s, dp);
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
    const int64_t row = (kp.at + split * kp.step + r) * p.Hk + hk;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      st4(p.part_dk + row * D + tx * 4 + 64 * c, dk[i][c]);
      st4(p.part_dv + row * D + tx * 4 + 64 * c, dv[i][c]);
    }
  }
}

// dK (blockIdx.z = 0), dV = the sum of the parts, in their order; a block a key
// tile and kv head
template <int D>
__global__ void __launch_bounds__(kXsThreads) wattn_join_simt_kernel(const WinParams w) {
  const XattnParams& p = w.x;
  grid_wait();
  const Segment g = segment_of_slot(p.cu_k, p.B, p.nk, kXs, blockIdx.x);
  if (g.tile * kXs >= g.n) return;
  int64_t q0, qn, k0, kn;
  segment_rows(p.cu_q, g.s, p.nq, q0, qn);
  win_keys(w, g.s, k0, kn);
  const int x0 = (int)g.tile * kXs, rows = (int)min((int64_t)kXs, g.n - x0), hk = blockIdx.y;
  int a, b;
  tiles_of(w, x0, (int)kn, (int)qn, a, b);
  const KeyParts kp = key_parts(w, g, k0, b - a);
  const bool is_v = blockIdx.z;
  const float* part = is_v ? p.part_dv : p.part_dk;
  const float f = is_v ? 1.f : p.scale;
  for (int e = threadIdx.x; e < rows * (D / 4); e += kXsThreads) {
    const int r = e / (D / 4), c = (e % (D / 4)) * 4;
    const int64_t key = k0 + x0 + r;
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int i = 0; i < kp.parts; ++i) {
      const float4 v = ld4(part + ((kp.at + i * kp.step + r) * p.Hk + hk) * D + c);
      sum.x += v.x;
      sum.y += v.y;
      sum.z += v.z;
      sum.w += v.w;
    }
    // a masked key's row is zero, and one behind the keys, also where a NaN or an
    // infinity of Q or dO met its P and dS of 0
    if (x0 + r >= kn || (p.mask && !p.mask[key])) sum = make_float4(0, 0, 0, 0);
    st4(static_cast<float*>(is_v ? p.dv : p.dk) + key * (is_v ? p.dvs : p.dks) + (int64_t)hk * D + c,
        make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f));
  }
}

// One launch for both: n_kv blocks of dK, dV (k slots fastest, then kv heads,
// parts; behind n_all those of the tiles with first keys that have more parts:
// their tiles fastest, then segments, kv heads, parts), then dQ (q slots, kv heads).
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads, D == 64 ? 2 : 1) wattn_bwd_simt_kernel(const WinParams w, uint32_t n_all, uint32_t n_kv,
                                                                    uint32_t kslots, uint32_t qslots) {
  extern __shared__ float sm[];
  grid_wait();
  const uint32_t x = blockIdx.x;
  if (x == 0) check_lens_of(w.x, w.k_len);
  if (x < n_kv) {
    const bool more = x >= n_all;
    const uint32_t i = more ? x - n_all : x, tiles = more ? (uint32_t)w.sb * w.x.B : kslots, y = i / tiles, z = i - y * tiles;
    Segment g;
    if (more) {
      g.s = (int)(z / w.sb);
      g.tile = z - g.s * w.sb;
      segment_rows(w.x.cu_k, g.s, w.x.nk, g.row, g.n);
    } else {
      g = segment_of_slot(w.x.cu_k, w.x.B, w.x.nk, kXs, z);
    }
    dkdv_tile<T, D>(w, sm, g, (int)(y % w.x.Hk), (int)(y / w.x.Hk) + (more ? w.parts : 0));
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
  const int64_t n_all = p.nk > 0 ? (int64_t)kslots * p.Hk * w.parts : 0;
  const int64_t n_kv = n_all + (p.nk > 0 && w.first_parts > w.parts ? (int64_t)w.sb * p.B * p.Hk * (w.first_parts - w.parts) : 0);
  const int64_t n_q = p.nq > 0 ? (int64_t)qslots * p.Hk : 0;
  if (n_kv + n_q > INT32_MAX) return cudaErrorInvalidValue;
  e = cudaFuncSetAttribute(wattn_bwd_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess)
    e = launch_next(wattn_bwd_simt_kernel<T, D>, dim3((unsigned)(n_kv + n_q)), dim3(kXsThreads), smem, s, w,
                    (uint32_t)n_all, (uint32_t)n_kv, kslots, qslots);
  if (e == cudaSuccess && p.nk > 0)
    e = launch_next(wattn_join_simt_kernel<D>, dim3(kslots, p.Hk, 2), dim3(kXsThreads), 0, s, w);
  return e;
}

}  // namespace

int64_t wattn_simt_items(const WinParams& w, bool backward) {
  const XattnParams& p = w.x;
  return (backward ? segment_slots(p.nk, p.B, kXs) : segment_slots(p.nq, p.B, kXs / p.G)) * p.Hk;
}

// Enough parts of the keys for two blocks an SM, none shorter than two blocks of
// n_k / n_seg rows (of caches their capacity), as far as a tile sees them.
int wattn_simt_splits(const WinParams& w) {
  const XattnParams& p = w.x;
  const int64_t tpt = kXs / p.G, rows = p.nk / p.B, near = (int64_t)w.left + w.right + w.sinks + tpt;
  const int64_t want = (2 * (int64_t)p.sms + wattn_simt_items(w, false) - 1) / wattn_simt_items(w, false);
  const int64_t most = ((near < rows ? near : rows) + kXs - 1) / kXs / 2, n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

// The most parts of a key tile, of `run` query tiles at least: of those that a
// window's tokens see, and of those with first keys, which all later tokens see
// (unless there are many of these).  A run has six tiles, or fewer, two at least,
// where the pairs of tiles do not make two such blocks for each that an SM holds
// (800 rows of 4 heads of 64: 76 us in runs of six, 50 in runs of two; 8,000 rows of
// 8: 895 and 977).
void wattn_simt_parts(WinParams& w) {
  const XattnParams& p = w.x;
  const int64_t tpt = kXs / p.G, all = (p.nq + tpt - 1) / tpt, seen = (int64_t)w.left + w.right + kXs;
  const int64_t near = seen < p.nq ? (seen + 2 * tpt - 2) / tpt : all;
  const int64_t span = (int64_t)w.left + w.right + tpt, blocks = ((span < p.nk ? span : p.nk) + kXs - 1) / kXs;
  const int64_t pairs = segment_slots(p.nk, p.B, kXs) * p.Hk * near + segment_slots(p.nq, p.B, (int)tpt) * p.Hk * blocks;
  w.run = (int)std::min<int64_t>(6, std::max<int64_t>(2, pairs / ((p.d == 64 ? 4 : 2) * (int64_t)p.sms)));
  auto parts = [&](int64_t tiles) { return (int)std::min<int64_t>(16, std::max<int64_t>(1, (tiles + w.run - 1) / w.run)); };
  const bool enough = segment_slots(p.nk, p.B, kXs) * p.Hk >= 8 * (int64_t)p.sms;
  w.parts = enough ? 1 : parts(near);
  w.sb = (int)((std::min<int64_t>(w.sinks, p.nk) + kXs - 1) / kXs);
  w.first_parts = w.sb > 0 && (int64_t)w.sb * p.B * p.Hk < 2 * p.sms ? parts(all) : w.parts;
}
size_t wattn_simt_part_rows(const WinParams& w) {  // of Hk * d values, each of dK and dV
  return (size_t)w.parts * w.x.nk + (w.first_parts > w.parts ? (size_t)w.x.B * w.sb * w.first_parts * kXs : 0);
}

cudaError_t launch_wattn_fwd_simt(const WinParams& w, cudaStream_t s) {
  return w.x.d == 64 ? fwd<float, 64>(w, s) : fwd<float, 128>(w, s);
}
cudaError_t launch_wattn_bwd_simt(const WinParams& w, cudaStream_t s) {
  return w.x.d == 64 ? bwd<float, 64>(w, s) : bwd<float, 128>(w, s);
}

}  // namespace ut
