// Cross attention to an encoder's states on the CUDA cores, in fp32 arithmetic.
//
// Per segment s, query head h and its kv head h' = h / G (G = H / H_kv):
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
//   D_i = dO_i . O_i,  P = exp(S - LSE),  dS = P o (dO V^T - D)
//   dQ = scale dS K,  dK = scale sum dS^T Q,  dV = sum P^T dO
// over the segment's keys whose mask is set.
//
// A tile holds 64 rows: the G heads that share a kv head of 64 / G
// consecutive tokens (row = token * G + head), so that K and V are read once
// for the group and dK, dV sum over its heads inside the tile products.  256
// threads as 16 x 16; a thread computes 4 x 4 of a 64 x 64 product (4 rows,
// columns tx + 16 j) and 4 x D/16 of a 64 x D product; all operands are
// row-major in shared memory with 4 floats of padding (16-byte reads without
// bank conflicts), the multiply-adds on pairs.  Rows and keys that do not exist
// or are masked are staged as zeros, so that whatever their memory holds never
// enters a product.
//
// Two blocks share an SM; bound by latency, of the staged rows and of the reads
// from shared memory (an instruction in 55% of the cycles, a multiply-add in
// half of them): 2,501 x 301, 8 / 4 heads of 64, forward 28 us, gradient 80.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "pairs.cuh"
#include "segments.cuh"
#include "xattn.cuh"
#include "xattn_simt.cuh"

namespace ut {

// grid (q slots, kv heads, key splits)
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads) xattn_fwd_simt_kernel(const XattnParams p) {
  extern __shared__ float sm[];
  float* qs = sm;
  float* ks = qs + kXs * (D + 4);
  float* vs = ks + kXs * (D + 4);
  float* ps = vs + kXs * (D + 4);
  float* on = ps + kXs * kXsLdP;
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) {
    check_cu(p.cu_q, p.B, p.nq, p.status);
    check_cu(p.cu_k, p.B, p.nk, p.status);
  }
  const int tpt = kXs / p.G;
  const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, tpt, blockIdx.x);
  if (g.tile * tpt >= g.n) return;
  const int hk = blockIdx.y, split = blockIdx.z;
  XsTile t{g.row + g.tile * tpt, (int)min((int64_t)tpt, g.n - g.tile * tpt) * p.G, hk * p.G, p.G};
  int64_t k0, kn;
  segment_rows(p.cu_k, g.s, p.nk, k0, kn);
  const int64_t nblk = (kn + kXs - 1) / kXs, per = (nblk + p.nsplit - 1) / p.nsplit;
  const int64_t b0 = per * split, b1 = min(nblk, b0 + per);
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
  for (int64_t b = b0; b < b1; ++b) {
    __syncthreads();
    if (!stage_mask(on, p.mask, k0 + b * kXs, kn - b * kXs)) continue;  // no key of the tile is left
    stage_k<T, D>(ks, p.k, k0 + b * kXs, on, hk, p.ks);
    stage_k<T, D>(vs, p.v, k0 + b * kXs, on, hk, p.vs);
    __syncthreads();
    float s[4][4];
    product_nt<D>(qs, ks, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = on[tx + 16 * j] != 0.f ? s[i][j] * p.scale : -INFINITY;
        mx = fmaxf(mx, s[i][j]);
      }
      mx = fmaxf(m[i], half_warp_max(mx));
      const float ref = mx == -INFINITY ? 0.f : mx;  // a row that saw no key yet
      const float alpha = expf(m[i] - ref);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = expf(s[i][j] - ref);
        sum += e;
        ps[(ty * 4 + i) * kXsLdP + tx + 16 * j] = e;
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
UT_DEV void probabilities(const XattnParams& p, const float* on, const float* lse, const float* dsum, float (&s)[4][4],
                          float (&dp)[4][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float le = lse[ty * 4 + i], ds = dsum[ty * 4 + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[i][j] = on[tx + 16 * j] != 0.f && le != -INFINITY ? expf(s[i][j] * p.scale - le) : 0.f;
      dp[i][j] = s[i][j] * (dp[i][j] - ds);
    }
  }
}

// dQ of a query tile over the segment's keys
template <typename T, int D>
UT_DEV void dq_tile(const XattnParams& p, float* sm, int64_t slot, int hk) {
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
  XsTile t{g.row + g.tile * tpt, (int)min((int64_t)tpt, g.n - g.tile * tpt) * p.G, hk * p.G, p.G};
  int64_t k0, kn;
  segment_rows(p.cu_k, g.s, p.nk, k0, kn);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  stage_q<T, D>(qs, p.q, t, p.qs);
  stage_q<T, D>(dos, p.dout, t, p.dos);
  stage_rows(lse, dsum, p, t);
  float4 acc[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) acc[i][c] = make_float4(0, 0, 0, 0);
  for (int64_t b = 0; b * kXs < kn; ++b) {
    __syncthreads();
    if (!stage_mask(on, p.mask, k0 + b * kXs, kn - b * kXs)) continue;  // no key of the tile is left
    stage_k<T, D>(ks, p.k, k0 + b * kXs, on, hk, p.ks);
    stage_k<T, D>(vs, p.v, k0 + b * kXs, on, hk, p.vs);
    __syncthreads();
    float s[4][4], dp[4][4];
    product_nt<D>(qs, ks, s);
    product_nt<D>(dos, vs, dp);
    probabilities(p, on, lse, dsum, s, dp);
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

// Partial dK, dV of a key tile over a range of the segment's query tiles
template <typename T, int D>
UT_DEV void dkdv_tile(const XattnParams& p, float* sm, int64_t slot, int hk, int split) {
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
  const int64_t key0 = g.row + g.tile * kXs, left = g.n - g.tile * kXs;
  int64_t q0, qn;
  segment_rows(p.cu_q, g.s, p.nq, q0, qn);
  const int tpt = kXs / p.G;
  const int64_t nt = (qn + tpt - 1) / tpt, per = (nt + p.nsplit - 1) / p.nsplit;
  const int64_t t0 = per * split, t1 = min(nt, t0 + per);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const bool any = stage_mask(on, p.mask, key0, left);
  stage_k<T, D>(ks, p.k, key0, on, hk, p.ks);
  stage_k<T, D>(vs, p.v, key0, on, hk, p.vs);
  float4 dk[4][D / 64], dv[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) dk[i][c] = dv[i][c] = make_float4(0, 0, 0, 0);
  for (int64_t tt = t0; any && tt < t1; ++tt) {
    XsTile t{q0 + tt * tpt, (int)min((int64_t)tpt, qn - tt * tpt) * p.G, hk * p.G, p.G};
    __syncthreads();
    stage_q<T, D>(qs, p.q, t, p.qs);
    stage_q<T, D>(dos, p.dout, t, p.dos);
    stage_rows(lse, dsum, p, t);
    __syncthreads();
    float s[4][4], dp[4][4];
    product_nt<D>(qs, ks, s);
    product_nt<D>(dos, vs, dp);
    probabilities(p, on, lse, dsum, s, dp);
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
    if (r >= left) continue;
    const int64_t row = ((int64_t)split * p.nk + key0 + r) * p.Hk + hk;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      st4(p.part_dk + row * D + tx * 4 + 64 * c, dk[i][c]);
      st4(p.part_dv + row * D + tx * 4 + 64 * c, dv[i][c]);
    }
  }
}

// One launch for both, the longer blocks first: n_kv blocks of dK, dV (k slots
// fastest, then kv heads, query splits), then dQ (q slots, kv heads).  Apart,
// each ended in a wave of a few blocks (2,501 x 301, 8 heads: 38 + 66 us).
template <typename T, int D>
__global__ void __launch_bounds__(kXsThreads) xattn_bwd_simt_kernel(const XattnParams p, uint32_t n_kv,
                                                                     uint32_t kslots, uint32_t qslots) {
  extern __shared__ float sm[];
  grid_wait();
  const uint32_t x = blockIdx.x;
  if (x < n_kv) {
    const uint32_t y = x / kslots;
    dkdv_tile<T, D>(p, sm, x - y * kslots, (int)(y % p.Hk), (int)(y / p.Hk));
  } else {
    const uint32_t y = (x - n_kv) / qslots;
    dq_tile<T, D>(p, sm, x - n_kv - y * qslots, (int)y);
  }
}

// D_i = dO_i . O_i -> [H, nq]: 16 bytes of O and dO a thread and step, the
// threads of a row side by side, four steps in flight.  Also checks the
// prefixes.  Bound by memory: 44 us for 23,959 x 24 x 128 in bf16 (295 MB).
constexpr int kDsumSteps = 4;
template <typename T, int D>
__global__ void __launch_bounds__(256) xattn_dsum_kernel(const XattnParams p) {
  constexpr int kVals = 16 / sizeof(T), kLanes = D / kVals;  // values of a thread, threads of a row
  grid_next();
  if (blockIdx.x == 0) {
    check_cu(p.cu_q, p.B, p.nq, p.status);
    check_cu(p.cu_k, p.B, p.nk, p.status);
  }
  const uint32_t first = blockIdx.x * (256 / kLanes * kDsumSteps) + threadIdx.x / kLanes;  // row and head: 2^32 would be 512 GB
  const int e = (int)(threadIdx.x % kLanes) * kVals;
  uint4 a[kDsumSteps], b[kDsumSteps];
  uint32_t tok[kDsumSteps], h[kDsumSteps];
#pragma unroll
  for (int i = 0; i < kDsumSteps; ++i) {
    const uint32_t x = first + i * (256 / kLanes);
    tok[i] = x / (uint32_t)p.H;
    h[i] = x - tok[i] * (uint32_t)p.H;
    a[i] = b[i] = make_uint4(0, 0, 0, 0);
    if (tok[i] < p.nq) {
      a[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.o) + (int64_t)tok[i] * p.os + h[i] * D + e);
      b[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.dout) + (int64_t)tok[i] * p.dos + h[i] * D + e);
    }
  }
#pragma unroll
  for (int i = 0; i < kDsumSteps; ++i) {
    const uint32_t x[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, y[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 4) {
        s = fmaf(__uint_as_float(x[q]), __uint_as_float(y[q]), s);
      } else {
        s = fmaf(__uint_as_float(x[q] << 16), __uint_as_float(y[q] << 16), s);
        s = fmaf(__uint_as_float(x[q] & 0xffff0000u), __uint_as_float(y[q] & 0xffff0000u), s);
      }
    }
#pragma unroll
    for (int q = kLanes / 2; q > 0; q >>= 1) s += __shfl_xor_sync(0xffffffffu, s, q);
    if (e == 0 && tok[i] < p.nq) p.dsum[(int64_t)h[i] * p.nq + tok[i]] = s;
  }
}

// dK (blockIdx.y = 0), dV = the sum of the splits' partials, in split order; 4
// values a thread, small blocks, 16 loads in flight
constexpr int kJoinThreads = 64;
__global__ void __launch_bounds__(kJoinThreads) xattn_dkdv_join_kernel(const XattnParams p) {
  const int64_t x = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
  const int per_row = p.Hk * p.d / 4;
  const int64_t n = p.nk * per_row;
  grid_wait();
  if (x >= n) return;
  const int64_t key = x / per_row;
  const int e = (int)(x % per_row) * 4;
  const bool is_v = blockIdx.y;
  const float* src = (is_v ? p.part_dv : p.part_dk) + x * 4;
  float4 a = make_float4(0, 0, 0, 0);
#pragma unroll 16
  for (int s = 0; s < p.nsplit; ++s) {
    const float4 b = ld4(src + (int64_t)s * n * 4);
    a.x += b.x;
    a.y += b.y;
    a.z += b.z;
    a.w += b.w;
  }
  const float f = is_v ? 1.f : p.scale;
  // a masked key's row is zero, also where a NaN or an infinity of Q or dO met its P and dS of 0
  if (p.mask && !p.mask[key]) a = make_float4(0, 0, 0, 0);
  st4(static_cast<float*>(is_v ? p.dv : p.dk) + key * (is_v ? p.dvs : p.dks) + e,
      make_float4(a.x * f, a.y * f, a.z * f, a.w * f));
}

// O, LSE from the key splits' partials; half a warp a token and head
template <typename T, int D>
__global__ void __launch_bounds__(256) xattn_join_kernel(const XattnParams p) {
  const int64_t x = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 4;
  const int lane = threadIdx.x & 15;
  const int64_t rows = p.nq * p.H;
  grid_wait();
  if (x >= rows) return;
  float m = -INFINITY;
  for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, p.part_ml[s * rows + x].x);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  float4 o[D / 64];
#pragma unroll
  for (int c = 0; c < D / 64; ++c) o[c] = make_float4(0, 0, 0, 0);
  for (int s = 0; s < p.nsplit; ++s) {
    const float2 ml = p.part_ml[s * rows + x];
    const float w = exp2f(ml.x - ref);
    l = fmaf(ml.y, w, l);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const float4 v = ld4(p.part_o + (s * rows + x) * D + lane * 4 + 64 * c);
      o[c].x = fmaf(v.x, w, o[c].x);
      o[c].y = fmaf(v.y, w, o[c].y);
      o[c].z = fmaf(v.z, w, o[c].z);
      o[c].w = fmaf(v.w, w, o[c].w);
    }
  }
  const int64_t tok = x / p.H;
  const int h = (int)(x % p.H);
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
    st4(static_cast<T*>(p.o) + tok * p.os + (int64_t)h * D + lane * 4 + 64 * c,
        make_float4(o[c].x * inv, o[c].y * inv, o[c].z * inv, o[c].w * inv));
  if (lane == 0) p.lse[(int64_t)h * p.nq + tok] = (m + log2f(l)) * kLn2;
}

// ----------------------------------------------------------------- launchers
template <typename F>
static cudaError_t launch(F kern, dim3 grid, size_t smem, const XattnParams& p, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  kern<<<grid, kXsThreads, smem, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_xattn_dkdv_join(const XattnParams& p, cudaStream_t s) {
  return launch_next(xattn_dkdv_join_kernel, dim3((unsigned)((p.nk * p.Hk * p.d / 4 + kJoinThreads - 1) / kJoinThreads), 2),
                     dim3(kJoinThreads), 0, s, p);
}

template <typename T, int D>
static cudaError_t fwd(const XattnParams& p, cudaStream_t s) {
  const size_t smem = sizeof(float) * (3 * kXs * (D + 4) + kXs * kXsLdP + kXs);
  const dim3 grid((unsigned)segment_slots(p.nq, p.B, kXs / p.G), p.Hk, p.nsplit);
  return launch(xattn_fwd_simt_kernel<T, D>, grid, smem, p, s);
}

template <typename T, int D>
static cudaError_t bwd(const XattnParams& p, cudaStream_t s) {
  cudaError_t e = launch_xattn_dsum(p, sizeof(T) == 2, s);
  if (e != cudaSuccess) return e;
  const size_t tiles = sizeof(float) * 4 * kXs * (D + 4), pair = sizeof(float) * kXs * kXsLdP,
               vecs = sizeof(float) * 3 * kXs;
  const uint32_t kslots = (uint32_t)segment_slots(p.nk, p.B, kXs), qslots = (uint32_t)segment_slots(p.nq, p.B, kXs / p.G);
  const int64_t n_kv = p.nk > 0 ? (int64_t)kslots * p.Hk * p.nsplit : 0, n_q = p.nq > 0 ? (int64_t)qslots * p.Hk : 0;
  if (n_kv + n_q > INT32_MAX) return cudaErrorInvalidValue;
  const size_t smem = tiles + 2 * pair + vecs;
  e = cudaFuncSetAttribute(xattn_bwd_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess)
    e = launch_next(xattn_bwd_simt_kernel<T, D>, dim3((unsigned)(n_kv + n_q)), dim3(kXsThreads), smem, s, p,
                    (uint32_t)n_kv, kslots, qslots);
  if (e == cudaSuccess && p.nk > 0) e = launch_xattn_dkdv_join(p, s);
  return e;
}

int64_t xattn_items(const XattnParams& p, bool bf16, bool backward) {
  if (bf16) return backward ? xattn_bwd_tc_items(p) : xattn_fwd_tc_items(p);
  return (backward ? segment_slots(p.nk, p.B, kXs) : segment_slots(p.nq, p.B, kXs / p.G)) * p.Hk;
}

// In fp32 enough parts for two blocks an SM (four backward, where two share an
// SM and lengths differ), in bf16 whole waves; none shorter than two tiles of
// an average segment (one backward).
int xattn_splits(const XattnParams& p, bool bf16, bool backward) {
  if (bf16 && backward) return 1;
  const int64_t items = xattn_items(p, bf16, backward);
  int64_t want = ((backward ? 4 : 2) * (int64_t)p.sms + items - 1) / items;
  if (bf16) {
    // Persistent CTAs, one per SM: the fewest whole waves of items that fill
    // the SMs (to a tenth of the best of four).  One query of 24 heads over
    // 85,202 keys: 6 splits in one wave 157 us, 13 in three waves 205 us.
    double best = 0;
    want = 1;
    for (int w = 1; w <= 4; ++w) {
      const int64_t n = (int64_t)w * p.sms / items;
      const double use = (double)(n * items) / ((double)w * p.sms);
      if (n >= 1 && use > best + 0.1) {
        best = use;
        want = n;
      }
    }
  }
  const int64_t tile = backward ? kXs / p.G : (bf16 ? 128 : kXs);
  const int64_t tiles = ((backward ? p.nq : p.nk) / p.B + tile - 1) / tile, most = backward ? tiles : tiles / 2;
  const int64_t n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

cudaError_t launch_xattn_fwd_simt(const XattnParams& p, cudaStream_t s) {
  return p.d == 64 ? fwd<float, 64>(p, s) : fwd<float, 128>(p, s);
}

cudaError_t launch_xattn_join(const XattnParams& p, bool bf16, cudaStream_t s) {
  const dim3 grid((unsigned)((p.nq * p.H + 15) / 16)), block(kXsThreads);
  if (bf16)
    return p.d == 64 ? launch_next(xattn_join_kernel<__nv_bfloat16, 64>, grid, block, 0, s, p)
                     : launch_next(xattn_join_kernel<__nv_bfloat16, 128>, grid, block, 0, s, p);
  return p.d == 64 ? launch_next(xattn_join_kernel<float, 64>, grid, block, 0, s, p)
                   : launch_next(xattn_join_kernel<float, 128>, grid, block, 0, s, p);
}

template <typename T, int D>
static cudaError_t dsum(const XattnParams& p, cudaStream_t s) {
  constexpr int64_t rows = 256 * 16 / sizeof(T) / D * kDsumSteps;  // of a block
  return launch(xattn_dsum_kernel<T, D>, dim3((unsigned)((p.nq * p.H + rows) / rows)), 0, p, s);
}
cudaError_t launch_xattn_dsum(const XattnParams& p, bool bf16, cudaStream_t s) {
  if (bf16) return p.d == 64 ? dsum<__nv_bfloat16, 64>(p, s) : dsum<__nv_bfloat16, 128>(p, s);
  return p.d == 64 ? dsum<float, 64>(p, s) : dsum<float, 128>(p, s);
}

cudaError_t launch_xattn_bwd_simt(const XattnParams& p, cudaStream_t s) {
  return p.d == 64 ? bwd<float, 64>(p, s) : bwd<float, 128>(p, s);
}

}  // namespace ut
