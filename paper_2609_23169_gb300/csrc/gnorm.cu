// Group norm with an activation, channels last, over ragged segments.
//
// Segment s (n rows), group g of C/G channels, M = n C/G values:
//   mu = mean, var = mean of (x - mu)^2,  r = 1 / sqrt(var + eps)
//   xh = (x - mu) r,  u = gamma xh + beta,  y = act(u)
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du xh,
//   a = sum_g gamma du,  b = sum_g gamma du xh,
//   dx = r (gamma du - (a + xh b) / M)
//
// Forward: statistics of each slot (R rows of one segment), the segments'
// statistics from their slots', then the rows.  Backward: the sums of du and
// du xh per slot and channel, their sums per segment, then the rows.  A
// thread owns one 16-byte column of channels, so any number of channels per
// group works, and reads rows in batches, all loads of a batch in flight.
//
// Statistics are never sums of squares: a batch's mean and its sum of squared
// distances from that mean are merged pairwise into the running ones,
//   M2 = M2a + M2b + (mean_b - mean_a)^2 na nb / (na + nb),
// so a mean far from zero costs no digits.  All sums are in 32 bits, of a
// batch first and of batches then, in an order that the sizes fix.
#include <math.h>

#include "common.cuh"
#include "gnorm.cuh"
#include "kernels.h"
#include "segments.cuh"

namespace ut {

constexpr int kGnThreads = 256;
constexpr int kGnBatch = 8;  // rows a thread has in flight

template <typename T>
struct Vec;  // 16 bytes of channels
template <>
struct Vec<float> {
  static constexpr int n = 4;
  UT_DEV static void load(const float* p, float (&v)[4]) { *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p); }
  UT_DEV static void store(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(v); }
  UT_DEV static void unpack(const uint4& u, float (&v)[4]) { *reinterpret_cast<uint4*>(v) = u; }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  UT_DEV static void unpack(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  UT_DEV static void store(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
};

UT_DEV float sigmoid(float u) { return 1.f / (1.f + __expf(-u)); }

// A block's rows of a slot: the threads cover `cols` 16-byte columns from
// col0, and `lanes` rows at a time.
struct GnLayout {
  int cols, lanes, col, lane;
  bool on;
  UT_DEV GnLayout(int cv, int col0) {
    cols = min(cv - col0, kGnThreads);
    lanes = kGnThreads / cols;
    col = col0 + threadIdx.x % cols;
    lane = threadIdx.x / cols;
    on = lane < lanes;
  }
  UT_DEV int rows_of(int lane_, int64_t n) const { return lane_ < n ? (int)((n - lane_ + lanes - 1) / lanes) : 0; }
};

// part[slot][G] = (mean, M2) of the slot's values of each group
template <typename T>
__global__ void __launch_bounds__(kGnThreads) gn_stats_kernel(const GnormParams p, float2* __restrict__ part) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ float sm[];
  float2* lane_stat = reinterpret_cast<float2*>(sm);               // [V][256]
  float2* chan = lane_stat + V * kGnThreads;                       // [C]
  if (blockIdx.x == 0) check_cu(p.cu, p.B, p.n, p.status);
  const Segment g = segment_of_slot(p.cu, p.B, p.n, p.R, blockIdx.x);
  const int64_t r0 = g.tile * p.R, n = min((int64_t)p.R, g.n - r0);
  if (n <= 0) return;
  const int cv = p.C / V;
  for (int col0 = 0; col0 < cv; col0 += kGnThreads) {
    const GnLayout L(cv, col0);
    float mean[V], m2[V];
#pragma unroll
    for (int c = 0; c < V; ++c) mean[c] = m2[c] = 0.f;
    float cnt = 0.f;
    if (L.on) {
      const T* src = static_cast<const T*>(p.x) + (g.row + r0) * p.xs + (int64_t)L.col * V;
      for (int64_t r = L.lane; r < n; r += (int64_t)L.lanes * kGnBatch) {
        uint4 w[kGnBatch];
        int have = 0;
#pragma unroll
        for (int b = 0; b < kGnBatch; ++b) {
          const int64_t row = r + (int64_t)b * L.lanes;
          if (row < n) {
            w[b] = ld_nc_v4(src + row * p.xs);
            ++have;
          }
        }
        const float nb = (float)have, inv = 1.f / nb, tot = cnt + nb;
        const float wb = nb / tot, wm = cnt * wb;
        float v[kGnBatch][V];
#pragma unroll
        for (int b = 0; b < kGnBatch; ++b) Vec<T>::unpack(w[b], v[b]);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          float s = 0.f, q = 0.f;
#pragma unroll
          for (int b = 0; b < kGnBatch; ++b)
            if (b < have) s += v[b][c];
          const float mb = s * inv;
#pragma unroll
          for (int b = 0; b < kGnBatch; ++b)
            if (b < have) q = fmaf(v[b][c] - mb, v[b][c] - mb, q);
          const float d = mb - mean[c];
          m2[c] += fmaf(d * d, wm, q);
          mean[c] = fmaf(d, wb, mean[c]);
        }
        cnt = tot;
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < V; ++c) lane_stat[c * kGnThreads + threadIdx.x] = make_float2(mean[c], m2[c]);
    __syncthreads();
    for (int ch = threadIdx.x; ch < L.cols * V; ch += kGnThreads) {
      const float2* st = lane_stat + (ch % V) * kGnThreads + ch / V;
      float s = 0.f, q = 0.f;
      for (int l = 0; l < L.lanes; ++l) s = fmaf((float)L.rows_of(l, n), st[l * L.cols].x, s);
      const float m = s / (float)n;
      for (int l = 0; l < L.lanes; ++l) {
        const float2 a = st[l * L.cols];
        q += fmaf((float)L.rows_of(l, n) * (a.x - m), a.x - m, a.y);
      }
      chan[col0 * V + ch] = make_float2(m, q);
    }
  }
  __syncthreads();
  const int cpg = p.C / p.G, lane = threadIdx.x & 31;
  for (int gr = threadIdx.x >> 5; gr < p.G; gr += kGnThreads / 32) {
    float s = 0.f, q = 0.f;
    for (int c = lane; c < cpg; c += 32) s += chan[gr * cpg + c].x;
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const float m = s / (float)cpg;
    for (int c = lane; c < cpg; c += 32) {
      const float2 a = chan[gr * cpg + c];
      q += fmaf((float)n * (a.x - m), a.x - m, a.y);
    }
    for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
    if (lane == 0) part[(int64_t)blockIdx.x * p.G + gr] = make_float2(m, q);
  }
}

// first slot of segment s, whose rows start at `row`
UT_DEV int64_t first_slot(const GnormParams& p, int s, int64_t row) { return row / p.R + s; }

// grid (segments): statistics of the segment; a warp a group
__global__ void __launch_bounds__(kGnThreads) gn_final_kernel(const GnormParams p, const float2* __restrict__ part) {
  const int s = blockIdx.x, lane = threadIdx.x & 31;
  int64_t row, n;
  segment_rows(p.cu, s, p.n, row, n);
  const int64_t slots = (n + p.R - 1) / p.R;
  const float2* src = part + first_slot(p, s, row) * p.G;
  const float cpg = (float)(p.C / p.G);
  for (int g = threadIdx.x >> 5; g < p.G; g += kGnThreads / 32) {
    float m = 0.f, q = 0.f;
    for (int64_t i = lane; i < slots; i += 32) m = fmaf((float)min((int64_t)p.R, n - i * p.R), src[i * p.G + g].x, m);
    for (int o = 16; o; o >>= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
    m = n > 0 ? m / (float)n : 0.f;
    for (int64_t i = lane; i < slots; i += 32) {
      const float2 a = src[i * p.G + g];
      q += fmaf((float)min((int64_t)p.R, n - i * p.R) * cpg * (a.x - m), a.x - m, a.y);
    }
    for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
    if (lane == 0) {
      p.mean[(int64_t)s * p.G + g] = m;
      p.rstd[(int64_t)s * p.G + g] = 1.f / sqrtf((n > 0 ? q / ((float)n * cpg) : 0.f) + p.eps);
    }
  }
}

// this thread's channels: mean, rstd, gamma, beta
template <int V>
struct GnChannels {
  float mean[V], rstd[V], gamma[V], beta[V];
  UT_DEV GnChannels(const GnormParams& p, int s, int c0) {
    const int cpg = p.C / p.G;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int g = (c0 + c) / cpg;
      mean[c] = p.mean[(int64_t)s * p.G + g];
      rstd[c] = p.rstd[(int64_t)s * p.G + g];
      gamma[c] = p.gamma ? p.gamma[c0 + c] : 1.f;
      beta[c] = p.beta ? p.beta[c0 + c] : 0.f;
    }
  }
};

template <typename T, bool kAct>
__global__ void __launch_bounds__(kGnThreads) gn_apply_kernel(const GnormParams p) {
  constexpr int V = 16 / sizeof(T);
  const Segment g = segment_of_slot(p.cu, p.B, p.n, p.R, blockIdx.x);
  const int64_t r0 = g.tile * p.R, n = min((int64_t)p.R, g.n - r0);
  if (n <= 0) return;
  const int cv = p.C / V;
  for (int col0 = 0; col0 < cv; col0 += kGnThreads) {
    const GnLayout L(cv, col0);
    if (!L.on) continue;
    const GnChannels<V> ch(p, g.s, L.col * V);
    const T* src = static_cast<const T*>(p.x) + (g.row + r0) * p.xs + (int64_t)L.col * V;
    T* dst = static_cast<T*>(p.y) + (g.row + r0) * p.ys + (int64_t)L.col * V;
    for (int64_t r = L.lane; r < n; r += (int64_t)L.lanes * kGnBatch) {
      uint4 w[kGnBatch];
#pragma unroll
      for (int b = 0; b < kGnBatch; ++b) {
        const int64_t row = r + (int64_t)b * L.lanes;
        if (row < n) w[b] = ld_nc_v4(src + row * p.xs);
      }
#pragma unroll
      for (int b = 0; b < kGnBatch; ++b) {
        const int64_t row = r + (int64_t)b * L.lanes;
        if (row >= n) break;
        float v[V];
        Vec<T>::unpack(w[b], v);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float u = fmaf(v[c] - ch.mean[c], ch.rstd[c] * ch.gamma[c], ch.beta[c]);
          v[c] = kAct ? u * sigmoid(u) : u;
        }
        Vec<T>::store(dst + row * p.ys, v);
      }
    }
  }
}

// xh and du of one value
template <bool kAct>
UT_DEV float gn_du(float x, float dy, float mean, float rstd, float gamma, float beta, float& xh) {
  xh = (x - mean) * rstd;
  if (!kAct) return dy;
  const float u = fmaf(xh, gamma, beta), s = sigmoid(u);
  return dy * (s * fmaf(u, 1.f - s, 1.f));
}

// part[slot][2][C]: sums of du and of du xh over the slot's rows
template <typename T, bool kAct>
__global__ void __launch_bounds__(kGnThreads) gn_bwd_sums_kernel(const GnormParams p, float* __restrict__ part) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ float sm[];
  float2* lane_sum = reinterpret_cast<float2*>(sm);  // [V][256]
  if (blockIdx.x == 0) check_cu(p.cu, p.B, p.n, p.status);
  const Segment g = segment_of_slot(p.cu, p.B, p.n, p.R, blockIdx.x);
  const int64_t r0 = g.tile * p.R, n = min((int64_t)p.R, g.n - r0);
  if (n <= 0) return;
  const int cv = p.C / V;
  for (int col0 = 0; col0 < cv; col0 += kGnThreads) {
    const GnLayout L(cv, col0);
    float s1[V], s2[V];
#pragma unroll
    for (int c = 0; c < V; ++c) s1[c] = s2[c] = 0.f;
    if (L.on) {
      const GnChannels<V> ch(p, g.s, L.col * V);
      const T* xp = static_cast<const T*>(p.x) + (g.row + r0) * p.xs + (int64_t)L.col * V;
      const T* dp = static_cast<const T*>(p.dy) + (g.row + r0) * p.dys + (int64_t)L.col * V;
      for (int64_t r = L.lane; r < n; r += (int64_t)L.lanes * 4) {
        uint4 w[4], d[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int64_t row = r + (int64_t)b * L.lanes;
          if (row < n) {
            w[b] = ld_nc_v4(xp + row * p.xs);
            d[b] = ld_nc_v4(dp + row * p.dys);
          }
        }
        float b1[V], b2[V];
#pragma unroll
        for (int c = 0; c < V; ++c) b1[c] = b2[c] = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (r + (int64_t)b * L.lanes >= n) break;
          float v[V], e[V];
          Vec<T>::unpack(w[b], v);
          Vec<T>::unpack(d[b], e);
#pragma unroll
          for (int c = 0; c < V; ++c) {
            float xh;
            const float du = gn_du<kAct>(v[c], e[c], ch.mean[c], ch.rstd[c], ch.gamma[c], ch.beta[c], xh);
            b1[c] += du;
            b2[c] = fmaf(du, xh, b2[c]);
          }
        }
#pragma unroll
        for (int c = 0; c < V; ++c) {
          s1[c] += b1[c];
          s2[c] += b2[c];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < V; ++c) lane_sum[c * kGnThreads + threadIdx.x] = make_float2(s1[c], s2[c]);
    __syncthreads();
    for (int ch = threadIdx.x; ch < L.cols * V; ch += kGnThreads) {
      const float2* st = lane_sum + (ch % V) * kGnThreads + ch / V;
      float a = 0.f, b = 0.f;
      for (int l = 0; l < L.lanes; ++l) {
        a += st[l * L.cols].x;
        b += st[l * L.cols].y;
      }
      float* out = part + (int64_t)blockIdx.x * 2 * p.C + col0 * V + ch;
      out[0] = a;
      out[p.C] = b;
    }
  }
}

// grid (segments, 2 C / 32), block (32, 8): seg[s][2][C] from the slots' sums
__global__ void __launch_bounds__(256) gn_bwd_slots_kernel(const GnormParams p, const float* __restrict__ part,
                                                           float* __restrict__ seg) {
  __shared__ float sum[8][33];
  const int s = blockIdx.x, c = blockIdx.y * 32 + threadIdx.x;
  int64_t row, n;
  segment_rows(p.cu, s, p.n, row, n);
  const int64_t slots = (n + p.R - 1) / p.R, first = first_slot(p, s, row);
  float a = 0.f;
  if (c < 2 * p.C)
    for (int64_t i = threadIdx.y; i < slots; i += 8) a += part[(first + i) * 2 * p.C + c];
  sum[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y == 0 && c < 2 * p.C) {
    for (int l = 1; l < 8; ++l) a += sum[l][threadIdx.x];
    seg[(int64_t)s * 2 * p.C + c] = a;
  }
}

// blocks 0 .. B-1: coef[s][G] = (a, b) / M; the others: dgamma, dbeta
__global__ void __launch_bounds__(256) gn_bwd_final_kernel(const GnormParams p, const float* __restrict__ seg,
                                                           float2* __restrict__ coef) {
  if ((int)blockIdx.x < p.B) {
    const int s = blockIdx.x, lane = threadIdx.x & 31, cpg = p.C / p.G;
    int64_t row, n;
    segment_rows(p.cu, s, p.n, row, n);
    const float inv = n > 0 ? 1.f / ((float)n * (float)cpg) : 0.f;
    const float* src = seg + (int64_t)s * 2 * p.C;
    for (int g = threadIdx.x >> 5; g < p.G; g += 8) {
      float a = 0.f, b = 0.f;
      for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 32) {
        const float w = p.gamma ? p.gamma[c] : 1.f;
        a = fmaf(w, src[c], a);
        b = fmaf(w, src[p.C + c], b);
      }
      for (int o = 16; o; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
      }
      if (lane == 0) coef[(int64_t)s * p.G + g] = make_float2(a * inv, b * inv);
    }
    return;
  }
  const int c = ((int)blockIdx.x - p.B) * 256 + threadIdx.x;
  if (c >= p.C) return;
  float a = 0.f, b = 0.f;
  for (int s = 0; s < p.B; ++s) {
    a += seg[(int64_t)s * 2 * p.C + c];
    b += seg[(int64_t)s * 2 * p.C + p.C + c];
  }
  if (p.dbeta) p.dbeta[c] = a;
  if (p.dgamma) p.dgamma[c] = b;
}

template <typename T, bool kAct>
__global__ void __launch_bounds__(kGnThreads) gn_dx_kernel(const GnormParams p, const float2* __restrict__ coef) {
  constexpr int V = 16 / sizeof(T);
  const Segment g = segment_of_slot(p.cu, p.B, p.n, p.R, blockIdx.x);
  const int64_t r0 = g.tile * p.R, n = min((int64_t)p.R, g.n - r0);
  if (n <= 0) return;
  const int cv = p.C / V, cpg = p.C / p.G;
  for (int col0 = 0; col0 < cv; col0 += kGnThreads) {
    const GnLayout L(cv, col0);
    if (!L.on) continue;
    const GnChannels<V> ch(p, g.s, L.col * V);
    float2 ab[V];
#pragma unroll
    for (int c = 0; c < V; ++c) ab[c] = coef[(int64_t)g.s * p.G + (L.col * V + c) / cpg];
    const T* xp = static_cast<const T*>(p.x) + (g.row + r0) * p.xs + (int64_t)L.col * V;
    const T* dp = static_cast<const T*>(p.dy) + (g.row + r0) * p.dys + (int64_t)L.col * V;
    T* out = static_cast<T*>(p.dx) + (g.row + r0) * p.dxs + (int64_t)L.col * V;
    for (int64_t r = L.lane; r < n; r += (int64_t)L.lanes * 4) {
      uint4 w[4], d[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int64_t row = r + (int64_t)b * L.lanes;
        if (row < n) {
          w[b] = ld_nc_v4(xp + row * p.xs);
          d[b] = ld_nc_v4(dp + row * p.dys);
        }
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int64_t row = r + (int64_t)b * L.lanes;
        if (row >= n) break;
        float v[V], e[V];
        Vec<T>::unpack(w[b], v);
        Vec<T>::unpack(d[b], e);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          float xh;
          const float du = gn_du<kAct>(v[c], e[c], ch.mean[c], ch.rstd[c], ch.gamma[c], ch.beta[c], xh);
          v[c] = ch.rstd[c] * (fmaf(ch.gamma[c], du, -ab[c].x) - xh * ab[c].y);
        }
        Vec<T>::store(out + row * p.dxs, v);
      }
    }
  }
}

// ----------------------------------------------------------------- launchers
// Rows of a slot: about 32 KB of a tensor, so that a block has a few batches
// of 16-byte columns to overlap, but no fewer than 4 blocks an SM.
int gnorm_rows_per_slot(int64_t n, int C, int elem, int sms) {
  int64_t r = 32768 / ((int64_t)C * elem), most = (n + 4 * (int64_t)sms - 1) / (4 * (int64_t)sms);
  const int64_t big = (n + 8 * (int64_t)sms - 1) / (8 * (int64_t)sms);  // at most about 8 blocks an SM
  if (r > most) r = most;
  if (r < big) r = big;
  return (int)(r < 1 ? 1 : r);
}

size_t gnorm_ws(const GnormParams& p, bool backward) {
  const size_t slots = (size_t)segment_slots(p.n, p.B, p.R);
  if (!backward) return slots * p.G * sizeof(float2);
  return (slots + p.B) * 2 * p.C * sizeof(float) + (size_t)p.B * p.G * sizeof(float2);
}

template <typename F>
static cudaError_t allow(F kern, size_t smem) {
  return smem > 48 * 1024 ? cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)
                          : cudaSuccess;
}

template <typename T>
static cudaError_t fwd(const GnormParams& p, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const unsigned slots = (unsigned)segment_slots(p.n, p.B, p.R);
  float2* part = static_cast<float2*>(p.ws);
  const size_t smem = sizeof(float2) * (V * kGnThreads + (size_t)p.C);
  cudaError_t e = allow(gn_stats_kernel<T>, smem);
  if (e != cudaSuccess) return e;
  gn_stats_kernel<T><<<slots, kGnThreads, smem, s>>>(p, part);
  gn_final_kernel<<<p.B, kGnThreads, 0, s>>>(p, part);
  if (p.act) gn_apply_kernel<T, true><<<slots, kGnThreads, 0, s>>>(p);
  else gn_apply_kernel<T, false><<<slots, kGnThreads, 0, s>>>(p);
  return cudaGetLastError();
}

template <typename T, bool kAct>
static cudaError_t bwd(const GnormParams& p, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const unsigned slots = (unsigned)segment_slots(p.n, p.B, p.R);
  float* part = static_cast<float*>(p.ws);
  float* seg = part + (size_t)slots * 2 * p.C;
  float2* coef = reinterpret_cast<float2*>(seg + (size_t)p.B * 2 * p.C);
  gn_bwd_sums_kernel<T, kAct><<<slots, kGnThreads, sizeof(float2) * V * kGnThreads, s>>>(p, part);
  gn_bwd_slots_kernel<<<dim3(p.B, (2 * p.C + 31) / 32), dim3(32, 8), 0, s>>>(p, part, seg);
  gn_bwd_final_kernel<<<p.B + (p.C + 255) / 256, 256, 0, s>>>(p, seg, coef);
  gn_dx_kernel<T, kAct><<<slots, kGnThreads, 0, s>>>(p, coef);
  return cudaGetLastError();
}

cudaError_t launch_gnorm_fwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  return bf16 ? fwd<__nv_bfloat16>(p, s) : fwd<float>(p, s);
}
cudaError_t launch_gnorm_bwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  if (bf16) return p.act ? bwd<__nv_bfloat16, true>(p, s) : bwd<__nv_bfloat16, false>(p, s);
  return p.act ? bwd<float, true>(p, s) : bwd<float, false>(p, s);
}

}  // namespace ut
