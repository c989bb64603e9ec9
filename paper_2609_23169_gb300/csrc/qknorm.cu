// RMS norms of the heads of Q and K with the position rotation in the same
// pass.  For a token's head x (d values), weights w and position t:
//   r = 1 / sqrt(mean(x^2) + eps),   y = R(t) (x r w)
// and backward, given dy, with g = R(t)^T dy and xh = x r:
//   dw = sum over tokens and heads of g xh
//   dx = r (g w - xh mean(g w xh))
// R(t) turns the pair (2j, 2j + 1) by coordinate * frequency (the axes of
// ut_rope).  The forward also puts K, and V unchanged, into given rows of a
// cache.
//
// Positions run to 2^31, where the fp32 product coordinate * frequency is off
// by whole radians.  So a pair's frequency is held in turns as a 64-bit
// fraction; the product with the integer coordinate wraps at whole turns, which
// is all that sin and cos want: its upper 32 bits are the turn, exact to 2^-32.
//
// One warp takes a token; a head's 16-byte vectors lie in neighbouring lanes (8
// to 32 of them), a lane meets the same pairs in every head, so it takes their
// sines once a token, and its columns of w and dw stay in registers.  Where
// there are few tokens their heads are dealt out to several warps.  Up to kVec
// loads a lane in flight.  Bound by memory: Q and K are read once and written
// once (backward: x and dy read, dx written).
// dw: a lane's sums over its tokens, then over the block's warps in shared
// memory, then over blocks by a second kernel, always in the same order.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "qknorm.cuh"
#include "xattn.cuh"

namespace ut {

namespace {

constexpr int kQnThreads = 256, kQnWarps = kQnThreads / 32;

template <typename T>
struct Vec {
  static constexpr int kVals = 16 / sizeof(T);
};

template <typename T>
UT_DEV void unpack(const uint4& u, float (&x)[Vec<T>::kVals]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}
template <typename T>
UT_DEV uint4 pack(const float (&x)[Vec<T>::kVals]) {
  if constexpr (sizeof(T) == 2)
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
  else
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <int kLanes>
UT_DEV float head_sum(float x) {  // over the lanes of a head
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// What a lane keeps: its pairs, and their sines at the token's position.
template <typename T, int D>
struct Lane {
  static constexpr int kVals = Vec<T>::kVals, kPairs = kVals / 2, kLanes = D / kVals, kHeads = 32 / kLanes;
  uint64_t turn[kPairs];
  uint32_t axis[kPairs];
  float cs[kPairs], sn[kPairs];
  int group, col;  // the head of a step, the first of its columns

  UT_DEV void init(const QkNormParams& p, int lane) {
    group = lane / kLanes;
    col = (lane % kLanes) * kVals;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      turn[e] = p.turn[col / 2 + e];
      axis[e] = p.axis[col / 2 + e];
    }
  }
  UT_DEV void turn_to(const QkNormParams& p, int32_t pos) {
    const uint32_t t = (uint32_t)max(0, pos - min(pos, p.prefix));  // before the images: (0, 0, 0)
    const uint32_t image = t / p.area, in = t - image * p.area, y = in / p.side, x = in - y * p.side;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      const uint32_t c = axis[e] == 0 ? image : (axis[e] == 1 ? y : x);
      const int32_t part = (int32_t)(((uint64_t)c * turn[e]) >> 32);  // in half turns of 2^-31
      sincospif((float)part * 4.656612873077393e-10f, &sn[e], &cs[e]);
    }
  }
  UT_DEV void weights(const float* w, float (&out)[kVals]) const {
#pragma unroll
    for (int e = 0; e < kVals; ++e) out[e] = w ? w[col + e] : 1.f;
  }
};

// Steps [s, end) of one tensor of a token, kHeads heads each: y = R (x r w), or
// a copy.  With the weights in the rotation, a w cos and so on, a pair takes four
// multiplications and a head its r at the end.
template <typename T, int D, int kVec, bool kNorm>
UT_DEV void forward_part(const Lane<T, D>& me, const T* src, T* dst, int heads, int s, int end, const float* wt,
                         const QkNormParams& p) {
  using L = Lane<T, D>;
  if (s >= end) return;
  float wc[L::kVals], ws[L::kVals];  // w cos, w sin
  bool ready = false;
  for (; s < end; s += kVec) {
    uint4 w[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int h = (s + j) * L::kHeads + me.group;
      w[j] = make_uint4(0, 0, 0, 0);
      if (s + j < end && h < heads) w[j] = *reinterpret_cast<const uint4*>(src + h * D + me.col);
    }
    if (kNorm && !ready) {  // while the loads fly
      float v[L::kVals];
      me.weights(wt, v);
#pragma unroll
      for (int e = 0; e < L::kVals; ++e) {
        wc[e] = v[e] * me.cs[e / 2];
        ws[e] = v[e] * me.sn[e / 2];
      }
      ready = true;
    }
    if constexpr (kNorm) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        float v[L::kVals], sum = 0.f;
        unpack<T>(w[j], v);
#pragma unroll
        for (int e = 0; e < L::kVals; ++e) sum = fmaf(v[e], v[e], sum);
        const float r = rsqrtf(head_sum<L::kLanes>(sum) * (1.f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < L::kVals; e += 2) {
          const float x = v[e] * r, y = v[e + 1] * r;
          v[e] = fmaf(x, wc[e], -y * ws[e + 1]);
          v[e + 1] = fmaf(x, ws[e], y * wc[e + 1]);
        }
        w[j] = pack<T>(v);
      }
    }
    if (!dst) continue;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int h = (s + j) * L::kHeads + me.group;
      if (s + j < end && h < heads) *reinterpret_cast<uint4*>(dst + h * D + me.col) = w[j];
    }
  }
}

// grid: warps take (token, part of its steps)
template <typename T, int D, int kVec>
__global__ void __launch_bounds__(kQnThreads, 3) qknorm_fwd_kernel(const __grid_constant__ QkNormParams p, int parts,
                                                                   int per) {
  using L = Lane<T, D>;
  const int lane = threadIdx.x & 31;
  L me;
  me.init(p, lane);
  const int nq = (p.H + L::kHeads - 1) / L::kHeads, nk = (p.Hk + L::kHeads - 1) / L::kHeads;  // steps
  const int64_t warps = (int64_t)gridDim.x * kQnWarps, units = p.n * parts;
  int64_t u = (int64_t)blockIdx.x * kQnWarps + (threadIdx.x >> 5);
  auto pos_of = [&](int64_t unit) -> int32_t {
    const int64_t row = unit / parts;
    return p.pos ? p.pos[row] : (int32_t)row;
  };
  int32_t next = u < units ? pos_of(u) : 0;
  for (; u < units; u += warps) {
    const int64_t row = u / parts;
    const int s0 = (int)(u - row * parts) * per, s1 = s0 + per;
    const int32_t pos = next;
    if (u + warps < units) next = pos_of(u + warps);  // a token ahead
    int64_t to = row;  // of K and V
    bool keep = true;
    if (p.rows) {
      to = p.rows[row];
      keep = to >= 0 && to < p.cache_rows;
      if (to >= p.cache_rows && lane == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    }
    if (s0 < nq + nk) me.turn_to(p, pos);
    forward_part<T, D, kVec, true>(me, static_cast<const T*>(p.q) + row * p.qs, static_cast<T*>(p.qo) + row * p.qos, p.H,
                                   s0, min(s1, nq), p.wq, p);
    forward_part<T, D, kVec, true>(me, static_cast<const T*>(p.k) + row * p.ks,
                                   keep ? static_cast<T*>(p.ko) + to * p.kos : nullptr, p.Hk, max(s0 - nq, 0),
                                   min(s1 - nq, nk), p.wk, p);
    if (p.vo)
      forward_part<T, D, kVec, false>(me, static_cast<const T*>(p.v) + row * p.vs,
                                      keep ? static_cast<T*>(p.vo) + to * p.vos : nullptr, p.Hk, max(s0 - nq - nk, 0),
                                      min(s1 - nq - nk, nk), nullptr, p);
  }
}

// The heads of one tensor of a token, backward; dw += its terms.
template <typename T, int D, int kVec>
UT_DEV void backward_part(const Lane<T, D>& me, const T* src, const T* grad, T* dst, int heads, const float* wt,
                          float (&dw)[Vec<T>::kVals], const QkNormParams& p) {
  using L = Lane<T, D>;
  const int end = (heads + L::kHeads - 1) / L::kHeads;
  float wv[L::kVals];
  me.weights(wt, wv);
  for (int s = 0; s < end; s += kVec) {
    uint4 w[kVec], dy[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int h = (s + j) * L::kHeads + me.group;
      w[j] = dy[j] = make_uint4(0, 0, 0, 0);
      if (s + j < end && h < heads) {
        w[j] = *reinterpret_cast<const uint4*>(src + h * D + me.col);
        dy[j] = *reinterpret_cast<const uint4*>(grad + h * D + me.col);
      }
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      float v[L::kVals], g[L::kVals], ss = 0.f, sg = 0.f;
      unpack<T>(w[j], v);
      unpack<T>(dy[j], g);
#pragma unroll
      for (int e = 0; e < L::kPairs; ++e) {
        const float a = g[2 * e], b = g[2 * e + 1];
        g[2 * e] = fmaf(a, me.cs[e], b * me.sn[e]);
        g[2 * e + 1] = fmaf(b, me.cs[e], -a * me.sn[e]);
      }
      float t[L::kVals];  // g x
#pragma unroll
      for (int e = 0; e < L::kVals; ++e) {
        t[e] = g[e] * v[e];
        ss = fmaf(v[e], v[e], ss);
        sg = fmaf(t[e], wv[e], sg);
      }
      const float r = rsqrtf(head_sum<L::kLanes>(ss) * (1.f / D) + p.eps);
      const float c = head_sum<L::kLanes>(sg) * (1.f / D) * r * r;  // mean(g w xh) r
#pragma unroll
      for (int e = 0; e < L::kVals; ++e) {
        dw[e] = fmaf(t[e], r, dw[e]);
        v[e] = r * fmaf(-v[e], c, g[e] * wv[e]);
      }
      const int h = (s + j) * L::kHeads + me.group;
      if (s + j < end && h < heads) *reinterpret_cast<uint4*>(dst + h * D + me.col) = pack<T>(v);
    }
  }
}

template <typename T, int D, int kVec>
__global__ void __launch_bounds__(kQnThreads, kQnBlocksPerSm) qknorm_bwd_kernel(const __grid_constant__ QkNormParams p) {
  using L = Lane<T, D>;
  __shared__ float sums[kQnWarps * L::kHeads][2][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_next();
  L me;
  me.init(p, lane);
  float dwq[L::kVals], dwk[L::kVals];
#pragma unroll
  for (int e = 0; e < L::kVals; ++e) dwq[e] = dwk[e] = 0.f;
  const int64_t warps = (int64_t)gridDim.x * kQnWarps;
  int64_t row = (int64_t)blockIdx.x * kQnWarps + warp;
  auto pos_of = [&](int64_t at) -> int32_t { return p.pos ? p.pos[at] : (int32_t)at; };
  int32_t next = row < p.n ? pos_of(row) : 0;
  for (; row < p.n; row += warps) {
    me.turn_to(p, next);
    if (row + warps < p.n) next = pos_of(row + warps);  // a token ahead
    backward_part<T, D, kVec>(me, static_cast<const T*>(p.q) + row * p.qs, static_cast<const T*>(p.dqo) + row * p.dqos,
                              static_cast<T*>(p.qo) + row * p.qos, p.H, p.wq, dwq, p);
    backward_part<T, D, kVec>(me, static_cast<const T*>(p.k) + row * p.ks, static_cast<const T*>(p.dko) + row * p.dkos,
                              static_cast<T*>(p.ko) + row * p.kos, p.Hk, p.wk, dwk, p);
  }
#pragma unroll
  for (int e = 0; e < L::kVals; ++e) {
    sums[warp * L::kHeads + me.group][0][me.col + e] = dwq[e];
    sums[warp * L::kHeads + me.group][1][me.col + e] = dwk[e];
  }
  __syncthreads();
  for (int x = threadIdx.x; x < 2 * D; x += kQnThreads) {
    float a = 0.f;
    for (int i = 0; i < kQnWarps * L::kHeads; ++i) a += sums[i][x / D][x % D];
    p.part[(int64_t)blockIdx.x * 2 * D + x] = a;
  }
}

// dw = the sum of the blocks' parts; a block 32 columns, 16 threads a column
__global__ void __launch_bounds__(512) qknorm_dw_kernel(const float* part, int blocks, int d, float* dwq, float* dwk) {
  __shared__ float sums[16][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), i0 = threadIdx.x >> 5;
  grid_wait();
  float a = 0.f;
#pragma unroll 8
  for (int i = i0; i < blocks; i += 16) a += part[(int64_t)i * 2 * d + col];
  sums[i0][threadIdx.x & 31] = a;
  __syncthreads();
  if (i0 > 0) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) a += sums[i][threadIdx.x];
  float* out = col < d ? dwq : dwk;
  if (out) out[col < d ? col : col - d] = a;
}

template <typename T, int D>
cudaError_t fwd(const QkNormParams& p, cudaStream_t s) {
  constexpr int kHeads = 32 / (D / Vec<T>::kVals), kVec = 4;
  const int one = (p.Hk + kHeads - 1) / kHeads, all = (p.H + kHeads - 1) / kHeads + one * (p.vo ? 2 : 1);
  // a whole token a warp where that fills 16 warps an SM, else fewer steps each
  int64_t parts = ((int64_t)p.sms * 16 + p.n - 1) / p.n;
  if (parts > all) parts = all;
  const int per = (int)((all + parts - 1) / parts);
  parts = (all + per - 1) / per;
  const int64_t want = (p.n * parts + kQnWarps - 1) / kQnWarps, most = (int64_t)p.sms * 6;
  qknorm_fwd_kernel<T, D, kVec><<<(unsigned)(want < most ? want : most), kQnThreads, 0, s>>>(p, (int)parts, per);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t bwd(const QkNormParams& p, cudaStream_t s) {
  const int64_t blocks = qknorm_bwd_blocks(p.n, p.sms);
  if (blocks > 0) {
    qknorm_bwd_kernel<T, D, 2><<<(unsigned)blocks, kQnThreads, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!p.dwq && !p.dwk) return cudaSuccess;
  return launch_next(qknorm_dw_kernel, dim3(2 * D / 32), dim3(512), 0, s, (const float*)p.part, (int)blocks, D, p.dwq,
                     p.dwk);
}

}  // namespace

cudaError_t launch_qknorm_fwd(const QkNormParams& p, bool bf16, cudaStream_t s) {
  if (bf16) return p.d == 64 ? fwd<__nv_bfloat16, 64>(p, s) : fwd<__nv_bfloat16, 128>(p, s);
  return p.d == 64 ? fwd<float, 64>(p, s) : fwd<float, 128>(p, s);
}
cudaError_t launch_qknorm_bwd(const QkNormParams& p, bool bf16, cudaStream_t s) {
  if (bf16) return p.d == 64 ? bwd<__nv_bfloat16, 64>(p, s) : bwd<__nv_bfloat16, 128>(p, s);
  return p.d == 64 ? bwd<float, 64>(p, s) : bwd<float, 128>(p, s);
}

}  // namespace ut
