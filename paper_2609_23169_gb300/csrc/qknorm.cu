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

// what a lane keeps: its pairs and its columns of the weights
template <typename T, int D>
struct Lane {
  static constexpr int kVals = Vec<T>::kVals, kPairs = kVals / 2, kLanes = D / kVals, kHeads = 32 / kLanes;
  uint64_t turn[kPairs];
  uint32_t axis[kPairs];
  float wq[kVals], wk[kVals], cs[kPairs], sn[kPairs];
  int group, col;  // the head of a step, the first of its columns

  UT_DEV void init(const QkNormParams& p, int lane) {
    group = lane / kLanes;
    col = (lane % kLanes) * kVals;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      turn[e] = p.turn[col / 2 + e];
      axis[e] = p.axis[col / 2 + e];
    }
#pragma unroll
    for (int e = 0; e < kVals; ++e) {
      wq[e] = p.wq ? p.wq[col + e] : 1.f;
      wk[e] = p.wk ? p.wk[col + e] : 1.f;
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
};

// The steps of a token: kHeads heads each, of Q, then K, then V.
template <int kHeads>
struct Steps {
  int q, k, all;
  UT_DEV Steps(const QkNormParams& p, bool with_v) {
    q = (p.H + kHeads - 1) / kHeads;
    k = q + (p.Hk + kHeads - 1) / kHeads;
    all = k + (with_v ? (p.Hk + kHeads - 1) / kHeads : 0);
  }
  // head of a lane's group at step s, -1 where there is none
  UT_DEV int head(const QkNormParams& p, int s, int group) const {
    const int h = (s < q ? s : (s < k ? s - q : s - k)) * kHeads + group;
    return h < (s < q ? p.H : p.Hk) ? h : -1;
  }
};

// grid: warps take (token, part of its steps)
template <typename T, int D, int kVec>
__global__ void __launch_bounds__(kQnThreads) qknorm_fwd_kernel(const __grid_constant__ QkNormParams p, int parts,
                                                                int per) {
  using L = Lane<T, D>;
  const int lane = threadIdx.x & 31;
  L me;
  me.init(p, lane);
  const Steps<L::kHeads> st(p, p.vo != nullptr);
  const int64_t warps = (int64_t)gridDim.x * kQnWarps, units = p.n * parts;
  for (int64_t u = (int64_t)blockIdx.x * kQnWarps + (threadIdx.x >> 5); u < units; u += warps) {
    const int64_t row = u / parts;
    const int s0 = (int)(u - row * parts) * per, s1 = min(st.all, s0 + per);
    int64_t to = row;  // of K and V
    bool keep = true;
    if (p.rows) {
      to = p.rows[row];
      keep = to >= 0 && to < p.cache_rows;
      if (to >= p.cache_rows && lane == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    }
    const int32_t pos = p.pos ? p.pos[row] : (int32_t)row;
    bool turned = false;
    for (int s = s0; s < s1; s += kVec) {
      uint4 w[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int x = s + j, h = x < s1 ? st.head(p, x, me.group) : -1;
        w[j] = make_uint4(0, 0, 0, 0);
        if (h < 0) continue;
        const T* src = x < st.q ? static_cast<const T*>(p.q) + row * p.qs
                                : (x < st.k ? static_cast<const T*>(p.k) + row * p.ks
                                            : static_cast<const T*>(p.v) + row * p.vs);
        w[j] = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + me.col);
      }
      if (!turned) me.turn_to(p, pos);  // while the loads fly
      turned = true;
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int x = s + j;
        if (x >= s1) break;  // the same in all lanes
        const int h = st.head(p, x, me.group);
        const bool is_q = x < st.q;
        if (x < st.k) {
          float v[L::kVals], sum = 0.f;
          unpack<T>(w[j], v);
#pragma unroll
          for (int e = 0; e < L::kVals; ++e) sum = fmaf(v[e], v[e], sum);
          const float r = rsqrtf(head_sum<L::kLanes>(sum) * (1.f / D) + p.eps);
#pragma unroll
          for (int e = 0; e < L::kVals; ++e) v[e] *= r * (is_q ? me.wq[e] : me.wk[e]);
#pragma unroll
          for (int e = 0; e < L::kPairs; ++e) {
            const float a = v[2 * e], b = v[2 * e + 1];
            v[2 * e] = fmaf(a, me.cs[e], -b * me.sn[e]);
            v[2 * e + 1] = fmaf(a, me.sn[e], b * me.cs[e]);
          }
          w[j] = pack<T>(v);
        }
        if (h < 0 || !(is_q || keep)) continue;
        T* dst = is_q ? static_cast<T*>(p.qo) + row * p.qos
                      : (x < st.k ? static_cast<T*>(p.ko) + to * p.kos : static_cast<T*>(p.vo) + to * p.vos);
        *reinterpret_cast<uint4*>(dst + (int64_t)h * D + me.col) = w[j];
      }
    }
  }
}

template <typename T, int D, int kVec>
__global__ void __launch_bounds__(kQnThreads) qknorm_bwd_kernel(const __grid_constant__ QkNormParams p) {
  using L = Lane<T, D>;
  __shared__ float sums[kQnWarps * L::kHeads][2][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_next();
  L me;
  me.init(p, lane);
  const Steps<L::kHeads> st(p, false);
  float dwq[L::kVals], dwk[L::kVals];
#pragma unroll
  for (int e = 0; e < L::kVals; ++e) dwq[e] = dwk[e] = 0.f;
  const int64_t warps = (int64_t)gridDim.x * kQnWarps;
  for (int64_t row = (int64_t)blockIdx.x * kQnWarps + warp; row < p.n; row += warps) {
    const int32_t pos = p.pos ? p.pos[row] : (int32_t)row;
    for (int s = 0; s < st.all; s += kVec) {
      uint4 w[kVec], dy[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int x = s + j, h = x < st.all ? st.head(p, x, me.group) : -1;
        w[j] = dy[j] = make_uint4(0, 0, 0, 0);
        if (h < 0) continue;
        const bool is_q = x < st.q;
        const int64_t at = (int64_t)h * D + me.col;
        w[j] = *reinterpret_cast<const uint4*>((is_q ? static_cast<const T*>(p.q) + row * p.qs
                                                     : static_cast<const T*>(p.k) + row * p.ks) + at);
        dy[j] = *reinterpret_cast<const uint4*>((is_q ? static_cast<const T*>(p.dqo) + row * p.dqos
                                                      : static_cast<const T*>(p.dko) + row * p.dkos) + at);
      }
      if (s == 0) me.turn_to(p, pos);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int x = s + j;
        if (x >= st.all) break;
        const int h = st.head(p, x, me.group);
        const bool is_q = x < st.q;
        float v[L::kVals], g[L::kVals], ss = 0.f, sg = 0.f;
        unpack<T>(w[j], v);
        unpack<T>(dy[j], g);
#pragma unroll
        for (int e = 0; e < L::kPairs; ++e) {
          const float a = g[2 * e], b = g[2 * e + 1];
          g[2 * e] = fmaf(a, me.cs[e], b * me.sn[e]);
          g[2 * e + 1] = fmaf(b, me.cs[e], -a * me.sn[e]);
        }
#pragma unroll
        for (int e = 0; e < L::kVals; ++e) {
          ss = fmaf(v[e], v[e], ss);
          sg = fmaf(g[e] * (is_q ? me.wq[e] : me.wk[e]), v[e], sg);
        }
        const float r = rsqrtf(head_sum<L::kLanes>(ss) * (1.f / D) + p.eps);
        const float c = head_sum<L::kLanes>(sg) * (1.f / D) * r * r;  // mean(g w xh) r
#pragma unroll
        for (int e = 0; e < L::kVals; ++e) {
          if (is_q) dwq[e] = fmaf(g[e], v[e] * r, dwq[e]);
          else dwk[e] = fmaf(g[e], v[e] * r, dwk[e]);
          v[e] = r * fmaf(-v[e], c, g[e] * (is_q ? me.wq[e] : me.wk[e]));
        }
        if (h < 0) continue;
        T* dst = is_q ? static_cast<T*>(p.qo) + row * p.qos : static_cast<T*>(p.ko) + row * p.kos;
        *reinterpret_cast<uint4*>(dst + (int64_t)h * D + me.col) = pack<T>(v);
      }
    }
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

// Steps in flight: 6 forward (of 12 for 24 heads of 128 in bf16), 3 backward,
// where a step is two vectors.
template <typename T, int D>
cudaError_t fwd(const QkNormParams& p, cudaStream_t s) {
  constexpr int kHeads = 32 / (D / Vec<T>::kVals), kVec = 6;
  const int one = (p.Hk + kHeads - 1) / kHeads, all = (p.H + kHeads - 1) / kHeads + one * (p.vo ? 2 : 1);
  // a whole token a warp where that fills 16 warps an SM, else fewer steps each
  int64_t parts = ((int64_t)p.sms * 16 + p.n - 1) / p.n;
  if (parts > all) parts = all;
  const int per = (int)((all + parts - 1) / parts);
  parts = (all + per - 1) / per;
  const int64_t want = (p.n * parts + kQnWarps - 1) / kQnWarps, most = (int64_t)p.sms * 8;
  qknorm_fwd_kernel<T, D, kVec><<<(unsigned)(want < most ? want : most), kQnThreads, 0, s>>>(p, (int)parts, per);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t bwd(const QkNormParams& p, cudaStream_t s) {
  const int64_t blocks = qknorm_bwd_blocks(p.n, p.sms);
  if (blocks > 0) {
    qknorm_bwd_kernel<T, D, 3><<<(unsigned)blocks, kQnThreads, 0, s>>>(p);
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
