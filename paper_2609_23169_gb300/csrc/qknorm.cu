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
// is all that sin and cos want: its upper 32 bits are the turn, to 2^-32 and the
// error of the frequency as a double times the coordinate.  Of the 32 bits fp32
// keeps 24: up to 2^-26 turns, as much as sin and cos round near 1.
//
// One warp takes a token; a head's 16-byte vectors lie in neighbouring lanes (8
// to 32 of them), a lane meets the same pairs in every head, so it takes their
// sines once a token, and its columns of w and dw stay in registers.  Where
// whole tokens do not fill the warps evenly, the forward deals out their heads.  What a warp
// reads is asked for up to six steps ahead into shared memory (cp.async), which
// keeps the reads of a warp in flight across tokens without registers: with
// loads into registers, a token's at a time, the 2048 canvas took 359 us.
// Bound by memory: Q and K are read once and written once (backward: x and dy
// read, dx written).  Measured, 24 + 24 heads of 128: 85,714 rows 337 us, 6.24
// TB/s or 0.92 of a copy; 23,959 rows forward 103, backward 145 and dw 9 us.
// dw: a lane's sums over its tokens, then over the block's warps in shared
// memory, then over blocks by a second kernel, always in the same order.
#include <math.h>

#include <type_traits>

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

// The steps of a token: kHeads heads each, of Q, then of K, then of V.
struct Steps {
  int q, k, all;  // where K's begin, V's begin, the end
};
template <int kHeads>
UT_DEV Steps steps_of(const QkNormParams& p, bool with_v) {
  const int q = (p.H + kHeads - 1) / kHeads, k = (p.Hk + kHeads - 1) / kHeads;
  return Steps{q, q + k, q + k + (with_v ? k : 0)};
}

// What a warp reads is asked for kAhead steps before it is used, through shared
// memory, where it costs no registers; each lane reads what it asked for itself.
template <int kSlots>
struct Ahead {
  static constexpr int kAhead = kSlots - 1;  // a slot is filled again a step after it was read
  UT_DEV static void copy(uint4* dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
  }
  UT_DEV static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  template <int kPending>
  UT_DEV static void wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
  }
};

constexpr int kFwdSlots = 8, kBwdSlots = 6;

// Warps take units: a token, or `per` of its steps.
template <typename T, int D>
__global__ void __launch_bounds__(kQnThreads, kQnFwdBlocksPerSm) qknorm_fwd_kernel(const __grid_constant__ QkNormParams p,
                                                                                   int parts, int per) {
  using L = Lane<T, D>;
  using A = Ahead<kFwdSlots>;
  constexpr int kTwo = 2;  // steps at a time
  __shared__ uint4 slots[kQnWarps][kFwdSlots][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  L me;
  me.init(p, lane);
  const Steps st = steps_of<L::kHeads>(p, p.vo != nullptr);
  const int64_t warps = (int64_t)gridDim.x * kQnWarps, units = p.n * parts;
  const int64_t first = (int64_t)blockIdx.x * kQnWarps + warp;
  uint4* const mine = &slots[warp][0][lane];
  int64_t au = first;  // unit and step to ask for next
  int as = 0, aend = 0, at = 0;
  const T *aq = nullptr, *ak = nullptr, *av = nullptr;
  auto begin = [&]() {
    if (au >= units) return;
    const int64_t row = au / parts;
    as = (int)(au - row * parts) * per;
    aend = min(st.all, as + per);
    aq = static_cast<const T*>(p.q) + row * p.qs + me.col;
    ak = static_cast<const T*>(p.k) + row * p.ks + me.col;
    av = static_cast<const T*>(p.v) + row * p.vs + me.col;
  };
  auto ask = [&]() {
    if (au < units) {
      const bool is_q = as < st.q;
      const int h = (is_q ? as : (as < st.k ? as - st.q : as - st.k)) * L::kHeads + me.group;
      const T* src = is_q ? aq : (as < st.k ? ak : av);
      const bool there = h < (is_q ? p.H : p.Hk);
      A::copy(mine + (at & (kFwdSlots - 1)) * 32, there ? src + h * D : src, there);
      if (++as == aend) {
        au += warps;
        begin();
      }
    }
    ++at;
    A::commit();
  };
  begin();
#pragma unroll
  for (int i = 0; i < A::kAhead - 1; ++i) ask();
  auto pos_of = [&](int64_t unit) -> int32_t {
    const int64_t row = unit / parts;
    return p.pos ? p.pos[row] : (int32_t)row;
  };
  int32_t next = first < units ? pos_of(first) : 0;
  int use = 0;  // steps used
  for (int64_t u = first; u < units; u += warps) {
    const int64_t row = u / parts;
    int s = (int)(u - row * parts) * per;
    const int s1 = min(st.all, s + per);
    const int32_t pos = next;
    if (u + warps < units) next = pos_of(u + warps);  // a token ahead
    int64_t to = row;  // of K and V
    bool keep = true;
    if (p.rows) {
      to = p.rows[row];
      keep = to >= 0 && to < p.cache_rows;
      if (to >= p.cache_rows && lane == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    }
    if (s < st.k) me.turn_to(p, pos);
    // one tensor's steps up to `end`: y = R (x r w), or a copy.  With the weights in
    // the rotation (w cos and so on), a pair takes four multiplications and its r.
    auto part = [&](auto norm, T* dst, int heads, int begin, int end, const float* wt) {
      constexpr bool kNorm = decltype(norm)::value;
      if (s >= end) return;
      float wc[L::kVals], ws[L::kVals];
      if constexpr (kNorm) {
        me.weights(wt, wc);
#pragma unroll
        for (int e = 0; e < L::kVals; ++e) {
          ws[e] = wc[e] * me.sn[e / 2];
          wc[e] *= me.cs[e / 2];
        }
      }
      for (; s < end; s += kTwo) {
        const int some = min(kTwo, end - s);
        ask();
        if (some == kTwo) ask();
        A::template wait<A::kAhead - 1>();  // all but the last kAhead - 1 asked for: those of now are there
        uint4 w[kTwo];
#pragma unroll
        for (int j = 0; j < kTwo; ++j) w[j] = mine[((use + j) & (kFwdSlots - 1)) * 32];
        use += some;
#pragma unroll
        for (int j = 0; j < kTwo; ++j) {
          if constexpr (kNorm) {
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
          const int h = (s + j - begin) * L::kHeads + me.group;
          if (dst && j < some && h < heads) *reinterpret_cast<uint4*>(dst + h * D + me.col) = w[j];
        }
      }
      s = end;
    };
    part(std::true_type{}, static_cast<T*>(p.qo) + row * p.qos, p.H, 0, min(s1, st.q), p.wq);
    part(std::true_type{}, keep ? static_cast<T*>(p.ko) + to * p.kos : nullptr, p.Hk, st.q, min(s1, st.k), p.wk);
    part(std::false_type{}, keep && p.vo ? static_cast<T*>(p.vo) + to * p.vos : nullptr, p.Hk, st.k, s1, nullptr);
  }
  A::template wait<0>();
}

template <typename T, int D>
__global__ void __launch_bounds__(kQnThreads, kQnBlocksPerSm) qknorm_bwd_kernel(const __grid_constant__ QkNormParams p) {
  using L = Lane<T, D>;
  using A = Ahead<kBwdSlots>;
  extern __shared__ __align__(16) uint8_t smem[];
  auto& slots = *reinterpret_cast<uint4(*)[kQnWarps][kBwdSlots][2][32]>(smem);
  auto& sums = *reinterpret_cast<float(*)[kQnWarps * L::kHeads][2][D]>(smem);
  static_assert(sizeof(sums) <= sizeof(slots), "the sums take the slots' place");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_next();
  L me;
  me.init(p, lane);
  const Steps st = steps_of<L::kHeads>(p, false);
  float dwq[L::kVals], dwk[L::kVals];
#pragma unroll
  for (int e = 0; e < L::kVals; ++e) dwq[e] = dwk[e] = 0.f;
  const int64_t warps = (int64_t)gridDim.x * kQnWarps, first = (int64_t)blockIdx.x * kQnWarps + warp;
  uint4* const mine = &slots[warp][0][0][lane];
  int64_t arow = first;  // row and step to ask for next
  int as = 0, at = 0;
  auto ask = [&]() {
    if (arow < p.n) {
      const bool is_q = as < st.q;
      const int h = (is_q ? as : as - st.q) * L::kHeads + me.group;
      const bool there = h < (is_q ? p.H : p.Hk);
      const int off = there ? h * D + me.col : me.col;
      const T* x = (is_q ? static_cast<const T*>(p.q) + arow * p.qs : static_cast<const T*>(p.k) + arow * p.ks) + off;
      const T* g = (is_q ? static_cast<const T*>(p.dqo) + arow * p.dqos : static_cast<const T*>(p.dko) + arow * p.dkos) + off;
      A::copy(mine + at * 64, x, there);
      A::copy(mine + at * 64 + 32, g, there);
      if (++as == st.all) {
        as = 0;
        arow += warps;
      }
    }
    at = at + 1 == kBwdSlots ? 0 : at + 1;
    A::commit();
  };
#pragma unroll
  for (int i = 0; i < A::kAhead; ++i) ask();
  auto pos_of = [&](int64_t row) -> int32_t { return p.pos ? p.pos[row] : (int32_t)row; };
  int32_t next = first < p.n ? pos_of(first) : 0;
  int use = 0;
  for (int64_t row = first; row < p.n; row += warps) {
    me.turn_to(p, next);
    if (row + warps < p.n) next = pos_of(row + warps);  // a token ahead
    auto part = [&](T* dst, int heads, const float* wt, float(&dw)[L::kVals]) {
      float wv[L::kVals];
      me.weights(wt, wv);
      for (int h = me.group; h - me.group < heads; h += L::kHeads) {
        A::template wait<A::kAhead - 1>();
        const uint4 w = mine[use * 64], dy = mine[use * 64 + 32];
        use = use + 1 == kBwdSlots ? 0 : use + 1;
        float v[L::kVals], g[L::kVals], ss = 0.f, sg = 0.f;
        unpack<T>(w, v);
        unpack<T>(dy, g);
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
        ask();
        const float r = rsqrtf(head_sum<L::kLanes>(ss) * (1.f / D) + p.eps);
        const float c = head_sum<L::kLanes>(sg) * (1.f / D) * r * r;  // mean(g w xh) r
#pragma unroll
        for (int e = 0; e < L::kVals; ++e) {
          dw[e] = fmaf(t[e], r, dw[e]);
          v[e] = r * fmaf(-v[e], c, g[e] * wv[e]);
        }
        if (h < heads) *reinterpret_cast<uint4*>(dst + h * D + me.col) = pack<T>(v);
      }
    };
    part(static_cast<T*>(p.qo) + row * p.qos, p.H, p.wq, dwq);
    part(static_cast<T*>(p.ko) + row * p.kos, p.Hk, p.wk, dwk);
  }
  A::template wait<0>();
  __syncthreads();
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

// dw = the sum of the blocks' parts; a block 32 columns, 32 threads a column
__global__ void __launch_bounds__(1024) qknorm_dw_kernel(const float* part, int blocks, int d, float* dwq, float* dwk) {
  __shared__ float sums[32][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), i0 = threadIdx.x >> 5;
  grid_wait();
  float a = 0.f;
#pragma unroll 16
  for (int i = i0; i < blocks; i += 32) a += part[(int64_t)i * 2 * d + col];
  sums[i0][threadIdx.x & 31] = a;
  __syncthreads();
  if (i0 > 0) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) a += sums[i][threadIdx.x];
  float* out = col < d ? dwq : dwk;
  if (out) out[col < d ? col : col - d] = a;
}

template <typename T, int D>
cudaError_t fwd(const QkNormParams& p, cudaStream_t s) {
  constexpr int kHeads = 32 / (D / Vec<T>::kVals);
  const int one = (p.Hk + kHeads - 1) / kHeads, all = (p.H + kHeads - 1) / kHeads + one * (p.vo ? 2 : 1);
  // The parts of a token with the least work for the warps that get most: a part
  // takes as long as its steps and about kBegin more (sines, weights).  Instead of
  // whole tokens wherever they make four a warp: 7,781 rows, 24 / 8 / 8 heads of 64
  // in bf16 21 -> 16 us, 2,501 rows, 8 / 4 heads in fp32 14 -> 7.  (The backward
  // gains nothing: 23,959 rows 250 -> 260.)
  constexpr int kBegin = 4;
  const int64_t warps = (int64_t)p.sms * kQnFwdBlocksPerSm * kQnWarps;
  int64_t parts = 1, least = INT64_MAX;
  int per = all;
  for (int x = 1; x <= all && x <= 64; ++x) {
    const int64_t steps = (all + x - 1) / x, some = (all + steps - 1) / steps;
    const int64_t work = (p.n * some + warps - 1) / warps * (steps + kBegin);
    if (work >= least) continue;
    least = work;
    parts = some;
    per = (int)steps;
  }
  const int64_t want = (p.n * parts + kQnWarps - 1) / kQnWarps, most = (int64_t)p.sms * kQnFwdBlocksPerSm;
  qknorm_fwd_kernel<T, D><<<(unsigned)(want < most ? want : most), kQnThreads, 0, s>>>(p, (int)parts, per);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t bwd(const QkNormParams& p, cudaStream_t s) {
  const int64_t blocks = qknorm_bwd_blocks(p.n, p.sms);
  if (blocks > 0) {
    const int smem = kQnWarps * kBwdSlots * 2 * 32 * sizeof(uint4);
    cudaError_t e = cudaFuncSetAttribute(qknorm_bwd_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    qknorm_bwd_kernel<T, D><<<(unsigned)blocks, kQnThreads, smem, s>>>(p);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!p.dwq && !p.dwk) return cudaSuccess;
  return launch_next(qknorm_dw_kernel, dim3(2 * D / 32), dim3(1024), 0, s, (const float*)p.part, (int)blocks, D, p.dwq,
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
