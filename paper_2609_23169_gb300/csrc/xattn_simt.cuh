// Tiles of the CUDA-core attention kernels: 64 x 64 rows and keys, 256 threads
// as 16 x 16, all operands row-major in shared memory with 4 floats of padding.
#pragma once
#include "common.cuh"
#include "pairs.cuh"
#include "xattn.cuh"

namespace ut {

constexpr int kXs = 64;        // rows and keys of a tile
constexpr int kXsThreads = 256;
constexpr int kXsLdP = kXs + 4;

UT_DEV float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }
UT_DEV float4 ld4(const __nv_bfloat16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xFFFF0000u));
}
UT_DEV void st4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
UT_DEV void st4(__nv_bfloat16* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

struct XsTile {  // the query rows of a tile
  int64_t tok0;  // first token
  int rows;      // valid rows
  int head0;     // first query head
  int G;
  UT_DEV int64_t off(int r, int64_t stride, int d) const {
    return (tok0 + r / G) * stride + (int64_t)(head0 + r % G) * d;
  }
};

// dst[64][D + 4] <- the tile's rows of x (zeros past the valid ones)
template <typename T, int D>
UT_DEV void stage_q(float* dst, const void* x, const XsTile& t, int64_t stride) {
  for (int e = threadIdx.x; e < kXs * (D / 4); e += kXsThreads) {
    const int r = e / (D / 4), c = (e % (D / 4)) * 4;
    const float4 v = r < t.rows ? ld4(static_cast<const T*>(x) + t.off(r, stride, D) + c) : make_float4(0, 0, 0, 0);
    st4(dst + r * (D + 4) + c, v);
  }
}
// dst[64][D + 4] <- keys key0 .. of kv head hk (zeros where `on` is 0)
template <typename T, int D>
UT_DEV void stage_k(float* dst, const void* x, int64_t key0, const float* on, int hk, int64_t stride) {
  for (int e = threadIdx.x; e < kXs * (D / 4); e += kXsThreads) {
    const int r = e / (D / 4), c = (e % (D / 4)) * 4;
    const float4 v = on[r] != 0.f ? ld4(static_cast<const T*>(x) + (key0 + r) * stride + (int64_t)hk * D + c)
                                  : make_float4(0, 0, 0, 0);
    st4(dst + r * (D + 4) + c, v);
  }
}
// on[64] <- 1 where the key exists and is not masked; whether any is.  Synchronises the block.
UT_DEV bool stage_mask(float* on, const uint8_t* mask, int64_t key0, int64_t left) {
  const int r = threadIdx.x;
  const bool is = r < kXs && r < left && (!mask || mask[key0 + r]);
  if (r < kXs) on[r] = is ? 1.f : 0.f;
  return __syncthreads_or(is);
}

// acc[i][j] = a[ty * 4 + i] . b[tx + 16 j]
template <int D>
UT_DEV void product_nt(const float* a, const float* b, float (&acc)[4][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  uint64_t sum[4][4];  // of the even and of the odd columns
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[i][j] = 0;
#pragma unroll 4
  for (int e = 0; e < D; e += 4) {
    ulonglong2 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(a + (ty * 4 + i) * (D + 4) + e);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const ulonglong2*>(b + (tx + 16 * j) * (D + 4) + e);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[i][j] = fma_f32x2(x[i].y, y[j].y, fma_f32x2(x[i].x, y[j].x, sum[i][j]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float u, v;
      unpack_f32x2(sum[i][j], u, v);
      acc[i][j] = u + v;
    }
}
// acc[i][c] += sum_k p[ty * 4 + i][k] b[k][tx * 4 + ...]
UT_DEV void axpy4(float w, const ulonglong2& v, float4& acc) {
  const uint64_t ww = pack_f32x2(w, w);
  ulonglong2& a = reinterpret_cast<ulonglong2&>(acc);
  a.x = fma_f32x2(ww, v.x, a.x);
  a.y = fma_f32x2(ww, v.y, a.y);
}
template <int D>
UT_DEV void product_nn(const float* p, const float* b, float4 (&acc)[4][D / 64]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 4
  for (int k = 0; k < kXs; k += 4) {
    float w[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(w[i]) = ld4(p + (ty * 4 + i) * kXsLdP + k);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(b + (k + kk) * (D + 4) + tx * 4 + 64 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) axpy4(w[i][kk], v, acc[i][c]);
      }
  }
}
// acc[i][c] += sum_r p[r][ty * 4 + i] b[r][tx * 4 + ...]
template <int D>
UT_DEV void product_tn(const float* p, const float* b, float4 (&acc)[4][D / 64]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 4
  for (int r = 0; r < kXs; ++r) {
    float w[4];
    *reinterpret_cast<float4*>(w) = ld4(p + r * kXsLdP + ty * 4);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(b + r * (D + 4) + tx * 4 + 64 * c);
#pragma unroll
      for (int i = 0; i < 4; ++i) axpy4(w[i], v, acc[i][c]);
    }
  }
}

UT_DEV float half_warp_max(float x) {
#pragma unroll
  for (int o = 8; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
UT_DEV float half_warp_sum(float x) {
#pragma unroll
  for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// lse / D of the tile's rows (rows that do not exist: LSE = -inf, P = 0)
UT_DEV void stage_rows(float* lse, float* dsum, const XattnParams& p, const XsTile& t) {
  if (threadIdx.x < kXs) {
    const int r = threadIdx.x;
    const int64_t at = (int64_t)(t.head0 + r % p.G) * p.nq + t.tok0 + r / p.G;
    lse[r] = r < t.rows ? p.lse[at] : -INFINITY;
    dsum[r] = r < t.rows ? p.dsum[at] : 0.f;
  }
}

}  // namespace ut
