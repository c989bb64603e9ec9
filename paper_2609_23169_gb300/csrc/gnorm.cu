// Group norm with an activation, channels last, over ragged segments.
//
// Segment s (n rows), group g of C/G channels, M = n C/G values:
//   mu = mean, var = mean of (x - mu)^2,  r = 1 / sqrt(var + eps)
//   xh = (x - mu) r,  u = gamma xh + beta,  y = act(u)
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du xh,
//   a = sum_g gamma du,  b = sum_g gamma du xh,
//   dx = r (gamma du - (a + xh b) / M)
//
// One cooperative launch each way, at most one block per SM; every block has a
// contiguous share of the rows.  It reads its rows once for the statistics
// (forward) or the sums (backward) of each segment's piece in its share; after a
// grid barrier it merges the pieces of its segments and writes its rows, last
// read first: the last ones are still in its shared memory, others in L2.  The
// bound is DRAM bandwidth, with x (and dy) read once and in part twice.  (Batches
// of segments that stay in L2 between the passes were tried: 4 us of barrier and
// merge each and a loop around both passes cost more than the second reads, 225
// us instead of 204 for 6 x 65,536 x 512.)
// Measured: 2048 x 2048 x 128 forward 510 us (two reads and a write at the copy
// rate: 475), backward 815 us (790); 6 x 65,536 x 512 forward 204 us (178),
// backward 324 (297); 85,202 x 640 in 13 segments 61 and 107 us.
//
// Rows move in chunks of kPer rows a thread: a producer warp copies them to a
// ring in shared memory with bulk copies (several chunks in flight whatever
// the other warps do), which in the second pass runs backwards from where the
// first one stopped.  A thread owns one 16-byte column of channels, so any
// number of channels per group works; rows of more than a column a thread are
// taken in slabs (gnorm_rows.cuh).
//
// Statistics are never sums of squares: a window of rows is summed as
// differences from its first row, and the windows' means and squared distances
// merged pairwise,
//   M2 = M2a + M2b + (mean_b - mean_a)^2 na nb / (na + nb),
// so a mean far from zero costs no digits; means are averaged as differences
// from one of them, so that equal values have themselves as their mean.  All
// sums are in 32 bits, of a window first and of windows then, in an order that
// the sizes fix.
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"
#include "gnorm.cuh"
#include "gnorm_rows.cuh"
#include "kernels.h"
#include "pairs.cuh"
#include "segments.cuh"

namespace ut {

namespace {

constexpr int kWindow = 16;                          // rows summed before they are merged (forward)
constexpr int kMaxSlots = 16;
constexpr size_t kFwdSmem = 225 * 1024;              // 128 bytes of static shared memory beside it
constexpr size_t kBwdSmem = 227 * 1024;              // none beside it

template <typename T>
struct Vec;  // 16 bytes of channels as pairs of fp32
template <>
struct Vec<float> {
  static constexpr int n = 4;
  UT_DEV static void unpack(const uint4& u, uint64_t (&v)[2]) {
    v[0] = pack_u32x2(u.x, u.y);
    v[1] = pack_u32x2(u.z, u.w);
  }
  UT_DEV static uint4 pack(const uint64_t (&v)[2]) {
    float a, b, c, d;
    unpack_f32x2(v[0], a, b);
    unpack_f32x2(v[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  UT_DEV static void unpack(const uint4& u, uint64_t (&v)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_u32x2(w[i] << 16, w[i] & 0xFFFF0000u);
  }
  UT_DEV static uint4 pack(const uint64_t (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpack_f32x2(v[i], a, b);
      w[i] = pack_bf16x2(a, b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

UT_DEV uint64_t both(float x) { return pack_f32x2(x, x); }

UT_DEV float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / (1 + exp(-u)) of a pair.  Relative error below 2^-21 + |u| 2^-23 for
// negative u (the product u log2(e) is rounded, and the exponential turns its
// absolute error into a relative one; exponential and reciprocal add 2^-22 and
// 2^-23), below 2^-21 for positive u; 0 where the value is below 2^-126.
// Sharing one reciprocal between the two (1 / a = b / (a b)) takes a third off
// the special function pipe and adds four instructions: no faster forward, 8%
// slower backward.
UT_DEV uint64_t sigmoid2(uint64_t u) {
  float a, b;
  unpack_f32x2(mul_f32x2(u, both(-1.4426950408889634f)), a, b);
  unpack_f32x2(add_f32x2(pack_f32x2(ex2_approx(a), ex2_approx(b)), both(1.f)), a, b);
  return pack_f32x2(rcp_approx(a), rcp_approx(b));
}

// (n, mean, M2) of two sets of values
struct Stat {
  float n, mean, m2;
  UT_DEV void add(float nb, float mb, float qb) {
    if (nb <= 0.f) return;
    // the first set as it is: nb / nb by an approximate reciprocal need not be 1
    const bool first = n == 0.f;
    const float tot = n + nb, w = first ? 1.f : nb * rcp_approx(tot), d = mb - mean, e = first ? 0.f : d;
    m2 += fmaf(e * e, n * w, qb);
    mean = fmaf(d, w, mean);
    n = tot;
  }
};

struct RingState {
  uint64_t full[kMaxSlots], empty[kMaxSlots];
  int abort_flag;
};

// One side's view of the ring: which phase of each slot's barrier is next.  A
// wait that runs out leaves UT_ERR_TIMEOUT in the status word and ends the
// block's waits; the block still meets the others at the grid barriers and
// writes its rows (wrong ones, inside the tensors), the producer loads nothing
// more and sees that what it asked for has landed.
struct Ring {
  RingState* st;
  uint8_t* mem;
  int slots, slot_bytes;
  int32_t* status;
  uint64_t timeout_ns;
  uint32_t full_par, empty_par;  // bit per slot; the producer's full_par: loads asked for
  bool dead;
  UT_DEV int next(int s) const { return s + 1 < slots ? s + 1 : 0; }
  UT_DEV int before(int s) const { return s > 0 ? s - 1 : slots - 1; }
  UT_DEV void wait_full(int s) {
    mbar_wait(&st->full[s], (full_par >> s) & 1, &st->abort_flag, status, timeout_ns);
    full_par ^= 1u << s;
  }
  UT_DEV void release(int s) {  // by every warp that reads
    __syncwarp();
    if (lane_id() == 0) mbar_arrive(&st->empty[s]);
  }
  // producer: waits until the slot's last use is over (a first use waits for nothing)
  UT_DEV bool wait_empty(int s) {
    if (!dead) dead = !warp_wait(&st->empty[s], ((empty_par >> s) & 1) ^ 1, &st->abort_flag, status, timeout_ns);
    empty_par ^= 1u << s;
    return !dead;
  }
  // producer, at the end: its loads into the used slots have landed
  UT_DEV void finish(uint32_t used) {
    if (lane_id() == 0)
      for (int s = 0; s < slots; ++s)
        if ((used >> s) & 1)
          if (!mbar_drain(&st->full[s], ((full_par >> s) & 1) ^ 1, kDrainTimeoutNs)) set_status(status, UT_ERR_TIMEOUT);
  }
};

UT_DEV void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

// Rows [r, r + n) of a slab of 16-byte columns -> shared memory, packed; the
// whole producer warp.
UT_DEV void load_rows(uint8_t* dst, const void* x, int64_t row_stride, int r, int n, int col, int cols,
                      uint64_t* bar) {
  const uint8_t* src = static_cast<const uint8_t*>(x) + r * row_stride + (int64_t)col * 16;
  const uint32_t bytes = (uint32_t)cols * 16;
  if (row_stride == bytes) {
    if (lane_id() == 0) bulk_load(dst, src, bytes * n, bar);
  } else {
    for (int i = lane_id(); i < n; i += 32) bulk_load(dst + (uint32_t)i * bytes, src + i * row_stride, bytes, bar);
  }
}

template <int kThreads>
UT_DEV void sync_compute() {  // the computing warps
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
}

// The producer's part of both passes: tensors x (and dy).
template <int kThreads, int kPer, int kTensors>
UT_DEV void produce(const GnormParams& p, const Pieces& pieces, const Chunks<kThreads, kPer>& ck, Ring& ring,
                    uint32_t& used, int total, int elem) {
  auto load = [&](int at, int slab, int r, int n) {
    if (!ring.wait_empty(at)) return;
    ring.full_par ^= 1u << at;
    used |= 1u << at;
    uint64_t* bar = &ring.st->full[at];
    const int cols = ck.slab_cols(slab);
    if (lane_id() == 0) mbar_expect_tx(bar, (uint32_t)n * cols * 16 * kTensors);
    __syncwarp();
    uint8_t* dst = ring.mem + (int64_t)at * ring.slot_bytes;
    load_rows(dst, p.x, p.xs * elem, r, n, slab * kThreads, cols, bar);
    if (kTensors == 2)
      load_rows(dst + ring.slot_bytes / 2, p.dy, p.dys * elem, r, n, slab * kThreads, cols, bar);
  };
  int slot = 0;
  pieces.forward(p, [&](int s, int lo, int hi) {
    for (int slab = 0; slab < ck.slabs; ++slab)
      for (int r = lo; r < hi; r += ck.rows, slot = ring.next(slot)) load(slot, slab, r, min(ck.rows, hi - r));
  });
  cooperative_groups::this_grid().sync();
  // backwards; the last `slots` chunks are there
  int i = total - 1;
  slot = ring.before(slot);
  pieces.backward(p, [&](int s, int lo, int hi) {
    const int n = ck.row_chunks(hi - lo);
    for (int slab = ck.slabs - 1; slab >= 0; --slab)
      for (int c = n - 1; c >= 0; --c, --i, slot = ring.before(slot))
        if (total - 1 - i >= ring.slots) {
          const int r = lo + c * ck.rows;
          load(slot, slab, r, min(ck.rows, hi - r));
        }
  });
}

template <int kThreads>
UT_DEV void ring_init(RingState* st, int slots) {
  if (threadIdx.x == 0) {
    for (int s = 0; s < slots; ++s) {
      mbar_init(&st->full[s], 1);
      mbar_init(&st->empty[s], kThreads / 32);
    }
    st->abort_flag = 0;
    fence_barrier_init();
  }
  __syncthreads();
}

UT_DEV void store_stream(void* p, const uint4& v) { __stcs(reinterpret_cast<uint4*>(p), v); }

UT_DEV float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// gamma and beta are first read behind the first chunk or the grid barrier:
// fetch them while that is awaited.
UT_DEV void prefetch_affine(const GnormParams& p) {
  for (int c = threadIdx.x * 32; c < p.C; c += blockDim.x * 32) {
    if (p.gamma) asm volatile("prefetch.global.L1 [%0];" ::"l"(p.gamma + c));
    if (p.beta) asm volatile("prefetch.global.L1 [%0];" ::"l"(p.beta + c));
  }
}

// A thread's channels: their groups' values of a [G] table, their affine.
template <int V>
struct Channels {
  uint64_t neg_mean[V / 2], rstd[V / 2], gamma[V / 2], beta[V / 2];
  UT_DEV void load(const GnormParams& p, const float2* stat, int c0) {
    const int cpg = p.C / p.G;
    float w[V], b[V];
    load_or(p.gamma, c0, 1.f, w);
    load_or(p.beta, c0, 0.f, b);
    int g = c0 / cpg, left = cpg - (c0 - g * cpg);  // channels left in group g
#pragma unroll
    for (int c = 0; c < V; c += 2) {
      float2 t[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        t[x] = stat[g];
        if (--left == 0) {
          ++g;
          left = cpg;
        }
      }
      neg_mean[c / 2] = pack_f32x2(-t[0].x, -t[1].x);
      rstd[c / 2] = pack_f32x2(t[0].y, t[1].y);
      gamma[c / 2] = pack_f32x2(w[c], w[c + 1]);
      beta[c / 2] = pack_f32x2(b[c], b[c + 1]);
    }
  }
  UT_DEV static void load_or(const float* src, int c0, float otherwise, float (&v)[V]) {
    if (src) {  // all loads in flight
#pragma unroll
      for (int c = 0; c < V; ++c) v[c] = src[c0 + c];
    } else {
#pragma unroll
      for (int c = 0; c < V; ++c) v[c] = otherwise;
    }
  }
};

// ------------------------------------------------------------------- forward
// Mean and sum of squared distances of a thread's channels; the rows of the
// present window as differences from its first.
template <int V>
struct Moments {
  float mean[V], m2[V];
  uint64_t neg_first[V / 2], sum[V / 2], sq[V / 2];
  float cnt, have;
  UT_DEV Moments() : cnt(0.f), have(0.f) {
#pragma unroll
    for (int c = 0; c < V; ++c) mean[c] = m2[c] = 0.f;
#pragma unroll
    for (int c = 0; c < V / 2; ++c) neg_first[c] = sum[c] = sq[c] = 0;
  }
  UT_DEV void begin(const uint64_t (&v)[V / 2]) {  // the window's first row
#pragma unroll
    for (int c = 0; c < V / 2; ++c) neg_first[c] = mul_f32x2(v[c], both(-1.f));
  }
  UT_DEV void add(const uint64_t (&v)[V / 2]) {
#pragma unroll
    for (int c = 0; c < V / 2; ++c) {
      const uint64_t d = add_f32x2(v[c], neg_first[c]);
      sum[c] = add_f32x2(sum[c], d);
      sq[c] = fma_f32x2(d, d, sq[c]);
    }
  }
  UT_DEV void merge() {  // the window into the mean and M2
    if (have == 0.f) return;
    const float tot = cnt + have, wb = have / tot, wm = cnt * wb, inv = 1.f / have;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      float f[2], s[2], q[2];
      unpack_f32x2(neg_first[i], f[0], f[1]);
      unpack_f32x2(sum[i], s[0], s[1]);
      unpack_f32x2(sq[i], q[0], q[1]);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int c = 2 * i + x;
        const float off = s[x] * inv, m = fmaf(-off, s[x], q[x]), d = off - f[x] - mean[c];
        m2[c] += fmaf(d * d, wm, m > 0.f || m != m ? m : 0.f);
        mean[c] = fmaf(d, wb, mean[c]);
      }
      sum[i] = sq[i] = 0;
    }
    cnt = tot;
    have = 0.f;
  }
};

template <typename T, bool kAct>
__global__ void __launch_bounds__(kFwdThreads + 32, 1) gn_fwd_kernel(const GnormParams p) {
  constexpr int V = Vec<T>::n;
  extern __shared__ __align__(128) uint8_t smem[];
  RingState* st = reinterpret_cast<RingState*>(smem);
  float2* lane_stat = reinterpret_cast<float2*>(smem + sizeof(RingState) + 8);  // [V][threads]
  float2* chan = lane_stat + V * kFwdThreads;                                            // [C]
  float2* stat = chan + p.C;                                                    // [G]: mean, rstd
  __shared__ float warp_rows[kFwdThreads / 32];
  const int blocks = gridDim.x, me = blockIdx.x, cpg = p.C / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float inv_cpg = 1.f / (float)cpg;
  const Chunks<kFwdThreads, kFwdPer> ck(p.C / V);
  prefetch_affine(p);
  Ring ring{st, smem + p.ring_at, p.slots, p.slot_bytes, p.status, p.timeout_ns, 0, 0, false};
  float2* part = static_cast<float2*>(p.ws);  // [blocks + B][G]
  ring_init<kFwdThreads>(st, p.slots);
  if (warp < kFwdThreads / 32) {
    if (me == 0) check_cu(p.cu, p.B, p.n, p.status);
    // empty segments have no piece: 32 segments a warp at a time, a lane each
    constexpr int kStep = kFwdThreads;  // segments of a block
    for (int64_t s0 = (int64_t)me * kStep + warp * 32; s0 < p.B; s0 += (int64_t)blocks * kStep) {
      int64_t row, n = 1;
      if (s0 + lane < p.B) segment_rows(p.cu, (int)s0 + lane, p.n, row, n);
      for (uint32_t none = __ballot_sync(0xffffffffu, n == 0); none; none &= none - 1) {
        const int64_t at = (s0 + __ffs(none) - 1) * p.G;
        for (int g = lane; g < p.G; g += 32) {
          p.mean[at + g] = 0.f;
          p.rstd[at + g] = 1.f / sqrtf(p.eps);
        }
      }
    }
  }
  const Shares sh(p, blocks);
  const Pieces pieces(p, sh.first(me), sh.first(me + 1));
  int total = 0;  // chunks
  pieces.forward(p, [&](int, int lo, int hi) { total += ck.of_piece(hi - lo); });
  if (warp == kFwdThreads / 32) {
    uint32_t used = 0;  // slots loaded
    produce<kFwdThreads, kFwdPer, 1>(p, pieces, ck, ring, used, total, sizeof(T));
    ring.finish(used);
    return;
  }
  int i = 0, slot = 0;
  pieces.forward(p, [&](int s, int lo, int hi) {
    const int n = hi - lo;
    for (int slab = 0; slab < ck.slabs; ++slab) {
      const Layout<kFwdThreads, kFwdPer> L(ck, slab, threadIdx.x);
      Moments<V> mo;
      for (int r = 0; r < n; r += ck.rows, ++i, slot = ring.next(slot)) {
        ring.wait_full(slot);
        if (L.on) {
          const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kFwdThreads) * 16;
          const int step = L.lanes * L.cols * 16;
          uint64_t v[V / 2];
          if (r + ck.rows <= n) {  // a full chunk
            uint4 w[kFwdPer];
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k) w[k] = *reinterpret_cast<const uint4*>(src + k * step);
            if (mo.have == 0.f) {
              Vec<T>::unpack(w[0], v);
              mo.begin(v);
            }
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k) {
              Vec<T>::unpack(w[k], v);
              mo.add(v);
            }
            mo.have += (float)kFwdPer;
          } else {
            for (int k = 0; k < kFwdPer && r + L.lane + k * L.lanes < n; ++k) {
              Vec<T>::unpack(*reinterpret_cast<const uint4*>(src + k * step), v);
              if (mo.have == 0.f) mo.begin(v);
              mo.add(v);
              mo.have += 1.f;
            }
          }
          if (mo.have >= (float)kWindow) mo.merge();
        }
        if (i + ring.slots < total) ring.release(slot);  // else it stays for the second pass
      }
      mo.merge();
      sync_compute<kFwdThreads>();
      // over the lanes of a column, a thread a channel
#pragma unroll
      for (int c = 0; c < V; ++c) lane_stat[c * kFwdThreads + threadIdx.x] = make_float2(mo.mean[c], mo.m2[c]);
      sync_compute<kFwdThreads>();
      const int each = n / L.lanes, more = n - each * L.lanes;  // rows of a lane
      const float inv = 1.f / (float)n;
      for (int x = threadIdx.x; x < L.cols * V; x += kFwdThreads) {
        const int c = x / L.cols, col = x - c * L.cols;
        const float2* ls = lane_stat + c * kFwdThreads + col;
        float m = 0.f, q = 0.f;
#pragma unroll 8
        for (int l = 0; l < L.lanes; ++l) m = fmaf((float)(each + (l < more)), ls[l * L.cols].x - ls[0].x, m);
        m = fmaf(m, inv, ls[0].x);
#pragma unroll 8
        for (int l = 0; l < L.lanes; ++l) {
          const float2 t = ls[l * L.cols];
          q += fmaf((float)(each + (l < more)) * (t.x - m), t.x - m, t.y);
        }
        chan[(slab * kFwdThreads + col) * V + c] = make_float2(m, q);
      }
    }
    sync_compute<kFwdThreads>();
    // over the channels of a group, p.group_lanes threads a group
    for (int g0 = 0; g0 < p.G; g0 += kFwdThreads / p.group_lanes) {
      const int g = g0 + threadIdx.x / p.group_lanes, l = threadIdx.x % p.group_lanes;
      const bool on = g < p.G && threadIdx.x < kFwdThreads / p.group_lanes * p.group_lanes;
      const float2* cs = chan + g * cpg;
      float m = 0.f, q = 0.f;
      if (on)
        for (int c = l; c < cpg; c += p.group_lanes) m += cs[c].x - cs[0].x;
      for (int o = p.group_lanes / 2; o; o >>= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
      if (on) m = fmaf(m, inv_cpg, cs[0].x);
      if (on)
        for (int c = l; c < cpg; c += p.group_lanes) {
          const float2 t = cs[c];
          q += fmaf((float)n * (t.x - m), t.x - m, t.y);
        }
      for (int o = p.group_lanes / 2; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
      if (on && l == 0) part[(int64_t)(me + s) * p.G + g] = make_float2(m, q);
    }
  });
  cooperative_groups::this_grid().sync();
  i = total - 1;
  slot = ring.before(slot);
  pieces.backward(p, [&](int s, int lo, int hi) {
    int row, n;
    rows_of_segment(p, s, row, n);
    const int c0 = sh.owner(row), c1 = sh.owner(row + n - 1);
    sync_compute<kFwdThreads>();
    // the segment's statistics from its pieces': lanes over the groups, warps
    // over the blocks (all of a warp's reads in flight), then one warp over the
    // warps
    for (int g0 = 0; g0 < p.G; g0 += 32) {
      const int g = g0 + lane;
      constexpr int kW = kFwdThreads / 32, kIn = 11;  // 11 x 15 blocks a round
      Stat t{0.f, 0.f, 0.f};
      for (int c = c0 + warp; c <= c1; c += kIn * kW) {
        float2 o[kIn];
#pragma unroll
        for (int x = 0; x < kIn; ++x) {
          const int at = c + x * kW;
          o[x] = at <= c1 && g < p.G ? part[(int64_t)(at + s) * p.G + g] : make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int x = 0; x < kIn; ++x) {
          const int at = c + x * kW;
          if (at <= c1) t.add((float)(min(sh.first(at + 1), row + n) - max(sh.first(at), row)), o[x].x, o[x].y * inv_cpg);
        }
      }
      lane_stat[threadIdx.x] = make_float2(t.mean, t.m2);
      if (lane == 0) warp_rows[warp] = t.n;
      sync_compute<kFwdThreads>();
      if (warp == 0 && g < p.G) {
        const float inv_n = 1.f / (float)n;
        float m = 0.f, q = 0.f;
#pragma unroll
        for (int x = 1; x < kW; ++x) m = fmaf(warp_rows[x], lane_stat[x * 32 + lane].x - t.mean, m);
        m = fmaf(m, inv_n, t.mean);
#pragma unroll
        for (int x = 0; x < kW; ++x) {
          const float2 o = lane_stat[x * 32 + lane];
          q += fmaf(warp_rows[x] * (o.x - m), o.x - m, o.y);
        }
        const float r = 1.f / sqrtf(q * inv_n + p.eps);
        stat[g] = make_float2(m, r);
        if (me == c0) {
          p.mean[(int64_t)s * p.G + g] = m;
          p.rstd[(int64_t)s * p.G + g] = r;
        }
      }
      sync_compute<kFwdThreads>();
    }
    const int chunks = ck.row_chunks(hi - lo);
    for (int slab = ck.slabs - 1; slab >= 0; --slab) {
      const Layout<kFwdThreads, kFwdPer> L(ck, slab, threadIdx.x);
      Channels<V> ch;
      if (L.on) ch.load(p, stat, L.col * V);
      // u = (x - mu) a + beta: with mu folded into beta, a row at its mean would be
      // the difference of two numbers of size |mu| a, which is far from beta where
      // the variance is at or below eps
#pragma unroll
      for (int c = 0; c < V / 2; ++c) ch.rstd[c] = mul_f32x2(ch.rstd[c], ch.gamma[c]);
      auto row_of = [&](const uint4& w) -> uint4 {
        uint64_t v[V / 2];
        Vec<T>::unpack(w, v);
#pragma unroll
        for (int x = 0; x < V / 2; ++x) {
          const uint64_t u = fma_f32x2(add_f32x2(v[x], ch.neg_mean[x]), ch.rstd[x], ch.beta[x]);
          v[x] = kAct ? mul_f32x2(u, sigmoid2(u)) : u;
        }
        return Vec<T>::pack(v);
      };
      uint8_t* dst = static_cast<uint8_t*>(p.y) + (int64_t)L.col * 16;
      for (int c = chunks - 1; c >= 0; --c, --i, slot = ring.before(slot)) {
        if (total - 1 - i >= ring.slots) ring.wait_full(slot);
        const int r = lo + c * ck.rows + L.lane;
        if (L.on) {
          const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kFwdThreads) * 16;
          const int step = L.lanes * L.cols * 16;
          uint8_t* to = dst + (int64_t)r * p.ys * (int64_t)sizeof(T);
          const int64_t to_step = L.lanes * p.ys * (int64_t)sizeof(T);
          if (lo + (c + 1) * ck.rows <= hi) {  // a full chunk
            uint4 w[kFwdPer];
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k) w[k] = *reinterpret_cast<const uint4*>(src + k * step);
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k) store_stream(to + k * to_step, row_of(w[k]));
          } else {
            for (int k = 0; k < kFwdPer && r + k * L.lanes < hi; ++k)
              store_stream(to + k * to_step, row_of(*reinterpret_cast<const uint4*>(src + k * step)));
          }
        }
        ring.release(slot);
      }
    }
  });
}

// ------------------------------------------------------------------ backward
// xh and du of a pair
template <bool kAct>
UT_DEV uint64_t du_of(uint64_t x, uint64_t dy, uint64_t neg_mean, uint64_t rstd, uint64_t gamma, uint64_t beta,
                      uint64_t& xh) {
  xh = mul_f32x2(add_f32x2(x, neg_mean), rstd);
  if (!kAct) return dy;
  const uint64_t u = fma_f32x2(xh, gamma, beta), s = sigmoid2(u);
  // s (1 + u (1 - s)) = s + u s (1 - s)
  const uint64_t us = mul_f32x2(u, s), rest = fma_f32x2(s, both(-1.f), both(1.f));
  return mul_f32x2(dy, fma_f32x2(us, rest, s));
}

template <typename T, bool kAct>
__global__ void __launch_bounds__(kBwdThreads + 32, 1) gn_bwd_kernel(const GnormParams p) {
  constexpr int V = Vec<T>::n;
  extern __shared__ __align__(128) uint8_t smem[];
  RingState* st = reinterpret_cast<RingState*>(smem);
  float2* lane_sum = reinterpret_cast<float2*>(smem + sizeof(RingState) + 8);  // [V][threads]
  float2* chan = lane_sum + V * kBwdThreads;                                            // [C]: this piece's sums
  float2* all = chan + p.C;                                                    // [C]: this block's, over all segments
  float2* stat = all + p.C;                                                    // [G]: mean, rstd
  float2* coef = chan;                                                         // [G], after pass 1: a / M, b / M
  const int blocks = gridDim.x, me = blockIdx.x, cpg = p.C / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Chunks<kBwdThreads, kBwdPer> ck(p.C / V);
  prefetch_affine(p);
  Ring ring{st, smem + p.ring_at, p.slots, p.slot_bytes, p.status, p.timeout_ns, 0, 0, false};
  float2* part = static_cast<float2*>(p.ws);            // [blocks + B][G]
  float2* sums = part + (int64_t)(blocks + p.B) * p.G;  // [blocks][C]
  ring_init<kBwdThreads>(st, p.slots);
  if (warp < kBwdThreads / 32) {
    if (me == 0) check_cu(p.cu, p.B, p.n, p.status);
    for (int c = threadIdx.x; c < p.C; c += kBwdThreads) all[c] = make_float2(0.f, 0.f);
  }
  auto load_stat = [&](int s) {
    for (int g = threadIdx.x; g < p.G; g += kBwdThreads)
      stat[g] = make_float2(p.mean[(int64_t)s * p.G + g], p.rstd[(int64_t)s * p.G + g]);
  };
  const Shares sh(p, blocks);
  const Pieces pieces(p, sh.first(me), sh.first(me + 1));
  int total = 0;  // chunks
  pieces.forward(p, [&](int, int lo, int hi) { total += ck.of_piece(hi - lo); });
  if (warp == kBwdThreads / 32) {
    uint32_t used = 0;  // slots loaded
    produce<kBwdThreads, kBwdPer, 2>(p, pieces, ck, ring, used, total, sizeof(T));
    ring.finish(used);
    return;
  }
  int i = 0, slot = 0;
  pieces.forward(p, [&](int s, int lo, int hi) {
    const int n = hi - lo;
    sync_compute<kBwdThreads>();
    load_stat(s);
    sync_compute<kBwdThreads>();
    for (int slab = 0; slab < ck.slabs; ++slab) {
      const Layout<kBwdThreads, kBwdPer> L(ck, slab, threadIdx.x);
      uint64_t t1[V / 2], t2[V / 2];
#pragma unroll
      for (int c = 0; c < V / 2; ++c) t1[c] = t2[c] = 0;
      Channels<V> ch;
      if (L.on) ch.load(p, stat, L.col * V);
      for (int r = 0; r < n; r += ck.rows, ++i, slot = ring.next(slot)) {
        ring.wait_full(slot);
        if (L.on) {
          const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kBwdThreads) * 16;
          uint64_t b1[V / 2], b2[V / 2];
#pragma unroll
          for (int c = 0; c < V / 2; ++c) b1[c] = b2[c] = 0;
          const int step = L.lanes * L.cols * 16;
          auto row = [&](const uint4& wx, const uint4& wg) {
            uint64_t v[V / 2], g[V / 2];
            Vec<T>::unpack(wx, v);
            Vec<T>::unpack(wg, g);
#pragma unroll
            for (int c = 0; c < V / 2; ++c) {
              uint64_t xh;
              const uint64_t du = du_of<kAct>(v[c], g[c], ch.neg_mean[c], ch.rstd[c], ch.gamma[c], ch.beta[c], xh);
              b1[c] = add_f32x2(b1[c], du);
              b2[c] = fma_f32x2(du, xh, b2[c]);
            }
          };
          if (r + ck.rows <= n) {  // a full chunk
            uint4 wx[kBwdPer], wg[kBwdPer];
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k) {
              wx[k] = *reinterpret_cast<const uint4*>(src + k * step);
              wg[k] = *reinterpret_cast<const uint4*>(src + k * step + ring.slot_bytes / 2);
            }
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k) row(wx[k], wg[k]);
          } else {
#pragma unroll 1
            for (int k = 0; k < kBwdPer && r + L.lane + k * L.lanes < n; ++k)
              row(*reinterpret_cast<const uint4*>(src + k * step),
                  *reinterpret_cast<const uint4*>(src + k * step + ring.slot_bytes / 2));
          }
#pragma unroll
          for (int c = 0; c < V / 2; ++c) {
            t1[c] = add_f32x2(t1[c], b1[c]);
            t2[c] = add_f32x2(t2[c], b2[c]);
          }
        }
        if (i + ring.slots < total) ring.release(slot);  // else it stays for the second pass
      }
      sync_compute<kBwdThreads>();
      float s1[V], s2[V];
#pragma unroll
      for (int c = 0; c < V / 2; ++c) {
        unpack_f32x2(t1[c], s1[2 * c], s1[2 * c + 1]);
        unpack_f32x2(t2[c], s2[2 * c], s2[2 * c + 1]);
      }
      // over the lanes of a column, a thread a channel
#pragma unroll
      for (int c = 0; c < V; ++c) lane_sum[c * kBwdThreads + threadIdx.x] = make_float2(s1[c], s2[c]);
      sync_compute<kBwdThreads>();
      for (int x = threadIdx.x; x < L.cols * V; x += kBwdThreads) {
        const int c = x / L.cols, col = x - c * L.cols;
        const float2* ls = lane_sum + c * kBwdThreads + col;
        float2 t = make_float2(0.f, 0.f);
#pragma unroll 8
        for (int l = 0; l < L.lanes; ++l) {
          const float2 o = ls[l * L.cols];
          t.x += o.x;
          t.y += o.y;
        }
        const int at = (slab * kBwdThreads + col) * V + c;
        chan[at] = t;
        all[at] = make_float2(all[at].x + t.x, all[at].y + t.y);
      }
    }
    sync_compute<kBwdThreads>();
    // over the channels of a group, p.group_lanes threads a group
    for (int g0 = 0; g0 < p.G; g0 += kBwdThreads / p.group_lanes) {
      const int g = g0 + threadIdx.x / p.group_lanes, l = threadIdx.x % p.group_lanes;
      const bool on = g < p.G && threadIdx.x < kBwdThreads / p.group_lanes * p.group_lanes;
      float2 t = make_float2(0.f, 0.f);
      if (on)
        for (int c = g * cpg + l; c < (g + 1) * cpg; c += p.group_lanes) {
          const float w = p.gamma ? p.gamma[c] : 1.f;
          t.x = fmaf(w, chan[c].x, t.x);
          t.y = fmaf(w, chan[c].y, t.y);
        }
      for (int o = p.group_lanes / 2; o; o >>= 1) {
        t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
        t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
      }
      if (on && l == 0) part[(int64_t)(me + s) * p.G + g] = t;
    }
  });
  sync_compute<kBwdThreads>();
  for (int c = threadIdx.x; c < p.C; c += kBwdThreads) sums[(int64_t)me * p.C + c] = all[c];
  cooperative_groups::this_grid().sync();
  if (p.dgamma || p.dbeta) {  // a warp a channel, lanes over the blocks
    for (int c = me + warp * blocks; c < p.C; c += blocks * (kBwdThreads / 32)) {
      float2 t = make_float2(0.f, 0.f);
      for (int x = lane; x < blocks; x += 32) {
        const float2 u = sums[(int64_t)x * p.C + c];
        t.x += u.x;
        t.y += u.y;
      }
      t.x = warp_sum(t.x);
      t.y = warp_sum(t.y);
      if (lane == 0) {
        if (p.dbeta) p.dbeta[c] = t.x;
        if (p.dgamma) p.dgamma[c] = t.y;
      }
    }
  }
  i = total - 1;
  slot = ring.before(slot);
  pieces.backward(p, [&](int s, int lo, int hi) {
    int row, n;
    rows_of_segment(p, s, row, n);
    const int c0 = sh.owner(row), c1 = sh.owner(row + n - 1);
    const float inv = 1.f / ((float)n * (float)cpg);
    sync_compute<kBwdThreads>();
    load_stat(s);
    // the segment's sums from its pieces': lanes over the groups, warps over
    // the blocks, then one warp over the warps
    for (int g0 = 0; g0 < p.G; g0 += 32) {
      const int g = g0 + lane;
      float2 t = make_float2(0.f, 0.f);
      constexpr int kW = kBwdThreads / 32, kIn = 14;  // 14 x 11 blocks a round
      for (int c = c0 + warp; c <= c1; c += kIn * kW) {
        float2 o[kIn];
#pragma unroll
        for (int x = 0; x < kIn; ++x) {
          const int at = c + x * kW;
          const bool there = at <= c1 && g < p.G && min(sh.first(at + 1), row + n) > max(sh.first(at), row);
          o[x] = there ? part[(int64_t)(at + s) * p.G + g] : make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int x = 0; x < kIn; ++x) {
          t.x += o[x].x;
          t.y += o[x].y;
        }
      }
      lane_sum[threadIdx.x] = t;
      sync_compute<kBwdThreads>();
      if (warp == 0 && g < p.G) {
#pragma unroll
        for (int x = 1; x < kW; ++x) {
          const float2 o = lane_sum[x * 32 + lane];
          t.x += o.x;
          t.y += o.y;
        }
        coef[g] = make_float2(t.x * inv, t.y * inv);
      }
      sync_compute<kBwdThreads>();
    }
    const int chunks = ck.row_chunks(hi - lo);
    for (int slab = ck.slabs - 1; slab >= 0; --slab) {
      const Layout<kBwdThreads, kBwdPer> L(ck, slab, threadIdx.x);
      Channels<V> ch;
      Channels<V> ab;  // -a / M and b / M (the affine is not used)
      if (L.on) {
        ch.load(p, stat, L.col * V);
        ab.load(p, coef, L.col * V);
      }
      uint8_t* dst = static_cast<uint8_t*>(p.dx) + (int64_t)L.col * 16;
      for (int c = chunks - 1; c >= 0; --c, --i, slot = ring.before(slot)) {
        if (total - 1 - i >= ring.slots) ring.wait_full(slot);
        const int r = lo + c * ck.rows + L.lane;
        if (L.on) {
          const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kBwdThreads) * 16;
          const int step = L.lanes * L.cols * 16;
          uint8_t* to = dst + (int64_t)r * p.dxs * (int64_t)sizeof(T);
          const int64_t to_step = L.lanes * p.dxs * (int64_t)sizeof(T);
          auto row = [&](const uint4& wx, const uint4& wg) -> uint4 {
            uint64_t v[V / 2], g[V / 2];
            Vec<T>::unpack(wx, v);
            Vec<T>::unpack(wg, g);
#pragma unroll
            for (int x = 0; x < V / 2; ++x) {
              uint64_t xh;
              const uint64_t du = du_of<kAct>(v[x], g[x], ch.neg_mean[x], ch.rstd[x], ch.gamma[x], ch.beta[x], xh);
              const uint64_t t = fma_f32x2(ch.gamma[x], du, ab.neg_mean[x]);
              v[x] = mul_f32x2(ch.rstd[x], fma_f32x2(mul_f32x2(xh, both(-1.f)), ab.rstd[x], t));
            }
            return Vec<T>::pack(v);
          };
          if (lo + (c + 1) * ck.rows <= hi) {  // a full chunk
            uint4 wx[kBwdPer], wg[kBwdPer];
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k) {
              wx[k] = *reinterpret_cast<const uint4*>(src + k * step);
              wg[k] = *reinterpret_cast<const uint4*>(src + k * step + ring.slot_bytes / 2);
            }
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k) store_stream(to + k * to_step, row(wx[k], wg[k]));
          } else {
#pragma unroll 1
            for (int k = 0; k < kBwdPer && r + k * L.lanes < hi; ++k)
              store_stream(to + k * to_step, row(*reinterpret_cast<const uint4*>(src + k * step),
                                                 *reinterpret_cast<const uint4*>(src + k * step + ring.slot_bytes / 2)));
          }
        }
        ring.release(slot);
      }
    }
  });
}

// ----------------------------------------------------------------- launchers
// Blocks: one per SM, fewer where a block would have under 8 KB of x and of the
// segments' statistics.
int blocks_of(const GnormParams& p, int elem) {
  const int64_t x = p.n * p.C * elem, stat = (int64_t)p.B * p.G * 8, want = ((x > stat ? x : stat) + 8191) / 8192;
  return (int)(want < 1 ? 1 : want > p.sms ? p.sms : want);
}

constexpr size_t ring_at(size_t tables) { return (tables + sizeof(RingState) + 8 + 127) & ~(size_t)127; }

// Tables in shared memory in front of the ring, in bytes.  The backward's go
// twice over the channels and once over the groups.
constexpr size_t tables(int vec, int C, int G, bool backward) {
  return sizeof(float2) * ((size_t)vec * (backward ? kBwdThreads : kFwdThreads) + (backward ? 2 : 1) * (size_t)C + G);
}
// Every accepted size leaves at least one slot, the largest tables being those
// of the most channels with the most groups beside them.
constexpr int kMostGroups = kGnMaxBoth - kGnMaxChannels;
static_assert(ring_at(tables(8, kGnMaxChannels, kMostGroups, false)) + kFwdThreads * kFwdPer * 16 <= kFwdSmem, "forward");
static_assert(ring_at(tables(8, kGnMaxChannels, kMostGroups, true)) + kBwdThreads * kBwdPer * 32 <= kBwdSmem, "backward");

template <typename F>
cudaError_t launch(F kern, GnormParams p, bool backward, int elem, cudaStream_t s) {
  const int threads = backward ? kBwdThreads : kFwdThreads, per = backward ? kBwdPer : kFwdPer;
  const int cv = p.C * elem / 16, cols = cv < threads ? cv : threads;
  p.ring_at = (int)ring_at(tables(16 / elem, p.C, p.G, backward));
  p.slot_bytes = threads / cols * per * cols * 16 * (backward ? 2 : 1);
  const int slots = (int)(((backward ? kBwdSmem : kFwdSmem) - p.ring_at) / p.slot_bytes);
  p.slots = slots < kMaxSlots ? slots : kMaxSlots;
  // threads a group of channels is summed by: all groups in one round if they fit
  p.group_lanes = 32;
  while (p.group_lanes > 1 && p.group_lanes * p.G > threads) p.group_lanes /= 2;
  const size_t smem = p.ring_at + (size_t)p.slots * p.slot_bytes;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  void* args[] = {&p};
  return cudaLaunchCooperativeKernel(reinterpret_cast<const void*>(kern), dim3(blocks_of(p, elem)), dim3(threads + 32),
                                     args, smem, s);
}

template <typename T>
cudaError_t fwd(const GnormParams& p, cudaStream_t s) {
  return launch(p.act ? gn_fwd_kernel<T, true> : gn_fwd_kernel<T, false>, p, false, sizeof(T), s);
}

template <typename T>
cudaError_t bwd(const GnormParams& p, cudaStream_t s) {
  return launch(p.act ? gn_bwd_kernel<T, true> : gn_bwd_kernel<T, false>, p, true, sizeof(T), s);
}

}  // namespace

size_t gnorm_ws(const GnormParams& p, bool backward) {
  const size_t part = (size_t)(p.sms + p.B) * p.G * sizeof(float2);
  return part + (backward ? (size_t)p.sms * p.C * sizeof(float2) : 0);
}

cudaError_t launch_gnorm_fwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  return bf16 ? fwd<__nv_bfloat16>(p, s) : fwd<float>(p, s);
}
cudaError_t launch_gnorm_bwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  return bf16 ? bwd<__nv_bfloat16>(p, s) : bwd<float>(p, s);
}

}  // namespace ut
