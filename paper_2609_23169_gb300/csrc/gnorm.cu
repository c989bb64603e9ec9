// Group norm with an activation, channels last, over ragged segments.
//
// Segment s (n rows), group g of C/G channels, M = n C/G values:
//   mu = mean, var = mean of (x - mu)^2,  r = 1 / sqrt(var + eps)
//   xh = (x - mu) r,  u = gamma xh + beta,  y = act(u)
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du xh,
//   a = sum_g gamma du,  b = sum_g gamma du xh,
//   dx = r (gamma du - (a + xh b) / M)
//
// One cooperative launch each way, at most one block per SM.  The segments
// are taken in batches that stay in L2 (kBatchBytes; a longer segment is a
// batch of its own); every block has a contiguous share of the batch's rows.
// It reads its rows once for the statistics (forward) or the sums (backward)
// of each segment's piece in its share; after a grid barrier it merges the
// pieces of its segments and writes its rows, last read first: the last ones
// are still in its shared memory, the others in L2.  So a batch crosses DRAM
// once in each direction, and the bound is DRAM bandwidth; a segment longer
// than L2 is read twice.
//
// Rows move in chunks of kPer rows a thread: a producer warp copies them to a
// ring in shared memory with bulk copies (several chunks in flight whatever
// the other warps do), which in the second pass runs backwards from where the
// first one stopped.  A thread owns one 16-byte column of channels, so any
// number of channels per group works; rows of more than a column a thread are
// taken in slabs.
//
// Statistics are never sums of squares: a window of rows is summed as
// differences from its first row, and the windows' means and squared distances
// merged pairwise,
//   M2 = M2a + M2b + (mean_b - mean_a)^2 na nb / (na + nb),
// so a mean far from zero costs no digits.  All sums are in 32 bits, of a
// window first and of windows then, in an order that the sizes fix.
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"
#include "gnorm.cuh"
#include "kernels.h"
#include "segments.cuh"

namespace ut {

namespace {

// threads that compute; with the producer warp after them a multiple of four warps
// (128 and 168 registers a thread)
constexpr int kFwdThreads = 480, kBwdThreads = 352;
constexpr int kFwdPer = 4, kBwdPer = 2;              // rows of a chunk for each thread
constexpr int kWindow = 16;                          // rows summed before they are merged (forward)
constexpr int kMaxSlots = 16;
constexpr int64_t kBatchBytes = 64ll << 20;          // of the tensors read, per batch
constexpr size_t kSmem = 227 * 1024;

template <typename T>
struct Vec;  // 16 bytes of channels
template <>
struct Vec<float> {
  static constexpr int n = 4;
  UT_DEV static void unpack(const uint4& u, float (&v)[4]) { *reinterpret_cast<uint4*>(v) = u; }
  UT_DEV static uint4 pack(const float (&v)[4]) { return *reinterpret_cast<const uint4*>(v); }
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
  UT_DEV static uint4 pack(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7]));
  }
};

UT_DEV float sigmoid(float u) { return __fdividef(1.f, 1.f + __expf(-u)); }

// A block's threads over a row: `cols` 16-byte columns from col0, `lanes` rows
// at a time.
template <int kThreads>
struct Layout {
  int cols, lanes, col, lane;
  bool on;
  UT_DEV Layout(int cv, int col0) {
    cols = min(cv - col0, kThreads);
    lanes = kThreads / cols;
    col = col0 + threadIdx.x % cols;
    lane = threadIdx.x / cols;
    on = lane < lanes;
  }
  UT_DEV int rows_of(int l, int64_t n) const { return l < n ? (int)((n - l + lanes - 1) / lanes) : 0; }
};

// Segments [s0, s1) with rows [row, row + n): as many whole segments as `most`
// rows hold, at least one.
struct Batch {
  int s0, s1;
  int64_t row, n;
};
UT_DEV Batch batch_from(const GnormParams& p, int s0) {
  Batch b{s0, p.B, 0, 0};
  int64_t row, n;
  segment_rows(p.cu, s0, p.n, row, n);
  b.row = row;
  if (p.n - row <= p.batch_rows || !p.cu) {
    b.n = p.n - row;
    return b;
  }
  int64_t end = row + n;
  b.s1 = s0 + 1;
  while (b.s1 < p.B) {
    segment_rows(p.cu, b.s1, p.n, row, n);
    if (row + n - b.row > p.batch_rows) break;
    end = max(end, row + n);
    ++b.s1;
  }
  b.n = end - b.row;
  return b;
}

// The blocks' shares of a batch: n / blocks rows each, the first n % blocks one more.
struct Shares {
  int64_t row, each;
  int more, blocks;
  UT_DEV Shares(const Batch& b, int blocks_) : row(b.row), blocks(blocks_) {
    each = b.n / blocks;
    more = (int)(b.n - each * blocks);
  }
  UT_DEV int64_t first(int block) const { return row + each * block + min(block, more); }
  // the block that has row r (in range whatever cu holds)
  UT_DEV int owner(int64_t r) const {
    const int64_t at = r - row, big = (each + 1) * more;
    const int64_t c = at < big ? at / (each + 1) : more + (at - big) / (each > 0 ? each : 1);
    return (int)(c < 0 ? 0 : c < blocks ? c : blocks - 1);
  }
};
// The last segment of the batch that starts at or before row r.
UT_DEV int segment_at(const GnormParams& p, const Batch& b, int64_t r) {
  if (!p.cu) return 0;
  int lo = b.s0, hi = b.s1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.cu[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Calls f(segment, first row, end) for the pieces of rows [a, e).
template <typename F>
UT_DEV void for_pieces(const GnormParams& p, const Batch& b, int64_t a, int64_t e, F f) {
  if (a >= e) return;
  for (int s = segment_at(p, b, a); s < b.s1; ++s) {
    int64_t row, n;
    segment_rows(p.cu, s, p.n, row, n);
    const int64_t lo = max(a, row), hi = min(e, row + n);
    if (row >= e) break;
    if (lo < hi) f(s, lo, hi);
  }
}

// The chunks of a block's share of a batch, in the order of the first pass:
// pieces ascending, slabs of columns, rows.
template <int kThreads, int kPer>
struct Chunks {
  int cv, slabs, cols;  // 16-byte columns of a row, slabs, columns of a (full) slab
  int rows;             // of a full chunk
  UT_DEV explicit Chunks(int cv_) {
    cv = cv_;
    cols = min(cv, kThreads);
    slabs = (cv + kThreads - 1) / kThreads;
    rows = kThreads / cols * kPer;
  }
  UT_DEV int slab_cols(int slab) const { return min(cols, cv - slab * kThreads); }
  UT_DEV int64_t row_chunks(int64_t n) const { return (n + rows - 1) / rows; }
  UT_DEV int64_t of_piece(int64_t n) const { return slabs * row_chunks(n); }
};

struct RingState {
  uint64_t full[kMaxSlots], empty[kMaxSlots];
  int abort_flag;
};

// One side's view of the ring: which phase of each slot's barrier is next.
struct Ring {
  RingState* st;
  uint8_t* mem;
  int slots, slot_bytes;
  int32_t* status;
  uint64_t timeout_ns;
  uint32_t full_par, empty_par;  // bit per slot
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
  UT_DEV void wait_empty(int s) {
    mbar_wait(&st->empty[s], ((empty_par >> s) & 1) ^ 1, &st->abort_flag, status, timeout_ns);
    empty_par ^= 1u << s;
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
UT_DEV void load_rows(uint8_t* dst, const void* x, int64_t row_stride, int64_t r, int n, int col, int cols,
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

// Pieces of rows [a, e), last first.
template <typename F>
UT_DEV void for_pieces_back(const GnormParams& p, const Batch& b, int64_t a, int64_t e, F f) {
  if (a >= e) return;
  for (int s = segment_at(p, b, e - 1); s >= b.s0; --s) {
    int64_t row, n;
    segment_rows(p.cu, s, p.n, row, n);
    const int64_t lo = max(a, row), hi = min(e, row + n);
    if (lo < hi) f(s, lo, hi);
    if (row <= a) break;
  }
}

// The producer's part of both passes over a batch: tensors x (and dy).
template <int kThreads, int kPer, int kTensors>
UT_DEV void produce(const GnormParams& p, const Batch& b, int64_t a, int64_t e, const Chunks<kThreads, kPer>& ck,
                    Ring& ring, int64_t total, int elem) {
  auto load = [&](int at, int slab, int64_t r, int n) {
    ring.wait_empty(at);
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
  for_pieces(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
    for (int slab = 0; slab < ck.slabs; ++slab)
      for (int64_t r = lo; r < hi; r += ck.rows, slot = ring.next(slot))
        load(slot, slab, r, (int)min((int64_t)ck.rows, hi - r));
  });
  cooperative_groups::this_grid().sync();
  // backwards; the last `slots` chunks are there
  int64_t i = total - 1;
  slot = ring.before(slot);
  for_pieces_back(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
    const int64_t n = ck.row_chunks(hi - lo);
    for (int slab = ck.slabs - 1; slab >= 0; --slab)
      for (int64_t c = n - 1; c >= 0; --c, --i, slot = ring.before(slot))
        if (total - 1 - i >= ring.slots) {
          const int64_t r = lo + c * ck.rows;
          load(slot, slab, r, (int)min((int64_t)ck.rows, hi - r));
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

// mean, rstd and the affine of a thread's channels
template <int V>
struct Channels {
  float mean[V], rstd[V], gamma[V], beta[V];
  UT_DEV void load(const GnormParams& p, const float2* stat, int c0) {
    const int cpg = p.C / p.G;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const float2 m = stat[(c0 + c) / cpg];
      mean[c] = m.x;
      rstd[c] = m.y;
      gamma[c] = p.gamma ? p.gamma[c0 + c] : 1.f;
      beta[c] = p.beta ? p.beta[c0 + c] : 0.f;
    }
  }
};

// ------------------------------------------------------------------- forward
// Mean and sum of squared distances of a thread's channels; the rows of the
// present window as differences from its first.
template <int V>
struct Moments {
  float mean[V], m2[V], first[V], sum[V], sq[V];
  float cnt, have;
  UT_DEV Moments() : cnt(0.f), have(0.f) {
#pragma unroll
    for (int c = 0; c < V; ++c) mean[c] = m2[c] = first[c] = sum[c] = sq[c] = 0.f;
  }
  UT_DEV void add(const float (&v)[V]) {
    if (have == 0.f) {
#pragma unroll
      for (int c = 0; c < V; ++c) first[c] = v[c];
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const float d = v[c] - first[c];
      sum[c] += d;
      sq[c] = fmaf(d, d, sq[c]);
    }
    have += 1.f;
  }
  UT_DEV void merge() {  // the window into the mean and M2
    if (have == 0.f) return;
    const float tot = cnt + have, wb = have / tot, wm = cnt * wb, inv = 1.f / have;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const float off = sum[c] * inv, q = fmaf(-off, sum[c], sq[c]);
      const float d = first[c] + off - mean[c];
      m2[c] += fmaf(d * d, wm, q > 0.f || q != q ? q : 0.f);
      mean[c] = fmaf(d, wb, mean[c]);
      sum[c] = sq[c] = 0.f;
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
  const int blocks = gridDim.x, me = blockIdx.x, cpg = p.C / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Chunks<kFwdThreads, kFwdPer> ck(p.C / V);
  Ring ring{st, smem + p.ring_at, p.slots, p.slot_bytes, p.status, p.timeout_ns, 0, 0};
  float2* part0 = static_cast<float2*>(p.ws);
  ring_init<kFwdThreads>(st, p.slots);
  if (me == 0 && warp < kFwdThreads / 32) {
    check_cu(p.cu, p.B, p.n, p.status);
    for (int x = threadIdx.x; x < p.B * p.G; x += kFwdThreads) {  // empty segments have no piece
      int64_t row, n;
      segment_rows(p.cu, x / p.G, p.n, row, n);
      if (n == 0) {
        p.mean[x] = 0.f;
        p.rstd[x] = 1.f / sqrtf(p.eps);
      }
    }
  }
  for (int s0 = 0, nb = 0; s0 < p.B; ++nb) {
    const Batch b = batch_from(p, s0);
    s0 = b.s1;
    float2* part = part0 + (int64_t)(nb & 1) * (blocks + p.B) * p.G;  // two batches may be under way
    const Shares sh(b, blocks);
    const int64_t a = sh.first(me), e = sh.first(me + 1);
    int64_t total = 0;  // chunks
    for_pieces(p, b, a, e, [&](int, int64_t lo, int64_t hi) { total += ck.of_piece(hi - lo); });
    if (warp == kFwdThreads / 32) {
      produce<kFwdThreads, kFwdPer, 1>(p, b, a, e, ck, ring, total, sizeof(T));
      continue;
    }
    int64_t i = 0;
    int slot = 0;
    for_pieces(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
      const int64_t n = hi - lo;
      for (int slab = 0; slab < ck.slabs; ++slab) {
        const Layout<kFwdThreads> L(ck.cv, slab * kFwdThreads);
        Moments<V> mo;
        for (int64_t r = 0; r < n; r += ck.rows, ++i, slot = ring.next(slot)) {
          ring.wait_full(slot);
          if (L.on) {
            const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kFwdThreads) * 16;
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k)
              if (r + L.lane + k * L.lanes < n) {
                float v[V];
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(src + k * L.lanes * L.cols * 16), v);
                mo.add(v);
              }
            if (mo.have >= (float)kWindow) mo.merge();
          }
          if (i + ring.slots < total) ring.release(slot);  // else it stays for the second pass
        }
        mo.merge();
        sync_compute<kFwdThreads>();
#pragma unroll
        for (int c = 0; c < V; ++c) lane_stat[c * kFwdThreads + threadIdx.x] = make_float2(mo.mean[c], mo.m2[c]);
        sync_compute<kFwdThreads>();
        for (int ch = threadIdx.x; ch < L.cols * V; ch += kFwdThreads) {
          const float2* ls = lane_stat + (ch % V) * kFwdThreads + ch / V;
          float m = 0.f, q = 0.f;
          for (int l = 0; l < L.lanes; ++l) m = fmaf((float)L.rows_of(l, n), ls[l * L.cols].x, m);
          m /= (float)n;
          for (int l = 0; l < L.lanes; ++l) {
            const float2 t = ls[l * L.cols];
            q += fmaf((float)L.rows_of(l, n) * (t.x - m), t.x - m, t.y);
          }
          chan[slab * kFwdThreads * V + ch] = make_float2(m, q);
        }
      }
      sync_compute<kFwdThreads>();
      for (int g = warp; g < p.G; g += kFwdThreads / 32) {
        float m = 0.f, q = 0.f;
        for (int c = lane; c < cpg; c += 32) m += chan[g * cpg + c].x;
        m = warp_sum(m) / (float)cpg;
        for (int c = lane; c < cpg; c += 32) {
          const float2 t = chan[g * cpg + c];
          q += fmaf((float)n * (t.x - m), t.x - m, t.y);
        }
        q = warp_sum(q);
        if (lane == 0) part[(int64_t)(me + s) * p.G + g] = make_float2(m, q);
      }
    });
    cooperative_groups::this_grid().sync();
    i = total - 1;
    slot = ring.before(slot);
    for_pieces_back(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
      int64_t row, n;
      segment_rows(p.cu, s, p.n, row, n);
      const int c0 = sh.owner(row), c1 = sh.owner(row + n - 1);
      sync_compute<kFwdThreads>();
      for (int g = warp; g < p.G; g += kFwdThreads / 32) {  // the segment's statistics from its pieces'
        auto rows = [&](int c) {
          return (float)(min(sh.first(c + 1), row + n) - max(sh.first(c), row));
        };
        float m = 0.f, q = 0.f;
        for (int c = c0 + lane; c <= c1; c += 32) {
          const float k = rows(c);
          if (k > 0.f) m = fmaf(k, part[(int64_t)(c + s) * p.G + g].x, m);
        }
        m = warp_sum(m) / (float)n;
        for (int c = c0 + lane; c <= c1; c += 32) {
          const float k = rows(c);
          if (k > 0.f) {
            const float2 t = part[(int64_t)(c + s) * p.G + g];
            q += fmaf(k * (float)cpg * (t.x - m), t.x - m, t.y);
          }
        }
        q = warp_sum(q);
        const float r = 1.f / sqrtf(q / ((float)n * (float)cpg) + p.eps);
        if (lane == 0) {
          stat[g] = make_float2(m, r);
          if (me == c0) {
            p.mean[(int64_t)s * p.G + g] = m;
            p.rstd[(int64_t)s * p.G + g] = r;
          }
        }
      }
      sync_compute<kFwdThreads>();
      const int64_t chunks = ck.row_chunks(hi - lo);
      for (int slab = ck.slabs - 1; slab >= 0; --slab) {
        const Layout<kFwdThreads> L(ck.cv, slab * kFwdThreads);
        Channels<V> ch;
        if (L.on) ch.load(p, stat, L.col * V);
#pragma unroll
        for (int c = 0; c < V; ++c) ch.rstd[c] *= ch.gamma[c];
        uint8_t* dst = static_cast<uint8_t*>(p.y) + (int64_t)L.col * 16;
        for (int64_t c = chunks - 1; c >= 0; --c, --i, slot = ring.before(slot)) {
          if (total - 1 - i >= ring.slots) ring.wait_full(slot);
          const int64_t r = lo + c * ck.rows + L.lane;
          if (L.on) {
            const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kFwdThreads) * 16;
#pragma unroll
            for (int k = 0; k < kFwdPer; ++k)
              if (r + k * L.lanes < hi) {
                float v[V];
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(src + k * L.lanes * L.cols * 16), v);
#pragma unroll
                for (int x = 0; x < V; ++x) {
                  const float u = fmaf(v[x] - ch.mean[x], ch.rstd[x], ch.beta[x]);
                  v[x] = kAct ? u * sigmoid(u) : u;
                }
                store_stream(dst + (r + k * L.lanes) * p.ys * (int64_t)sizeof(T), Vec<T>::pack(v));
              }
          }
          ring.release(slot);
        }
      }
    });
  }
}

// ------------------------------------------------------------------ backward
// xh and du of one value
template <bool kAct>
UT_DEV float du_of(float x, float dy, float mean, float rstd, float gamma, float beta, float& xh) {
  xh = (x - mean) * rstd;
  if (!kAct) return dy;
  const float u = fmaf(xh, gamma, beta), s = sigmoid(u);
  return dy * (s * fmaf(u, 1.f - s, 1.f));
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
  float2* coef = stat + p.G;                                                   // [G]: a / M, b / M
  const int blocks = gridDim.x, me = blockIdx.x, cpg = p.C / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Chunks<kBwdThreads, kBwdPer> ck(p.C / V);
  Ring ring{st, smem + p.ring_at, p.slots, p.slot_bytes, p.status, p.timeout_ns, 0, 0};
  float2* part0 = static_cast<float2*>(p.ws);                // [2][blocks + B][G]
  float2* sums = part0 + (int64_t)2 * (blocks + p.B) * p.G;  // [blocks][C]
  ring_init<kBwdThreads>(st, p.slots);
  if (warp < kBwdThreads / 32) {
    if (me == 0) check_cu(p.cu, p.B, p.n, p.status);
    for (int c = threadIdx.x; c < p.C; c += kBwdThreads) all[c] = make_float2(0.f, 0.f);
  }
  auto load_stat = [&](int s) {
    for (int g = threadIdx.x; g < p.G; g += kBwdThreads)
      stat[g] = make_float2(p.mean[(int64_t)s * p.G + g], p.rstd[(int64_t)s * p.G + g]);
  };
  for (int s0 = 0, nb = 0; s0 < p.B; ++nb) {
    const Batch b = batch_from(p, s0);
    s0 = b.s1;
    float2* part = part0 + (int64_t)(nb & 1) * (blocks + p.B) * p.G;
    const Shares sh(b, blocks);
    const int64_t a = sh.first(me), e = sh.first(me + 1);
    int64_t total = 0;  // chunks
    for_pieces(p, b, a, e, [&](int, int64_t lo, int64_t hi) { total += ck.of_piece(hi - lo); });
    if (warp == kBwdThreads / 32) {
      produce<kBwdThreads, kBwdPer, 2>(p, b, a, e, ck, ring, total, sizeof(T));
      continue;
    }
    int64_t i = 0;
    int slot = 0;
    for_pieces(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
      const int64_t n = hi - lo;
      sync_compute<kBwdThreads>();
      load_stat(s);
      sync_compute<kBwdThreads>();
      for (int slab = 0; slab < ck.slabs; ++slab) {
        const Layout<kBwdThreads> L(ck.cv, slab * kBwdThreads);
        float s1[V], s2[V];
#pragma unroll
        for (int c = 0; c < V; ++c) s1[c] = s2[c] = 0.f;
        Channels<V> ch;
        if (L.on) ch.load(p, stat, L.col * V);
        for (int64_t r = 0; r < n; r += ck.rows, ++i, slot = ring.next(slot)) {
          ring.wait_full(slot);
          if (L.on) {
            const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kBwdThreads) * 16;
            float b1[V], b2[V];
#pragma unroll
            for (int c = 0; c < V; ++c) b1[c] = b2[c] = 0.f;
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k)
              if (r + L.lane + k * L.lanes < n) {
                const uint8_t* at = src + k * L.lanes * L.cols * 16;
                float v[V], g[V];
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(at), v);
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(at + ring.slot_bytes / 2), g);
#pragma unroll
                for (int c = 0; c < V; ++c) {
                  float xh;
                  const float du = du_of<kAct>(v[c], g[c], ch.mean[c], ch.rstd[c], ch.gamma[c], ch.beta[c], xh);
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
          if (i + ring.slots < total) ring.release(slot);  // else it stays for the second pass
        }
        sync_compute<kBwdThreads>();
#pragma unroll
        for (int c = 0; c < V; ++c) lane_sum[c * kBwdThreads + threadIdx.x] = make_float2(s1[c], s2[c]);
        sync_compute<kBwdThreads>();
        for (int x = threadIdx.x; x < L.cols * V; x += kBwdThreads) {
          const float2* ls = lane_sum + (x % V) * kBwdThreads + x / V;
          float2 t = make_float2(0.f, 0.f);
          for (int l = 0; l < L.lanes; ++l) {
            t.x += ls[l * L.cols].x;
            t.y += ls[l * L.cols].y;
          }
          const int c = slab * kBwdThreads * V + x;
          chan[c] = t;
          all[c] = make_float2(all[c].x + t.x, all[c].y + t.y);
        }
      }
      sync_compute<kBwdThreads>();
      for (int g = warp; g < p.G; g += kBwdThreads / 32) {
        float2 t = make_float2(0.f, 0.f);
        for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 32) {
          const float w = p.gamma ? p.gamma[c] : 1.f;
          t.x = fmaf(w, chan[c].x, t.x);
          t.y = fmaf(w, chan[c].y, t.y);
        }
        t.x = warp_sum(t.x);
        t.y = warp_sum(t.y);
        if (lane == 0) part[(int64_t)(me + s) * p.G + g] = t;
      }
    });
    if (s0 >= p.B) {  // the last batch: this block's sums over all segments are complete
      sync_compute<kBwdThreads>();
      for (int c = threadIdx.x; c < p.C; c += kBwdThreads) sums[(int64_t)me * p.C + c] = all[c];
    }
    cooperative_groups::this_grid().sync();
    if (s0 >= p.B && (p.dgamma || p.dbeta)) {  // a warp a channel, lanes over the blocks
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
    for_pieces_back(p, b, a, e, [&](int s, int64_t lo, int64_t hi) {
      int64_t row, n;
      segment_rows(p.cu, s, p.n, row, n);
      const int c0 = sh.owner(row), c1 = sh.owner(row + n - 1);
      const float inv = 1.f / ((float)n * (float)cpg);
      sync_compute<kBwdThreads>();
      load_stat(s);
      for (int g = warp; g < p.G; g += kBwdThreads / 32) {
        float2 t = make_float2(0.f, 0.f);
        for (int c = c0 + lane; c <= c1; c += 32)
          if (min(sh.first(c + 1), row + n) > max(sh.first(c), row)) {
            const float2 u = part[(int64_t)(c + s) * p.G + g];
            t.x += u.x;
            t.y += u.y;
          }
        t.x = warp_sum(t.x);
        t.y = warp_sum(t.y);
        if (lane == 0) coef[g] = make_float2(t.x * inv, t.y * inv);
      }
      sync_compute<kBwdThreads>();
      const int64_t chunks = ck.row_chunks(hi - lo);
      for (int slab = ck.slabs - 1; slab >= 0; --slab) {
        const Layout<kBwdThreads> L(ck.cv, slab * kBwdThreads);
        Channels<V> ch;
        float2 ab[V];
        if (L.on) {
          ch.load(p, stat, L.col * V);
#pragma unroll
          for (int x = 0; x < V; ++x) ab[x] = coef[(L.col * V + x) / cpg];
        }
        uint8_t* dst = static_cast<uint8_t*>(p.dx) + (int64_t)L.col * 16;
        for (int64_t c = chunks - 1; c >= 0; --c, --i, slot = ring.before(slot)) {
          if (total - 1 - i >= ring.slots) ring.wait_full(slot);
          const int64_t r = lo + c * ck.rows + L.lane;
          if (L.on) {
            const uint8_t* src = ring.mem + (int64_t)slot * ring.slot_bytes + (L.lane * L.cols + L.col - slab * kBwdThreads) * 16;
#pragma unroll
            for (int k = 0; k < kBwdPer; ++k)
              if (r + k * L.lanes < hi) {
                const uint8_t* at = src + k * L.lanes * L.cols * 16;
                float v[V], g[V];
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(at), v);
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(at + ring.slot_bytes / 2), g);
#pragma unroll
                for (int x = 0; x < V; ++x) {
                  float xh;
                  const float du = du_of<kAct>(v[x], g[x], ch.mean[x], ch.rstd[x], ch.gamma[x], ch.beta[x], xh);
                  v[x] = ch.rstd[x] * (fmaf(ch.gamma[x], du, -ab[x].x) - xh * ab[x].y);
                }
                store_stream(dst + (r + k * L.lanes) * p.dxs * (int64_t)sizeof(T), Vec<T>::pack(v));
              }
          }
          ring.release(slot);
        }
      }
    });
  }
}

// ----------------------------------------------------------------- launchers
// Blocks: one per SM, fewer where a block would have under 8 KB of x.
int blocks_of(const GnormParams& p, int elem) {
  const int64_t want = (p.n * p.C * elem + 8191) / 8192;
  return (int)(want < 1 ? 1 : want > p.sms ? p.sms : want);
}

template <typename F>
cudaError_t launch(F kern, GnormParams p, size_t fixed, int tensors, int threads, int per, int elem, cudaStream_t s) {
  const int cv = p.C * elem / 16, cols = cv < threads ? cv : threads;
  fixed = (fixed + sizeof(RingState) + 8 + 127) & ~(size_t)127;
  p.ring_at = (int)fixed;
  p.slot_bytes = threads / cols * per * cols * 16 * tensors;
  const int slots = (int)((kSmem - fixed) / p.slot_bytes);
  p.slots = slots < kMaxSlots ? slots : kMaxSlots;
  if (p.slots < 1) return cudaErrorInvalidValue;
  p.batch_rows = kBatchBytes / ((int64_t)p.C * elem * tensors);
  const size_t smem = fixed + (size_t)p.slots * p.slot_bytes;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  void* args[] = {&p};
  return cudaLaunchCooperativeKernel(reinterpret_cast<const void*>(kern), dim3(blocks_of(p, elem)), dim3(threads + 32),
                                     args, smem, s);
}

template <typename T>
size_t fixed_smem(const GnormParams& p, bool backward) {
  const size_t n = (size_t)Vec<T>::n * (backward ? kBwdThreads : kFwdThreads) +
                   (backward ? 2 * ((size_t)p.C + p.G) : (size_t)p.C + p.G);
  return n * sizeof(float2);
}

template <typename T>
cudaError_t fwd(const GnormParams& p, cudaStream_t s) {
  const size_t fixed = fixed_smem<T>(p, false);
  return p.act ? launch(gn_fwd_kernel<T, true>, p, fixed, 1, kFwdThreads, kFwdPer, sizeof(T), s)
               : launch(gn_fwd_kernel<T, false>, p, fixed, 1, kFwdThreads, kFwdPer, sizeof(T), s);
}

template <typename T>
cudaError_t bwd(const GnormParams& p, cudaStream_t s) {
  const size_t fixed = fixed_smem<T>(p, true);
  return p.act ? launch(gn_bwd_kernel<T, true>, p, fixed, 2, kBwdThreads, kBwdPer, sizeof(T), s)
               : launch(gn_bwd_kernel<T, false>, p, fixed, 2, kBwdThreads, kBwdPer, sizeof(T), s);
}

}  // namespace

size_t gnorm_ws(const GnormParams& p, bool backward) {
  const size_t part = (size_t)2 * (p.sms + p.B) * p.G * sizeof(float2);
  return part + (backward ? (size_t)p.sms * p.C * sizeof(float2) : 0);
}

cudaError_t launch_gnorm_fwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  return bf16 ? fwd<__nv_bfloat16>(p, s) : fwd<float>(p, s);
}
cudaError_t launch_gnorm_bwd(const GnormParams& p, bool bf16, cudaStream_t s) {
  return bf16 ? bwd<__nv_bfloat16>(p, s) : bwd<float>(p, s);
}

}  // namespace ut
