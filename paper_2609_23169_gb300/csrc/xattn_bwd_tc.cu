// Cross attention to an encoder's states, backward, on the 5th-generation
// tensor cores (bf16 in, fp32 accumulate).  With P = exp(S - LSE) recomputed
// and D_i = dO_i . O_i:
//   dV = P^T dO,   dS = P o (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q
// over the keys of each segment whose mask is set, dK and dV summed over the
// query heads that share the kv head.
//
// A query tile holds 128 rows: the G heads of a kv head of 128 / G consecutive
// tokens of one segment (row = token * G + head).  Keys are few and queries
// many, so a work item is a run of R query tiles of one segment and kv head,
// against ALL the segment's key blocks (128 keys each):
//   for each group of kSub query tiles: for each key block j: for each tile t:
//     S^T  = K_j Q_t^T        (TMEM lanes = keys)
//     dP^T = V_j dO_t^T
//     dV_j += P^T dO_t,  dK_j += dS^T Q_t     (TMEM, over the tiles of the group)
//     dQ_t = dS K_j           (TMEM lanes = query rows)
// so S and dP are computed once per pair, and one CTA sees all key blocks of a
// query tile: its dQ is added up in a buffer of the CTA's own (kSub tiles in
// fp32, 512 KB at d = 128, 78 MB over the device: it stays in L2), first
// block stored, middle ones added, the last one read, added and written as
// bf16, always by the same thread.  No clear, no second pass, no atomic whose
// order changes the result.  A segment of one key block needs no buffer.
// dK_j, dV_j of an item go to partial sums of their own (by the item's place
// in its segment), which a last kernel adds in order.  Both buffers hold
// 16-byte pieces of neighbouring rows side by side, as the threads (a row
// each) write and read them.
//
// Roles (512 threads, registers rebalanced with setmaxnreg):
//   warp 0        TMA: K, V and the Q ring
//   warp 1        TMEM owner and MMA issuer
//   warp 2        zeroes the rows of a Q tile that are not this item's (past
//                 the segment's end, or between the rows of G heads and 128):
//                 what they hold (NaN, infinities) must not enter a sum over rows
//   warp 3        TMA: dO; zeroes its rows likewise, and the masked keys of K
//   warps 4-11    P^T and dS^T as bf16 into shared tiles; dK, dV out
//   warps 12-15   dQ out of TMEM (thread = row)
// TMEM columns: S^T / dP^T [0,128), dQ [128,128+d), dV [256,256+d), dK
// [384,384+d).
// Every wait is bounded; on expiry the kernel records UT_ERR_TIMEOUT, drains
// its own copies and MMAs, frees TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "xattn_tc.cuh"

namespace ut {

namespace {

constexpr int kT = 128;  // rows of a tile, keys of a block
constexpr int kSub = 8;  // query tiles whose dQ a CTA adds up at a time
constexpr int kThreads = 512;
constexpr int kRegLaunch = 128, kRegCtl = 80, kRegEw = 160, kRegDrain = 112;
static_assert(kRegCtl + 2 * kRegEw + kRegDrain == 4 * kRegLaunch, "setmaxnreg split must match the launch");
constexpr uint32_t kChunkB = 128 * 128;  // 128 rows x 64 bf16
constexpr int kQStages = 2;
constexpr uint32_t kColDq = 128, kColDv = 256, kColDk = 384;

template <int D>
struct BwdSmem {
  static constexpr int kC = D / 64;
  static constexpr uint32_t kTile = kT * D * 2;
  alignas(1024) uint8_t k[kTile];
  alignas(1024) uint8_t v[kTile];
  alignas(1024) uint8_t pt[2 * kChunkB];
  alignas(1024) uint8_t dst[2 * kChunkB];
  alignas(1024) uint8_t q[kQStages][kTile];
  alignas(1024) uint8_t dout[kTile];
  alignas(16) float lse2[2][kT];
  alignas(16) float dsum[2][kT];
  uint64_t kv_full, kv_ready, kv_empty, do_full, do_ready, do_empty;
  uint64_t q_full[kQStages], q_ready[kQStages], q_empty[kQStages], rows_full[2];
  uint64_t s_full, s_empty, dp_full, dp_empty, pt_full, pt_done, dst_full, ds_done, dq_empty;
  uint64_t acc_full, acc_empty, mma_done;
  uint32_t tmem_base;
  int abort_flag;
};

struct BwdParams {
  XattnParams x;
  uint32_t inv_g;   // ceil(2^16 / G)
  int tpt;          // tokens of a tile
  int R;            // tiles of an item
  int64_t slots;    // items along the query rows
  int64_t n_items;
  float scale_log2;
  int64_t kslots;   // key blocks of all segments (with idle ones): nk / 128 + n_seg
  bool wide;        // dq takes 32-byte stores
  float* dq_acc;    // [grid, kSub, d / 4, 128, 4]
};

struct Work {  // one item
  int hk, part, tiles, blocks;
  int64_t tok0, key0;
  int ntok, keys;  // tokens and keys of the item
  int64_t kslot;   // first key block's place among all segments'
};

// Item u; false where its slot is idle.
UT_DEV bool decode(const BwdParams& b, int64_t u, Work& w) {
  const XattnParams& p = b.x;
  w.hk = (int)(u % p.Hk);
  const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, b.R * b.tpt, u / p.Hk);
  const int64_t t0 = g.tile * b.R * b.tpt;
  if (t0 >= g.n) return false;
  int64_t k0, kn;
  segment_rows(p.cu_k, g.s, p.nk, k0, kn);
  w.part = (int)g.tile;
  w.tok0 = g.row + t0;
  w.ntok = (int)min((int64_t)b.R * b.tpt, g.n - t0);
  w.tiles = (w.ntok + b.tpt - 1) / b.tpt;
  w.key0 = k0;
  w.kslot = k0 / kT + g.s;
  w.keys = (int)kn;
  w.blocks = (int)((kn + kT - 1) / kT);
  return true;
}

UT_DEV void red_add4(float* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(a)), "f"(__uint_as_float(b)),
               "f"(__uint_as_float(c)), "f"(__uint_as_float(d))
               : "memory");
}
// a whole 32-byte sector (a pair of 16-byte stores would write it in halves)
UT_DEV void st_v8(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
UT_DEV float4 ld_l2(const float* p) {
  float4 v;
  asm volatile("ld.relaxed.gpu.global.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "l"(p)
               : "memory");
  return v;
}
UT_DEV void tmem_ld64(uint32_t taddr, uint32_t* r) {
  tmem_ld32(taddr, *reinterpret_cast<uint32_t(*)[32]>(r));
  tmem_ld32(taddr + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
  tmem_wait_ld();
}
// zero rows [first, 128) of a tile of `chunks` 128-byte-row sub-tiles; whole warp
UT_DEV void zero_tail(uint32_t base, int chunks, int first, uint32_t lane) {
  for (int r = first + (int)(lane >> 3); r < kT; r += 4)
    for (int c = 0; c < chunks; ++c) st_shared_v4(base + c * kChunkB + r * 128 + ((lane & 7) << 4), 0, 0, 0, 0);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    xattn_bwd_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                        const BwdParams prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = BwdSmem<D>;
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const XattnParams& p = prm.x;
  const uint32_t warp = warp_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    return;
  }
  if (threadIdx.x == 0) {
    uint64_t* one[] = {&sm.kv_full, &sm.kv_ready, &sm.kv_empty, &sm.do_full, &sm.do_ready, &sm.do_empty, &sm.s_full,
                       &sm.dp_full, &sm.pt_done, &sm.ds_done, &sm.acc_full, &sm.mma_done};
    for (uint64_t* b : one) mbar_init(b, 1);
    for (int s = 0; s < kQStages; ++s) {
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_ready[s], 1);
      mbar_init(&sm.q_empty[s], 1);
    }
    uint64_t* eight[] = {&sm.s_empty, &sm.dp_empty, &sm.pt_full, &sm.dst_full, &sm.acc_empty};
    for (uint64_t* b : eight) mbar_init(b, 8);
    mbar_init(&sm.dq_empty, 4);
    mbar_init(&sm.rows_full[0], 256);
    mbar_init(&sm.rows_full[1], 256);
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // all 512 columns are this CTA's, so they start at address 0
  if (sm.tmem_base != 0 && threadIdx.x == 0) {
    set_status(p.status, UT_ERR_CUDA);
    sm.abort_flag = 1;
  }
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // whole warp, converged
    return warp_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto wait1 = [&](uint64_t* bar, uint32_t parity) {  // one thread
    return mbar_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto drain = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_drain(bar, parity, kDrainTimeoutNs)) set_status(p.status, UT_ERR_TIMEOUT);
  };
  // tiles that dQ is added up for at a time
  auto group_of = [&](const Work& w) { return w.blocks > 1 ? kSub : w.tiles; };

  const uint32_t wg = warp >> 2;
  if (wg == 0) {
    setmaxnreg_dec<kRegCtl>();
    if (warp == 0) {
      if (lane == 0) {
        const uint64_t first_pol = policy_evict_first(), keep = policy_evict_last();
        const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kC;
        uint32_t nkv = 0, nt = 0;
        bool ok = true;
        for (int64_t u = blockIdx.x; u < prm.n_items && ok; u += gridDim.x) {
          Work w;
          if (!decode(prm, u, w)) continue;
          const int step = group_of(w);
          for (int s0 = 0; s0 < w.tiles && ok; s0 += step)
            for (int j = 0; j < w.blocks && ok; ++j) {
              if (!(ok = wait1(&sm.kv_empty, (nkv & 1) ^ 1))) break;
              mbar_expect_tx(&sm.kv_full, 2 * S::kTile);
              for (int c = 0; c < S::kC; ++c) {
                tma_load_3d(sm.k + c * kChunkB, &tm_k, &sm.kv_full, c * 64, w.hk, (int)w.key0 + j * kT, keep);
                tma_load_3d(sm.v + c * kChunkB, &tm_v, &sm.kv_full, c * 64, w.hk, (int)w.key0 + j * kT, keep);
              }
              ++nkv;
              // the last block's pass over a tile is the last reader of its rows
              const uint64_t pol = j == w.blocks - 1 ? first_pol : keep;
              for (int t = s0; t < min(s0 + step, w.tiles); ++t, ++nt) {
                const uint32_t st = nt % kQStages;
                if (!(ok = wait1(&sm.q_empty[st], ((nt / kQStages) & 1) ^ 1))) break;
                mbar_expect_tx(&sm.q_full[st], bytes);
                for (int c = 0; c < S::kC; ++c)
                  tma_load_3d(sm.q[st] + c * kChunkB, &tm_q, &sm.q_full[st], c * 64, w.hk * p.G,
                              (int)w.tok0 + t * prm.tpt, pol);
              }
            }
        }
        if (nkv > 0) drain(&sm.kv_full, (nkv - 1) & 1);
        for (uint32_t x = nt > kQStages ? nt - kQStages : 0; x < nt; ++x)
          drain(&sm.q_full[x % kQStages], (x / kQStages) & 1);
      }
    } else if (warp == 1) {
      constexpr uint32_t idesc_s = idesc_bf16_f32(kT, kT, false, false);
      constexpr uint32_t idesc_acc = idesc_bf16_f32(kT, D, false, true);
      constexpr uint32_t idesc_dq = idesc_bf16_f32(kT, D, true, true);
      const uint32_t k_lo = desc_lo(smem_u32(sm.k), 16), v_lo = desc_lo(smem_u32(sm.v), 16),
                     q_lo = desc_lo(smem_u32(sm.q[0]), 16), do_lo = desc_lo(smem_u32(sm.dout), 16),
                     pt_lo = desc_lo(smem_u32(sm.pt), 16), dst_lo = desc_lo(smem_u32(sm.dst), 16);
      // the same tiles read along their rows (MN-major operands)
      const uint32_t k_mn = desc_lo(smem_u32(sm.k), kChunkB), q_mn = desc_lo(smem_u32(sm.q[0]), kChunkB),
                     do_mn = desc_lo(smem_u32(sm.dout), kChunkB), dst_mn = desc_lo(smem_u32(sm.dst), kChunkB);
      uint32_t nkv = 0, nt = 0;
      bool ok = true;
      for (int64_t u = blockIdx.x; u < prm.n_items && ok; u += gridDim.x) {
        Work w;
        if (!warp_uniform(decode(prm, u, w))) continue;
        const int tiles = (int)warp_uniform((uint32_t)w.tiles), blocks = (int)warp_uniform((uint32_t)w.blocks);
        const int step = blocks > 1 ? kSub : tiles;
        for (int s0 = 0; s0 < tiles && ok; s0 += step)
          for (int j = 0; j < blocks && ok; ++j) {
            const int L = min(step, tiles - s0);
            if (!(ok = wait(&sm.kv_ready, nkv & 1))) break;
            auto issue_st = [&](uint32_t x) -> bool {  // S^T of tile number x
              const uint32_t st = x % kQStages;
              if (!wait(&sm.q_ready[st], (x / kQStages) & 1)) return false;
              if (!wait(&sm.dp_empty, (x & 1) ^ 1)) return false;
              tc_fence_after();
              mma_nt<D>(0, k_lo, q_lo + st * (S::kTile >> 4), idesc_s);
              mma_commit_w(&sm.s_full);
              return true;
            };
            if (!(ok = issue_st(nt))) break;
#pragma unroll 1
            for (int t = 0; t < L; ++t, ++nt) {
              const uint32_t par = nt & 1, qst = nt % kQStages;
              // dP^T once S^T has been read
              if (!(ok = wait(&sm.do_ready, par))) break;
              if (!(ok = wait(&sm.s_empty, par))) break;
              tc_fence_after();
              mma_nt<D>(0, v_lo, do_lo, idesc_s);
              mma_commit_w(&sm.dp_full);
              // dV += P^T dO
              if (!(ok = wait(&sm.pt_full, par))) break;
              if (t == 0 && !(ok = wait(&sm.acc_empty, (nkv & 1) ^ 1))) break;
              tc_fence_after();
              mma_nn128(kColDv, pt_lo, do_mn, idesc_acc, t > 0);
              mma_commit_w(&sm.pt_done);
              mma_commit_w(&sm.do_empty);
              // S^T of the next tile once dP^T has been read
              if (t + 1 < L && !(ok = issue_st(nt + 1))) break;
              // dK += dS^T Q
              if (!(ok = wait(&sm.dst_full, par))) break;
              tc_fence_after();
              mma_nn128(kColDk, dst_lo, q_mn + qst * (S::kTile >> 4), idesc_acc, t > 0);
              mma_commit_w(&sm.q_empty[qst]);
              // dQ = dS K once the previous one has been read
              if (!(ok = wait(&sm.dq_empty, par ^ 1))) break;
              tc_fence_after();
              mma_tt128(kColDq, dst_mn, k_mn, idesc_dq);
              mma_commit_w(&sm.ds_done);
            }
            if (!ok) break;
            mma_commit_w(&sm.kv_empty);
            mma_commit_w(&sm.acc_full);
            ++nkv;
          }
      }
      mma_commit_w(&sm.mma_done);
      drain(&sm.mma_done, 0);
    } else {
      // ------------- rows that must read as zero (warp 2: Q, warp 3: dO, K); dO loads
      const bool is_q = warp == 2;
      const uint32_t kv_base = smem_u32(sm.k), bytes = (uint32_t)prm.tpt * p.G * 128 * S::kC;
      const uint64_t first_pol = policy_evict_first(), keep = policy_evict_last();
      uint32_t nkv = 0, nt = 0;
      bool ok = true;
      for (int64_t u = blockIdx.x; u < prm.n_items && ok; u += gridDim.x) {
        Work w;
        if (!decode(prm, u, w)) continue;
        const int step = group_of(w);
        for (int s0 = 0; s0 < w.tiles && ok; s0 += step)
          for (int j = 0; j < w.blocks && ok; ++j) {
            for (int t = s0; t < min(s0 + step, w.tiles); ++t, ++nt) {
              if (!is_q) {
                if (!(ok = wait(&sm.do_empty, (nt & 1) ^ 1))) break;
                if (lane == 0) {
                  mbar_expect_tx(&sm.do_full, bytes);
                  for (int c = 0; c < S::kC; ++c)
                    tma_load_3d(sm.dout + c * kChunkB, &tm_do, &sm.do_full, c * 64, w.hk * p.G,
                                (int)w.tok0 + t * prm.tpt, j == w.blocks - 1 ? first_pol : keep);
                }
                __syncwarp();
                if (t == s0) {
                  const uint32_t keys = lane_keys(p.mask, w.key0 + j * kT, w.keys - j * kT, lane);
                  if (!(ok = wait(&sm.kv_full, nkv & 1))) break;
                  if (__any_sync(0xffffffffu, keys != 15u)) {
                    for (int g = 0; g < 4; ++g)
                      if (!((keys >> g) & 1u))
                        for (int x = 0; x < 8 * S::kC; ++x)
                          st_shared_v4(kv_base + (x >> 3) * kChunkB + (lane + 32 * g) * 128 + (((x + lane) & 7) << 4),
                                       0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                  }
                  if (lane == 0) mbar_arrive(&sm.kv_ready);
                  ++nkv;
                }
              }
              const int rows = min(prm.tpt, w.ntok - t * prm.tpt) * p.G;
              const uint32_t st = is_q ? nt % kQStages : 0, f = is_q ? nt / kQStages : nt;
              if (!(ok = wait(is_q ? &sm.q_full[st] : &sm.do_full, f & 1))) break;
              if (rows < kT) {
                zero_tail(smem_u32(is_q ? sm.q[st] : sm.dout), S::kC, rows, lane);
                fence_proxy_async_smem();
                __syncwarp();
              }
              if (lane == 0) mbar_arrive(is_q ? &sm.q_ready[st] : &sm.do_ready);
            }
          }
      }
      if (!is_q) {  // every copy it issued has landed (the last may not have been waited for on an abort)
        const bool fine = __all_sync(0xffffffffu, ok);
        if (!fine && lane == 0 && nt > 0) drain(&sm.do_full, (nt - 1) & 1);
      }
    }
  } else if (wg < 3) {
    setmaxnreg_inc<kRegEw>();
    // warps w and w + 4 share the 32 keys of a TMEM lane quarter and split the
    // 128 query columns (and the d output columns) into halves
    const uint32_t quarter = warp & 3, half = (warp - 4) >> 2;
    const uint32_t krow = quarter * 32 + lane, tid = threadIdx.x - 128;
    const uint32_t lane_base = (quarter * 32) << 16;
    constexpr int HC = kT / 2, HD = D / 2;
    const float c = prm.scale_log2;
    const uint32_t pt_row = smem_u32(sm.pt) + half * kChunkB + krow * 128;
    const uint32_t dst_row = smem_u32(sm.dst) + half * kChunkB + krow * 128;
    const int col = (int)(tid & (kT - 1)), rt = (int)(((uint32_t)col * prm.inv_g) >> 16), rg = col - rt * p.G;
    uint32_t nt = 0, ng = 0;
    bool ok = true;
    for (int64_t u = blockIdx.x; u < prm.n_items && ok; u += gridDim.x) {
      Work w;
      if (!decode(prm, u, w)) continue;
      const int step = group_of(w);
      // this thread's query column: LSE (threads 0-127) or D (128-255), a tile ahead
      const float* vec = (tid < kT ? p.lse : p.dsum) + (int64_t)(w.hk * p.G + rg) * p.nq + w.tok0 + rt;
      auto row_value = [&](int t) -> float {
        const bool there = rt < min(prm.tpt, w.ntok - t * prm.tpt);
        if (tid >= kT) return there ? vec[t * prm.tpt] : 0.f;
        const float l = there ? vec[t * prm.tpt] : -INFINITY;
        return l == -INFINITY ? INFINITY : l * kLog2e;  // no such row, or a row without keys: P = 0
      };
      for (int s0 = 0; s0 < w.tiles && ok; s0 += step)
        for (int j = 0; j < w.blocks && ok; ++j, ++ng) {
          const int key = j * kT + (int)krow, L = min(step, w.tiles - s0);
          // P and dS of a masked key are zero: as a mask of the packed pairs
          const uint32_t on = key < w.keys && (!p.mask || p.mask[w.key0 + key]) ? 0xffffffffu : 0u;
          float rv = row_value(s0);
          for (int t = 0; t < L; ++t, ++nt) {
            const uint32_t par = nt & 1;
            if (tid < kT) sm.lse2[par][col] = rv;
            else sm.dsum[par][col] = rv;
            mbar_arrive(&sm.rows_full[par]);
            if (t + 1 < L) rv = row_value(s0 + t + 1);
            if (!(ok = wait(&sm.rows_full[par], (nt >> 1) & 1))) break;
            const float* ls = sm.lse2[par] + half * HC;
            const float* dv = sm.dsum[par] + half * HC;
            if (!(ok = wait(&sm.s_full, par))) break;
            tc_fence_after();
            float pr[HC];
            {
              uint32_t r[HC];
              tmem_ld64(lane_base + half * HC, r);
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sm.s_empty);
#pragma unroll
              for (int x = 0; x < HC; x += 4) {
                const float4 l4 = *reinterpret_cast<const float4*>(ls + x);
                pr[x + 0] = ex2_approx(fmaf(__uint_as_float(r[x + 0]), c, -l4.x));
                pr[x + 1] = ex2_approx(fmaf(__uint_as_float(r[x + 1]), c, -l4.y));
                pr[x + 2] = ex2_approx(fmaf(__uint_as_float(r[x + 2]), c, -l4.z));
                pr[x + 3] = ex2_approx(fmaf(__uint_as_float(r[x + 3]), c, -l4.w));
              }
            }
            if (!(ok = wait(&sm.pt_done, par ^ 1))) break;  // the previous dV has read the P^T tile
#pragma unroll
            for (int x = 0; x < HC / 8; ++x)
              st_shared_v4(pt_row + ((x ^ (krow & 7)) << 4), pack_bf16x2(pr[8 * x], pr[8 * x + 1]) & on,
                           pack_bf16x2(pr[8 * x + 2], pr[8 * x + 3]) & on,
                           pack_bf16x2(pr[8 * x + 4], pr[8 * x + 5]) & on,
                           pack_bf16x2(pr[8 * x + 6], pr[8 * x + 7]) & on);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.pt_full);
            if (!(ok = wait(&sm.dp_full, par))) break;
            tc_fence_after();
            uint32_t r[HC];
            tmem_ld64(lane_base + half * HC, r);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.dp_empty);  // S^T of the next tile may be computed
#pragma unroll
            for (int x = 0; x < HC; x += 4) {
              const float4 d4 = *reinterpret_cast<const float4*>(dv + x);
              r[x / 2] = pack_bf16x2(pr[x] * (__uint_as_float(r[x]) - d4.x),
                                     pr[x + 1] * (__uint_as_float(r[x + 1]) - d4.y)) & on;
              r[x / 2 + 1] = pack_bf16x2(pr[x + 2] * (__uint_as_float(r[x + 2]) - d4.z),
                                         pr[x + 3] * (__uint_as_float(r[x + 3]) - d4.w)) & on;
            }
            if (!(ok = wait(&sm.ds_done, par ^ 1))) break;  // the previous dK and dQ have read the dS^T tile
#pragma unroll
            for (int x = 0; x < HC / 8; ++x)
              st_shared_v4(dst_row + ((x ^ (krow & 7)) << 4), r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.dst_full);
          }
          if (!ok) break;
          // dV, dK of the group: stored by the item's first group, added by the others
          if (!(ok = wait(&sm.acc_full, ng & 1))) break;
          tc_fence_after();
          const int64_t at = ((((int64_t)w.part * prm.kslots + w.kslot + j) * p.Hk + w.hk) * (D / 4) + half * (HD / 4)) * kT + krow;
#pragma unroll
          for (int which = 0; which < 2; ++which) {
            float* dst = (which ? p.part_dk : p.part_dv) + at * 4;
#pragma unroll
            for (int g = 0; g < HD / 32; ++g) {
              uint32_t r[32];
              tmem_ld32(lane_base + (which ? kColDk : kColDv) + half * HD + g * 32, r);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                float* at4 = dst + (g * 8 + x) * kT * 4;
                if (s0 == 0) *reinterpret_cast<uint4*>(at4) = make_uint4(r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
                else red_add4(at4, r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.acc_empty);
        }
    }
  } else {
    setmaxnreg_dec<kRegDrain>();
    // dQ: TMEM lane = query row, column = d
    const uint32_t quarter = warp & 3, row = quarter * 32 + lane, lane_base = (quarter * 32) << 16;
    const int rt = (int)((row * prm.inv_g) >> 16);
    const int64_t row_off = (int64_t)rt * p.dqs + (int)(row - rt * p.G) * D;
    // the CTA's buffer: 16-byte pieces, [tile][d / 4][row]
    float* acc = prm.dq_acc + ((int64_t)blockIdx.x * kSub * (D / 4) * kT + row) * 4;
    uint32_t nt = 0;
    bool ok = true;
    for (int64_t u = blockIdx.x; u < prm.n_items && ok; u += gridDim.x) {
      Work w;
      if (!decode(prm, u, w)) continue;
      const int step = group_of(w);
      __nv_bfloat16* out0 = static_cast<__nv_bfloat16*>(p.dq) + w.tok0 * p.dqs + (int64_t)w.hk * p.G * D + row_off;
      if (w.blocks == 0) {  // no keys: dQ = 0
        for (int t = 0; t < w.tiles; ++t)
          if (rt < min(prm.tpt, w.ntok - t * prm.tpt))
            for (int x = 0; x < D; x += 8)
              *reinterpret_cast<uint4*>(out0 + (int64_t)t * prm.tpt * p.dqs + x) = make_uint4(0, 0, 0, 0);
        continue;
      }
      for (int s0 = 0; s0 < w.tiles && ok; s0 += step)
        for (int j = 0; j < w.blocks && ok; ++j) {
          const bool last = j == w.blocks - 1, add = j > 0;
          for (int t = s0; t < min(s0 + step, w.tiles); ++t, ++nt) {
            float* a = acc + (int64_t)(t - s0) * (D / 4) * kT * 4;
            const bool there = rt < min(prm.tpt, w.ntok - t * prm.tpt);
            __nv_bfloat16* out = out0 + (int64_t)t * prm.tpt * p.dqs;
            float4 pre[16];  // the sum so far, 64 columns at a time, the first before the wait
            if (last && add) {
#pragma unroll
              for (int x = 0; x < 16; ++x) pre[x] = ld_l2(a + x * kT * 4);
            }
            if (!(ok = wait(&sm.ds_done, nt & 1))) break;
            tc_fence_after();
#pragma unroll
            for (int g = 0; g < D / 16; ++g) {
              uint32_t r[16];
              tmem_ld16(lane_base + kColDq + g * 16, r);
              tmem_wait_ld();
              if (g == D / 16 - 1) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.dq_empty);
              }
              float* ag = a + g * 4 * kT * 4;
              if (!last) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  if (add) red_add4(ag + x * kT * 4, r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
                  else
                    *reinterpret_cast<uint4*>(ag + x * kT * 4) =
                        make_uint4(r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
                }
                continue;
              }
              float v[16];
#pragma unroll
              for (int x = 0; x < 16; ++x) v[x] = __uint_as_float(r[x]);
              if (add) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  const float4 f = pre[(g & 3) * 4 + x];
                  v[4 * x] += f.x;
                  v[4 * x + 1] += f.y;
                  v[4 * x + 2] += f.z;
                  v[4 * x + 3] += f.w;
                  if (g + 4 < D / 16) pre[(g & 3) * 4 + x] = ld_l2(ag + (16 + x) * kT * 4);
                }
              }
              if (there) {
                uint32_t o[8];
#pragma unroll
                for (int y = 0; y < 8; ++y) o[y] = pack_bf16x2(v[2 * y] * p.scale, v[2 * y + 1] * p.scale);
                if (prm.wide) {
                  st_v8(out + g * 16, o);
                } else {
                  *reinterpret_cast<uint4*>(out + g * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                  *reinterpret_cast<uint4*>(out + g * 16 + 8) = make_uint4(o[4], o[5], o[6], o[7]);
                }
              }
            }
          }
        }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(sm.tmem_base, 512);
}

// dK, dV: the sum of the partials of the key's segment, in order.  grid (key
// slots, kv heads, dK / dV), a block one key block: read 16 bytes a thread
// along the keys, written as rows through shared memory.
template <int D>
__global__ void __launch_bounds__(256) xattn_bwd_join_kernel(const BwdParams prm) {
  __shared__ __align__(16) uint8_t rows[kT * (D * 2 + 16)];
  const XattnParams& p = prm.x;
  const Segment g = segment_of_slot(p.cu_k, p.B, p.nk, kT, blockIdx.x);
  const int keys = (int)min((int64_t)kT, g.n - g.tile * kT);
  if (keys <= 0) return;
  int64_t row, nq;
  segment_rows(p.cu_q, g.s, p.nq, row, nq);
  const int64_t tiles = (nq + prm.tpt - 1) / prm.tpt;
  const int parts = (int)((tiles + prm.R - 1) / prm.R);
  const int64_t kslot = min(g.row / kT + g.s + g.tile, prm.kslots - 1);
  const bool is_k = blockIdx.z == 0;
  const float* src = (is_k ? p.part_dk : p.part_dv) + (kslot * p.Hk + blockIdx.y) * (D * kT);
  const int64_t step = prm.kslots * p.Hk * (D * kT);
  const float f = is_k ? p.scale : 1.f;
  for (int x = threadIdx.x; x < D / 4 * kT; x += 256) {
    float4 a = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
      const float4 b = *reinterpret_cast<const float4*>(src + i * step + x * 4);
      a.x += b.x;
      a.y += b.y;
      a.z += b.z;
      a.w += b.w;
    }
    *reinterpret_cast<uint2*>(rows + (x % kT) * (D * 2 + 16) + (x / kT) * 8) =
        make_uint2(pack_bf16x2(a.x * f, a.y * f), pack_bf16x2(a.z * f, a.w * f));
  }
  __syncthreads();
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(is_k ? p.dk : p.dv) + (int64_t)blockIdx.y * D;
  const int64_t stride = is_k ? p.dks : p.dvs;
  for (int x = threadIdx.x; x < keys * (D / 8); x += 256) {
    const int r = x / (D / 8), e = x % (D / 8);
    *reinterpret_cast<uint4*>(out + (g.row + g.tile * kT + r) * stride + e * 8) =
        *reinterpret_cast<const uint4*>(rows + r * (D * 2 + 16) + e * 16);
  }
}

static_assert(sizeof(BwdSmem<128>) <= 232448, "shared layout exceeds the block limit");

template <int D>
cudaError_t launch_d(const BwdParams& prm, const CUtensorMap* tm, cudaStream_t s) {
  const size_t smem = sizeof(BwdSmem<D>);
  cudaError_t e = cudaFuncSetAttribute(xattn_bwd_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // the setmaxnreg split assumes exactly kRegLaunch registers per thread at
  // launch: with fewer, the increases would wait for registers that never come
  cudaFuncAttributes fa;
  e = cudaFuncGetAttributes(&fa, xattn_bwd_tc_kernel<D>);
  if (e != cudaSuccess) return e;
  if (fa.numRegs != kRegLaunch) return cudaErrorInvalidConfiguration;
  const int grid = (int)(prm.n_items < prm.x.sms ? prm.n_items : prm.x.sms);
  xattn_bwd_tc_kernel<D><<<grid, kThreads, smem, s>>>(tm[0], tm[1], tm[2], tm[3], prm);
  return cudaGetLastError();
}

// Tiles of an item: the smallest number of whole waves of CTAs (up to four)
// that keeps them busy to within 8% of the best, so that the partial sums stay
// few; more tiles where the partial sums would pass 1 GB.
int tiles_per_item(const XattnParams& p) {
  const int64_t tpt = kT / p.G, tiles = (p.nq + tpt - 1) / tpt;
  int64_t best = 1;
  double best_use = 0.0;
  for (int waves = 1; waves <= 4; ++waves) {
    const int64_t runs = (int64_t)waves * p.sms / p.Hk;  // items along the rows
    if (runs < 1) continue;
    const int64_t R = (tiles + runs - 1) / runs, items = (tiles + R - 1) / R * p.Hk;
    const int64_t w = (items + p.sms - 1) / p.sms;
    const double use = (double)(tiles * p.Hk) / ((double)(w * p.sms) * R);
    if (use > best_use + 0.08) {
      best_use = use;
      best = R;
    }
  }
  if (best_use == 0.0) best = tiles;  // more kv heads than four waves
  const int64_t part = 2 * segment_slots(p.nk, p.B, kT) * kT * p.Hk * p.d * (int64_t)sizeof(float);
  const int64_t most = ((int64_t)1 << 30) / (part > 0 ? part : 1);
  const int64_t least = most > 0 ? (tiles + most - 1) / most : tiles;
  if (best < least) best = least;
  return (int)(best < 1 ? 1 : best);
}

// one of the two partial sums: [parts of a segment, key slots, kv heads, d / 4, 128, 4]
size_t part_bytes(const XattnParams& p, int R) {
  const int64_t tpt = kT / p.G, tiles = (p.nq + tpt - 1) / tpt;
  return (size_t)((tiles + R - 1) / R) * segment_slots(p.nk, p.B, kT) * p.Hk * p.d * kT * sizeof(float);
}

}  // namespace

int64_t xattn_bwd_tc_items(const XattnParams& p) {
  return segment_slots(p.nq, p.B, tiles_per_item(p) * (kT / p.G)) * p.Hk;
}

// partial dK, dV; the CTAs' dQ buffers
size_t xattn_bwd_tc_ws(const XattnParams& p) {
  return 2 * part_bytes(p, tiles_per_item(p)) + (size_t)p.sms * kSub * kT * p.d * sizeof(float);
}

cudaError_t launch_xattn_bwd_tc(const XattnParams& p, void* ws, cudaStream_t s) {
  BwdParams prm{};
  prm.x = p;
  prm.inv_g = (65536u + p.G - 1) / p.G;
  prm.tpt = kT / p.G;
  prm.R = tiles_per_item(p);
  const size_t part = part_bytes(p, prm.R);
  prm.kslots = segment_slots(p.nk, p.B, kT);
  prm.wide = (reinterpret_cast<uintptr_t>(p.dq) & 31u) == 0 && (p.dqs * 2) % 32 == 0;
  prm.x.part_dk = static_cast<float*>(ws);
  prm.x.part_dv = reinterpret_cast<float*>(static_cast<char*>(ws) + part);
  prm.dq_acc = reinterpret_cast<float*>(static_cast<char*>(ws) + 2 * part);
  prm.slots = segment_slots(p.nq, p.B, prm.R * prm.tpt);
  prm.n_items = prm.slots * p.Hk;
  prm.scale_log2 = p.scale * kLog2e;
  cudaError_t e = cudaSuccess;
  if (p.nq > 0) {
    // without keys the K and V maps are never used
    const void* k = p.nk > 0 ? p.k : p.q;
    const void* v = p.nk > 0 ? p.v : p.q;
    const int64_t ks = p.nk > 0 ? p.ks : p.qs, vs = p.nk > 0 ? p.vs : p.qs, nk = p.nk > 0 ? p.nk : 1;
    CUtensorMap tm[4];
    if (!encode_tmap_heads_bf16(&tm[0], p.q, p.d, p.H, p.nq, p.qs * 2, p.G, prm.tpt) ||
        !encode_tmap_heads_bf16(&tm[1], k, p.d, p.Hk, nk, ks * 2, 1, kT) ||
        !encode_tmap_heads_bf16(&tm[2], v, p.d, p.Hk, nk, vs * 2, 1, kT) ||
        !encode_tmap_heads_bf16(&tm[3], p.dout, p.d, p.H, p.nq, p.dos * 2, p.G, prm.tpt))
      return cudaErrorInvalidValue;
    e = p.d == 64 ? launch_d<64>(prm, tm, s) : launch_d<128>(prm, tm, s);
    if (e != cudaSuccess) return e;
  }
  if (p.nk > 0) {
    const dim3 grid((unsigned)prm.kslots, p.Hk, 2);
    if (p.d == 64) xattn_bwd_join_kernel<64><<<grid, 256, 0, s>>>(prm);
    else xattn_bwd_join_kernel<128><<<grid, 256, 0, s>>>(prm);
    e = cudaGetLastError();
  }
  return e;
}

}  // namespace ut
