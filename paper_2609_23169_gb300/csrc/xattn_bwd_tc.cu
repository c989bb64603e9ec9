// Cross attention to an encoder's states, backward, on the 5th-generation
// tensor cores (bf16 in, fp32 accumulate).  With P = exp(S - LSE) recomputed
// and D_i = dO_i . O_i:
//   dV = P^T dO,   dS = P o (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q
// over the keys of each segment whose mask is set, dK and dV summed over the
// query heads that share the kv head.
//
// A query tile holds 128 rows: the G heads of a kv head of 128 / G consecutive
// tokens of one segment (row = token * G + head); a key block 128 keys.
//
// Two kernels, S and dP computed in each:
//   xattn_dq_kernel    a query tile over its segment's key blocks j:
//       S = Q K_j^T,  dP = dO V_j^T  ->  dS over S in TMEM,  dQ += dS K_j
//     dQ stays in TMEM until it is whole: no partial sums, no atomics.
//   xattn_dkdv_kernel  a key block over a run of R query tiles t:
//       S^T = K Q_t^T -> P^T over it,  dV += P^T dO_t
//       dP^T = V dO_t^T -> dS^T over it,  dK += dS^T Q_t
//     A run's dK, dV go to partial sums of their own, which a last kernel adds
//     in order.
// That is seven products of 128 x 128 x d a pair of tiles against five of a
// fused kernel.  The fused form was built first: its dQ parts, 64 KB of fp32 a
// pair, have to be added up through L2, and its P^T and dS^T pass through
// shared memory; it took 9,100 cycles a pair at 23,959 x 512 x 24 x 128 where
// the products need 2,560.  Here P and dS never leave TMEM (they are the A
// operands of the second products, written over the first ones' results), and
// the elementwise work of one tile runs beside the products of the next:
// 2,700 and 2,700 cycles a pair where the products need 1,536 and 2,048.
// Measured at that size: D 44 us (6.6 TB/s), dQ 172, dK and dV 191, their sum
// 14: 417 us a pass, 904 TFLOP/s of the five products.  dQ is bound by the
// elementwise warps and by shared memory (S and dP read both operands there,
// tensor pipe active 59%), dK and dV by shared memory (tensor pipe 72%).
//
// Roles of both kernels (registers rebalanced with setmaxnreg): warp 1 owns
// TMEM and issues the products, warps 0, 2, 3 load (TMA) and zero the rows
// that must not enter a sum over rows (masked keys, rows of other segments:
// what they hold, NaN or infinities, is never multiplied), warps 4-11 are the
// elementwise stage: warps w and w + 4 share 32 TMEM lanes and take 64 columns
// each, and write their bf16 pairs over the first half of their own columns.
// Every wait is bounded; on expiry a kernel records UT_ERR_TIMEOUT, drains its
// own copies and MMAs, frees TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "xattn_tc.cuh"

namespace ut {

namespace {

constexpr int kT = 128;  // rows of a tile, keys of a block
constexpr uint32_t kChunkB = 128 * 128;  // 128 rows x 64 bf16

struct BwdParams {
  XattnParams x;
  uint32_t inv_g;   // ceil(2^16 / G)
  int tpt;          // tokens of a tile
  int R;            // tiles of a run
  int ks;           // items of a run: item c has its key blocks c, c + ks, ...
  int64_t n_items;  // of the launch
  float scale_log2;
  int64_t kslots;   // key blocks of all segments (with idle ones): nk / 128 + n_seg
};

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

// =========================================================================
//                                   dQ
// =========================================================================
// TMEM columns: S_j / dS_j [0,128) and [256,384) in turn, dP [128,256), dQ
// [384,384+d).  With dS_i formed, the tensor core is given dP_{i+1}, dQ_i and
// S_{i+2}, across items: the elementwise warps find their next S there and
// take its exponentials while dP runs.
//   warp 0      TMA, in the order of their use: Q, K_0, V_0, dO, K_1, V_1, ...
//   warp 1      the products
//   warp 2      decodes the items into a ring, 32 at once, one a lane (one after
//               another each took 2,500 cycles, more than a block)
//   warp 3      zeroes the masked keys of K and V, says when a block has all it
//               needs
//   warps 12-15 dQ out
// kFew, where a segment may have one block of keys (several segments, or 128 keys
// in all): dS is rounded to bf16 for its product, as dQ is at the end, together
// 1.42 times the error of rounding dQ alone; with few keys the error of D = dO .
// O, whose O was rounded too, adds to that in dQ and dK (1.66 times at 10 keys,
// 1.50 at 62, 1.45 from 110).  So in such a segment D is taken anew, as the sum
// of P dP in fp32, and left for the next kernel; which form a segment gets does
// not depend on the others.  A form of its own because its code costs long
// segments up to 6% of a backward pass (23,959 rows and 13 segments of 257 keys at d =
// 64: 290 -> 309 us; 85,202 and 13 of 512 at d = 128: 1,836 -> 1,840 us).
// The issuing warp's instructions are fetched anew every block (the
// elementwise code lies between), and it bounded the first form: 700 of them a
// block, 3,900 cycles.  So it counts stages instead of dividing, follows one
// cursor, whose flags the later products take over, waits for two barriers a
// block, and calls the part of a wait that spins.
constexpr int kDqThreads = 512;
constexpr int kDqLaunch = 128, kDqCtl = 80, kDqEw = 152, kDqOut = 128;
static_assert(kDqCtl + 2 * kDqEw + kDqOut <= 4 * kDqLaunch, "setmaxnreg split must fit the launch");
constexpr int kDqSlots = 8, kDqReaders = 15;

struct DqItem {
  int32_t blocks;  // key blocks; 0: no more items
  int32_t hk;      // kv head
  int32_t tok0, ntok;
  int32_t key0, keys;
};

template <int D>
struct DqSmem {
  static constexpr int kC = D / 64;
  static constexpr uint32_t kTile = kT * D * 2;
  static constexpr int kQ = D == 128 ? 1 : 2, kK = D == 128 ? 3 : 4, kV = D == 128 ? 2 : 4;
  alignas(1024) uint8_t q[kQ][kTile];
  alignas(1024) uint8_t dout[kQ][kTile];
  alignas(1024) uint8_t k[kK][kTile];
  alignas(1024) uint8_t v[kV][kTile];
  uint64_t q_full[kQ], q_empty[kQ], do_full[kQ], do_empty[kQ];
  uint64_t k_full[kK], ready[kK], k_empty[kK], v_full[kV], dp_full[kV];  // dP done: V is free
  uint64_t s_full[2], ds_full[2], dq_full, dq_empty, mma_done;
  uint64_t pair_full[4];    // kFew: the two warps of 32 rows have their parts of D
  float pair[2][2][kT];
  uint64_t item_full[kDqSlots], item_empty[kDqSlots];
  DqItem item[kDqSlots];
  uint32_t tmem_base;
  int abort_flag;
};

template <int D, bool kFew>
__global__ void __launch_bounds__(kDqThreads, 1)
    xattn_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                    const BwdParams prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = DqSmem<D>;
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const XattnParams& p = prm.x;
  const uint32_t warp = warp_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    return;
  }
  if (threadIdx.x == 0) {
    uint64_t* one[] = {&sm.s_full[0], &sm.s_full[1], &sm.dq_full, &sm.mma_done};
    for (uint64_t* x : one) mbar_init(x, 1);
    for (int s = 0; s < S::kQ; ++s) {
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_empty[s], 1);
      mbar_init(&sm.do_full[s], 1);
      mbar_init(&sm.do_empty[s], 1);
    }
    for (int s = 0; s < S::kK; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.ready[s], 1);
      mbar_init(&sm.k_empty[s], 1);
    }
    for (int s = 0; s < S::kV; ++s) {
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.dp_full[s], 1);
    }
    mbar_init(&sm.ds_full[0], 8);
    mbar_init(&sm.ds_full[1], 8);
    mbar_init(&sm.dq_empty, 4);
    for (int s = 0; s < 4; ++s) mbar_init(&sm.pair_full[s], 2);
    for (int s = 0; s < kDqSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], kDqReaders);
    }
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  grid_next();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_wait();
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
  // The next item; false at the end or on an abort (then ok = false).
  auto next_item = [&](uint32_t& n, DqItem& it, bool& ok) -> bool {
    const uint32_t s = n % kDqSlots;
    ok = wait(&sm.item_full[s], (n / kDqSlots) & 1);
    if (!ok) return false;
    it = sm.item[s];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.item_empty[s]);
    ++n;
    return it.blocks > 0;
  };

  if (warp < 4) {
    setmaxnreg_dec<kDqCtl>();
    if (warp == 0 && lane == 0) {
      // --------------------------------------------------- items and loads
      tma_prefetch_desc(&tm_q);
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
      tma_prefetch_desc(&tm_do);
      const uint64_t keep = policy_evict_last();
      const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kC;
      uint32_t n = 0, at = 0, nv = 0, ndo = 0;  // items, K, V and dO tiles asked for
      bool ok = true;
      for (;;) {
        const uint32_t slot = n % kDqSlots;
        if (!(ok = wait1(&sm.item_full[slot], (n / kDqSlots) & 1))) break;
        const DqItem it = sm.item[slot];
        mbar_arrive(&sm.item_empty[slot]);
        if (it.blocks == 0) break;
        const uint32_t qs = n % S::kQ, qf = (n / S::kQ) & 1;
        if (!(ok = wait1(&sm.q_empty[qs], qf ^ 1))) break;
        mbar_expect_tx(&sm.q_full[qs], bytes);
        for (int c = 0; c < S::kC; ++c)
          tma_load_3d(sm.q[qs] + c * kChunkB, &tm_q, &sm.q_full[qs], c * 64, it.hk * p.G, it.tok0, keep);
        ++n;
        for (int j = 0; j < it.blocks; ++j) {
          const uint32_t ks = at % S::kK, vs = nv % S::kV;
          if (!(ok = wait1(&sm.k_empty[ks], ((at / S::kK) & 1) ^ 1))) break;
          mbar_expect_tx(&sm.k_full[ks], S::kTile);
          for (int c = 0; c < S::kC; ++c)
            tma_load_3d(sm.k[ks] + c * kChunkB, &tm_k, &sm.k_full[ks], c * 64, it.hk, it.key0 + j * kT, keep);
          ++at;
          if (!(ok = wait1(&sm.dp_full[vs], ((nv / S::kV) & 1) ^ 1))) break;
          mbar_expect_tx(&sm.v_full[vs], S::kTile);
          for (int c = 0; c < S::kC; ++c)
            tma_load_3d(sm.v[vs] + c * kChunkB, &tm_v, &sm.v_full[vs], c * 64, it.hk, it.key0 + j * kT, keep);
          ++nv;
          if (j > 0) continue;
          if (!(ok = wait1(&sm.do_empty[qs], qf ^ 1))) break;
          mbar_expect_tx(&sm.do_full[qs], bytes);
          for (int c = 0; c < S::kC; ++c)
            tma_load_3d(sm.dout[qs] + c * kChunkB, &tm_do, &sm.do_full[qs], c * 64, it.hk * p.G, it.tok0, keep);
          ++ndo;
        }
        if (!ok) break;
      }
      auto landed = [&](uint64_t* bar, uint32_t stages, uint32_t sent) {
        for (uint32_t x = sent > stages ? sent - stages : 0; x < sent; ++x) drain(bar + x % stages, (x / stages) & 1);
      };
      landed(sm.q_full, S::kQ, n);
      landed(sm.k_full, S::kK, at);
      landed(sm.v_full, S::kV, nv);
      landed(sm.do_full, S::kQ, ndo);
    } else if (warp == 2) {
      // ------------------------------------------------------------- items
      uint32_t n = 0;
      bool ok = true, end = false;
      for (int64_t u0 = blockIdx.x; ok && !end; u0 += (int64_t)32 * gridDim.x) {
        const int64_t u = u0 + (int64_t)lane * gridDim.x;
        DqItem it{};
        if (u < prm.n_items) {
          const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, prm.tpt, u / p.Hk);
          const int64_t t0 = g.tile * prm.tpt;
          int64_t k0, kn;
          segment_rows(p.cu_k, g.s, p.nk, k0, kn);
          if (t0 < g.n)  // else an idle slot
            it.blocks = (int)((kn + kT - 1) / kT);  // 0: no keys, the output warps have it
          it.hk = (int)(u % p.Hk);
          it.tok0 = (int)(g.row + t0);
          it.ntok = (int)min((int64_t)prm.tpt, g.n - t0);
          it.key0 = (int)k0;
          it.keys = (int)kn;
        }
        end = u0 + (int64_t)32 * gridDim.x >= prm.n_items;
        uint32_t have = __ballot_sync(0xffffffffu, it.blocks > 0);
        for (; have | (uint32_t)end; have &= have - 1, ++n) {
          const uint32_t s = n % kDqSlots;
          if (!(ok = wait(&sm.item_empty[s], ((n / kDqSlots) & 1) ^ 1))) break;
          if (have == 0) {  // no more items
            if (lane == 0) {
              sm.item[s].blocks = 0;
              mbar_arrive(&sm.item_full[s]);
            }
            break;
          }
          if ((int)lane == __ffs(have) - 1) {
            sm.item[s] = it;
            mbar_arrive(&sm.item_full[s]);
          }
          __syncwarp();
        }
      }
    } else if (warp == 3) {
      // Masked keys of K and V: S, dP and dQ's terms of theirs are then zero.
      // And when Q (of a first block), K and V are there.
      uint32_t n = 0, at = 0;
      bool ok = true;
      DqItem it;
      while (ok && next_item(n, it, ok))
        for (int j = 0; j < it.blocks; ++j, ++at) {
          const uint32_t st = at % S::kK;
          const uint32_t keys = lane_keys(p.mask, (int64_t)it.key0 + j * kT, it.keys - j * kT, lane);
          auto zero_keys = [&](uint32_t base) {
            for (int g = 0; g < 4; ++g)
              if (!((keys >> g) & 1u))
                for (int x = 0; x < 8 * S::kC; ++x)
                  st_shared_v4(base + (x >> 3) * kChunkB + (lane + 32 * g) * 128 + (((x + lane) & 7) << 4), 0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
          };
          const bool some = __any_sync(0xffffffffu, keys != 15u);
          if (!(ok = wait(&sm.k_full[st], (at / S::kK) & 1))) break;
          if (some) zero_keys(smem_u32(sm.k[st]));
          if (j == 0 && !(ok = wait(&sm.q_full[(n - 1) % S::kQ], ((n - 1) / S::kQ) & 1))) break;
          if (!(ok = wait(&sm.v_full[at % S::kV], (at / S::kV) & 1))) break;
          if (some) zero_keys(smem_u32(sm.v[at % S::kV]));
          if (lane == 0) mbar_arrive(&sm.ready[st]);
        }
    } else if (warp == 1) {
      // ---------------------------------------------------------- products
      constexpr uint32_t idesc_s = idesc_bf16_f32(kT, kT, false, false);
      constexpr uint32_t idesc_q = idesc_bf16_f32(kT, D, false, true);
      constexpr uint32_t kStep = S::kTile >> 4, kFirst = 2, kLast = 4;
      const uint32_t q_lo = desc_lo(smem_u32(sm.q[0]), 16), do_lo = desc_lo(smem_u32(sm.dout[0]), 16),
                     k_lo = desc_lo(smem_u32(sm.k[0]), 16), v_lo = desc_lo(smem_u32(sm.v[0]), 16),
                     k_mn = desc_lo(smem_u32(sm.k[0]), kChunkB);
      auto waitq = [&](uint64_t* bar, uint32_t parity) -> bool {
        return quick_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
      };
      uint32_t n = 0, left = 0;             // items begun; blocks left of the one of S
      uint32_t sk = 0, sf = 0;              // K stage and phase of S
      uint32_t pv = 0, qk = 0;              // V stage of dP, K stage of dQ
      uint32_t buf = 0, dsf = 0;            // S buffer of S (and of dQ), phases of ds_full
      uint32_t sq = S::kQ - 1, pq = sq;     // Q stage of S, dO stage of dP
      uint32_t pf = 1, dqf = 0;             // phases of do_full and dq_empty
      uint32_t f0 = 0, f1 = 0, f2;          // flags of the blocks of dQ, dP and S; 0: none
      bool ok = true, end = false;
#pragma unroll 1
      do {
        f2 = 0;
        if (left > 0) {
          f2 = left == 1 ? 1u | kLast : 1u;
          --left;
        } else if (!end) {
          const uint32_t s = n % kDqSlots;
          if (!(ok = waitq(&sm.item_full[s], (n / kDqSlots) & 1))) break;
          left = warp_uniform((uint32_t)sm.item[s].blocks);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.item_empty[s]);
          ++n;
          end = left == 0;
          if (!end) {
            sq = sq + 1 == S::kQ ? 0 : sq + 1;
            f2 = left == 1 ? 1u | kFirst | kLast : 1u | kFirst;
            --left;
          }
        }
        if (f0) {
          if (!(ok = waitq(&sm.ds_full[buf], (dsf >> buf) & 1))) break;
          dsf ^= 1u << buf;
          tc_fence_after();
        }
        if (f1) {
          if (f1 & kFirst) {
            pq = pq + 1 == S::kQ ? 0 : pq + 1;
            if (pq == 0) pf ^= 1;
            if (!(ok = waitq(&sm.do_full[pq], pf))) break;
            tc_fence_after();
          }
          mma_nt<D>(128, do_lo + pq * kStep, v_lo + pv * kStep, idesc_s);
          mma_commit_w(&sm.dp_full[pv]);
          if (f1 & kLast) mma_commit_w(&sm.do_empty[pq]);
          pv = (pv + 1) % S::kV;
        }
        if (f0) {
          if (f0 & kFirst) {  // dQ of the item before has been read
            dqf ^= 1;
            if (!(ok = waitq(&sm.dq_empty, dqf))) break;
            tc_fence_after();
          }
          mma_tnh(384, buf * 256, k_mn + qk * kStep, idesc_q, (f0 & kFirst) ^ kFirst);
          mma_commit_w(&sm.k_empty[qk]);
          if (f0 & kLast) mma_commit_w(&sm.dq_full);
          qk = qk + 1 == S::kK ? 0 : qk + 1;
        }
        if (f2) {
          if (!(ok = waitq(&sm.ready[sk], sf))) break;
          tc_fence_after();
          mma_nt<D>(buf * 256, q_lo + sq * kStep, k_lo + sk * kStep, idesc_s);
          mma_commit_w(&sm.s_full[buf]);
          if (f2 & kLast) mma_commit_w(&sm.q_empty[sq]);
          if (++sk == S::kK) {
            sk = 0;
            sf ^= 1;
          }
        }
        buf ^= 1;
        f0 = f1;
        f1 = f2;
      } while (f0 | f1);
      mma_commit_w(&sm.mma_done);
      drain(&sm.mma_done, 0);
    }
  } else if (warp < 12) {
    setmaxnreg_inc<kDqEw>();
    const uint32_t quarter = warp & 3, half = (warp - 4) >> 2, lane_base = (quarter * 32) << 16;
    const int row = (int)(quarter * 32 + lane), rt = (int)(((uint32_t)row * prm.inv_g) >> 16), rg = row - rt * p.G;
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    uint32_t n = 0, at = 0, pairs = 0;
    bool ok = true;
    DqItem it, nx;
    // LSE and D of this row, loaded an item ahead; +inf and 0 where there is none
    auto row_load = [&](const DqItem& x, float& l, float& d) {
      l = INFINITY;
      d = 0.f;
      if (x.blocks > 0 && rt < x.ntok) {
        const int64_t rv = (int64_t)(x.hk * p.G + rg) * p.nq + x.tok0 + rt;
        l = p.lse[rv];
        d = p.dsum[rv];
      }
    };
    float nl, nd;
    bool more = next_item(n, nx, ok);
    if (more) row_load(nx, nl, nd);
    while (ok && more) {
      it = nx;
      // P = 0 in a row that does not exist or has no keys, and dS too in the latter
      const uint32_t row_on = nl == -INFINITY ? 0u : ~0u;
      const float le = row_on ? -nl * kLog2e : -INFINITY;
      const uint64_t l2 = pack_f32x2(le, le);
      uint64_t d2 = pack_f32x2(-nd, -nd);
      more = next_item(n, nx, ok);
      if (!ok) break;
      row_load(nx, nl, nd);
      uint32_t keys = lane_keys(p.mask, it.key0, it.keys, lane);
      for (int j = 0; j < it.blocks; ++j, ++at) {
        const uint32_t now = keys;
        if (j + 1 < it.blocks) keys = lane_keys(p.mask, (int64_t)it.key0 + (j + 1) * kT, it.keys - (j + 1) * kT, lane);
        const uint32_t ts = lane_base + (at & 1) * 256 + half * 64;
        if (!(ok = wait(&sm.s_full[at & 1], (at >> 1) & 1))) break;
        tc_fence_after();
        uint32_t r[64];
        tmem_ld64(ts, r);
#pragma unroll
        for (int x = 0; x < 64; x += 2) {
          float a, b;
          unpack_f32x2(fma_f32x2(pack_u32x2(r[x], r[x + 1]), c2, l2), a, b);
          r[x] = __float_as_uint(ex2_approx(a));
          r[x + 1] = __float_as_uint(ex2_approx(b));
        }
        const bool whole = __all_sync(0xffffffffu, now == 15u);
        if (!whole) {  // P of a masked key (S = 0) may be infinite; the others' is at most 1, or NaN, which stays
#pragma unroll
          for (int x = 0; x < 64; ++x) r[x] = __float_as_uint(min_nan(__uint_as_float(r[x]), 2.f));
        }
        if (!(ok = wait(&sm.dp_full[at % S::kV], (at / S::kV) & 1))) break;
        tc_fence_after();
        if (kFew && it.blocks == 1) {
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t v[32];
            tmem_ld32(lane_base + 128 + half * 64 + h * 32, v);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; x += 2)
              sum[(x >> 1) & 1] = fma_f32x2(pack_u32x2(r[h * 32 + x], r[h * 32 + x + 1]), pack_u32x2(v[x], v[x + 1]),
                                            sum[(x >> 1) & 1]);
          }
          float a, b;
          unpack_f32x2(add_f32x2(sum[0], sum[1]), a, b);
          float(*part)[kT] = sm.pair[pairs & 1];
          part[half][row] = a + b;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.pair_full[quarter]);
          if (!(ok = wait(&sm.pair_full[quarter], pairs & 1))) break;
          ++pairs;
          const float d = part[0][row] + part[1][row];
          d2 = pack_f32x2(-d, -d);
          if (half == 0 && rt < it.ntok) p.dsum[(int64_t)(it.hk * p.G + rg) * p.nq + it.tok0 + rt] = d;
        }
        uint32_t ds[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v[32];
          tmem_ld32(lane_base + 128 + half * 64 + h * 32, v);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 32; x += 2) {
            float a, b;
            unpack_f32x2(mul_f32x2(pack_u32x2(r[h * 32 + x], r[h * 32 + x + 1]),
                                   add_f32x2(pack_u32x2(v[x], v[x + 1]), d2)),
                         a, b);
            ds[h * 16 + x / 2] = pack_bf16x2(a, b);
          }
        }
        if (!whole) {
#pragma unroll
          for (int x = 0; x < 32; ++x) ds[x] &= row_on;
        }
        tmem_st32(ts, ds);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.ds_full[at & 1]);
      }
    }
  } else {
    static_assert(kDqOut == kDqLaunch, "the output warps keep their registers");
    const uint32_t quarter = warp & 3, lane_base = (quarter * 32) << 16, c = lane & 3;
    auto token_of = [&](uint32_t r) -> uint32_t { return (r * prm.inv_g) >> 16; };
    // dQ of row y of a tile, nullptr where it has no such row
    auto row_of = [&](int64_t tok0, int ntok, int hk, uint32_t y) -> __nv_bfloat16* {
      const uint32_t yt = token_of(y);
      return (int)yt < ntok ? static_cast<__nv_bfloat16*>(p.dq) + (tok0 + yt) * p.dqs +
                                  ((int64_t)hk * p.G + (y - yt * p.G)) * D + c * 8
                            : nullptr;
    };
    // Tiles of segments without keys: dQ = 0.  32 items are looked at together.
    if (p.cu_k || p.nk == 0)
      for (int64_t u0 = blockIdx.x; u0 < prm.n_items; u0 += (int64_t)32 * gridDim.x) {
        const int64_t u = u0 + (int64_t)lane * gridDim.x;
        int64_t tok0 = 0, k0, kn;
        int ntok = 0;
        if (u < prm.n_items) {
          const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, prm.tpt, u / p.Hk);
          const int64_t t0 = g.tile * prm.tpt;
          segment_rows(p.cu_k, g.s, p.nk, k0, kn);
          tok0 = g.row + t0;
          if (t0 < g.n && kn == 0) ntok = (int)min((int64_t)prm.tpt, g.n - t0);
        }
        for (uint32_t found = __ballot_sync(0xffffffffu, ntok > 0); found; found &= found - 1) {
          const int who = __ffs(found) - 1;
          const int64_t tk = __shfl_sync(0xffffffffu, tok0, who);
          const int nt = __shfl_sync(0xffffffffu, ntok, who), hk = (int)((u0 + (int64_t)who * gridDim.x) % p.Hk);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            __nv_bfloat16* o = row_of(tk, nt, hk, quarter * 32 + (lane & ~3u) + i);
            if (o)
              for (int g = 0; g < D / 32; ++g) *reinterpret_cast<uint4*>(o + g * 32) = make_uint4(0, 0, 0, 0);
          }
        }
      }
    uint32_t n = 0;
    bool ok = true;
    DqItem it;
    while (ok && next_item(n, it, ok)) {
      __nv_bfloat16* out[4];  // the rows of this lane's quad, its 16-byte unit
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = row_of(it.tok0, it.ntok, it.hk, quarter * 32 + (lane & ~3u) + i);
      if (!(ok = wait(&sm.dq_full, (n - 1) & 1))) break;
      tc_fence_after();
#pragma unroll 2
      for (int g = 0; g < D / 32; ++g) {
        uint32_t r[32], u[4][4];
        tmem_ld32(lane_base + 384 + g * 32, r);
        tmem_wait_ld();
        if (g == D / 32 - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.dq_empty);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x)
          u[x >> 2][x & 3] =
              pack_bf16x2(__uint_as_float(r[2 * x]) * p.scale, __uint_as_float(r[2 * x + 1]) * p.scale);
        exchange_units<1>(u, c & 1, 0, 1);
        exchange_units<1>(u, c & 1, 2, 3);
        exchange_units<2>(u, c >> 1, 0, 2);
        exchange_units<2>(u, c >> 1, 1, 3);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (out[i]) *reinterpret_cast<uint4*>(out[i] + g * 32) = make_uint4(u[i][0], u[i][1], u[i][2], u[i][3]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(sm.tmem_base, 512);
}

// =========================================================================
//                                 dK, dV
// =========================================================================
// TMEM columns: S^T / P^T [0,128), dP^T / dS^T [128,256), dV [256,256+d), dK
// [384,384+d); lanes = keys.  Per tile t the tensor core runs dV_t, S^T_{t+1}
// while the elementwise warps form dS^T_t, and dK_t, dP^T_{t+1} while they form
// P^T_{t+1}.
//   warp 0   asks for the items (NextItem) and decodes them into a ring; TMA:
//            K, V and the Q ring
//   warp 2   zeroes Q rows that are not the item's; LSE and D of the rows
//   warp 3   TMA: the dO ring; zeroes its rows
// An item is published once all loads of the one before have been asked for, and
// nothing is loaded across items: no wait depends on the warp that waits.
constexpr int kKvThreads = 384;
constexpr int kKvLaunch = 168, kKvCtl = 104, kKvEw = 200;
static_assert(kKvCtl + 2 * kKvEw <= 3 * kKvLaunch, "setmaxnreg split must fit the launch");

constexpr int kKvSlots = 2, kKvReaders = 11;

struct Work {  // one item: a run of query tiles, a kv head, every ks-th key block
  int32_t hk, part, tiles, block0, blocks;  // blocks 0: no more items
  int32_t tok0, key0, ntok, keys;           // tokens of the run, keys of the segment
  int32_t kslot;                            // first key block's place among all segments'
};

// Item u, by a whole warp; blocks 0 where its slot is idle.
UT_DEV Work decode(const BwdParams& b, int u) {
  const XattnParams& p = b.x;
  Work w{};
  const int v = u / b.ks, slot = v / p.Hk;
  w.block0 = u - v * b.ks;
  w.hk = v - slot * p.Hk;
  const Segment g = warp_segment_of_slot(p.cu_q, p.B, p.nq, b.R * b.tpt, slot);
  const int64_t t0 = g.tile * b.R * b.tpt;
  if (t0 >= g.n) return w;
  int64_t k0, kn;
  segment_rows(p.cu_k, g.s, p.nk, k0, kn);
  w.part = (int)g.tile;
  w.tok0 = (int)(g.row + t0);
  w.ntok = (int)min((int64_t)b.R * b.tpt, g.n - t0);
  w.tiles = (w.ntok + b.tpt - 1) / b.tpt;
  w.key0 = (int)k0;
  w.kslot = (int)(k0 / kT) + g.s;
  w.keys = (int)kn;
  w.blocks = max(0, ((int)((kn + kT - 1) / kT) - w.block0 + b.ks - 1) / b.ks);
  return w;
}

template <int D>
struct KvSmem {
  static constexpr int kC = D / 64;
  static constexpr uint32_t kTile = kT * D * 2;
  static constexpr int kQ = D == 128 ? 3 : 4, kDo = D == 128 ? 2 : 4;
  alignas(1024) uint8_t k[kTile];
  alignas(1024) uint8_t v[kTile];
  alignas(1024) uint8_t q[kQ][kTile];
  alignas(1024) uint8_t dout[kDo][kTile];
  Work item[kKvSlots];
  NextItem next;
  alignas(16) float lse2[2][kT];  // -LSE log2(e) and -D of the rows of a tile
  alignas(16) float dsum[2][kT];
  uint64_t kv_full, kv_empty, q_full[kQ], q_empty[kQ], do_full[kDo], do_empty[kDo], q_ready[4], do_ready[4];
  uint64_t item_full[kKvSlots], item_empty[kKvSlots];
  uint64_t s_full, dp_full, p_full, ds_full, acc_full, acc_empty, mma_done;
  uint32_t tmem_base;
  int abort_flag;
};

template <int D>
__global__ void __launch_bounds__(kKvThreads, 1)
    xattn_dkdv_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                      const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                      const BwdParams prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = KvSmem<D>;
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const XattnParams& p = prm.x;
  const uint32_t warp = warp_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    return;
  }
  if (threadIdx.x == 0) {
    uint64_t* one[] = {&sm.kv_full, &sm.kv_empty, &sm.s_full, &sm.dp_full, &sm.acc_full, &sm.mma_done};
    for (uint64_t* x : one) mbar_init(x, 1);
    for (int s = 0; s < S::kQ; ++s) {
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_empty[s], 1);
    }
    for (int s = 0; s < S::kDo; ++s) {
      mbar_init(&sm.do_full[s], 1);
      mbar_init(&sm.do_empty[s], 1);
    }
    uint64_t* eight[] = {&sm.p_full, &sm.ds_full, &sm.acc_empty};
    for (uint64_t* x : eight) mbar_init(x, 8);
    for (int s = 0; s < kKvSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], kKvReaders);
    }
    next_item_init(sm.next);
    for (int s = 0; s < 4; ++s) {
      mbar_init(&sm.q_ready[s], 1);
      mbar_init(&sm.do_ready[s], 1);
    }
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  grid_next();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_wait();
  if (sm.tmem_base != 0 && threadIdx.x == 0) {  // as in the dQ kernel
    set_status(p.status, UT_ERR_CUDA);
    sm.abort_flag = 1;
  }
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // whole warp, converged
    return warp_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto drain = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_drain(bar, parity, kDrainTimeoutNs)) set_status(p.status, UT_ERR_TIMEOUT);
  };

  // The next item; false at the end or on an abort (then ok = false).  Whole warp.
  auto next_item = [&](uint32_t& n, Work& w, bool& ok) -> bool {
    const uint32_t s = n % kKvSlots;
    if (!(ok = wait(&sm.item_full[s], (n / kKvSlots) & 1))) return false;
    w = sm.item[s];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.item_empty[s]);
    ++n;
    return w.blocks > 0;
  };

  if (warp < 4) {
    setmaxnreg_dec<kKvCtl>();
    if (warp == 0) {
      const uint64_t keep = policy_evict_last();
      const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kC;
      uint32_t nkv = 0, nt = 0, n = 0, asked = 0;
      bool ok = true;
      for (int u = (int)blockIdx.x; ok;) {
        Work w{};
        if (u >= 0) w = decode(prm, u);
        if (u < 0 || w.blocks > 0) {
          const uint32_t s = n % kKvSlots;
          if (!(ok = wait(&sm.item_empty[s], ((n / kKvSlots) & 1) ^ 1))) break;
          if (lane == 0) {
            sm.item[s] = w;
            mbar_arrive(&sm.item_full[s]);
          }
          __syncwarp();
          ++n;
          if (u < 0) break;  // no more items
          for (int b = 0; b < w.blocks && ok; ++b) {
            const int j = w.block0 + b * prm.ks;
            if (!(ok = wait(&sm.kv_empty, (nkv & 1) ^ 1))) break;
            if (lane == 0) {
              mbar_expect_tx(&sm.kv_full, 2 * S::kTile);
              for (int c = 0; c < S::kC; ++c) {
                tma_load_3d(sm.k + c * kChunkB, &tm_k, &sm.kv_full, c * 64, w.hk, w.key0 + j * kT, keep);
                tma_load_3d(sm.v + c * kChunkB, &tm_v, &sm.kv_full, c * 64, w.hk, w.key0 + j * kT, keep);
              }
            }
            __syncwarp();
            ++nkv;
            for (int t = 0; t < w.tiles; ++t, ++nt) {
              const uint32_t st = nt % S::kQ;
              if (!(ok = wait(&sm.q_empty[st], ((nt / S::kQ) & 1) ^ 1))) break;
              if (lane == 0) {
                mbar_expect_tx(&sm.q_full[st], bytes);
                for (int c = 0; c < S::kC; ++c)
                  tma_load_3d(sm.q[st] + c * kChunkB, &tm_q, &sm.q_full[st], c * 64, w.hk * p.G,
                              w.tok0 + t * prm.tpt, keep);
              }
              __syncwarp();
            }
          }
          if (!ok) break;
        }
        // asked for now, two or three tiles before this item's end, not at its
        // begin: who asks first should be who is done first
        if (lane == 0) next_item_ask(sm.next, asked);
        __syncwarp();
        ++asked;
        if (!(ok = wait(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1))) break;
        u = (int)warp_uniform((uint32_t)next_item_answer(sm.next, asked - 1));
        fence_proxy_async_smem();  // the answer is read before its place is used again
        __syncwarp();
      }
      if (lane == 0) {
        if (asked > 0) drain(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1);
        if (nkv > 0) drain(&sm.kv_full, (nkv - 1) & 1);
        for (uint32_t x = nt > S::kQ ? nt - S::kQ : 0; x < nt; ++x) drain(&sm.q_full[x % S::kQ], (x / S::kQ) & 1);
      }
    } else if (warp == 1) {
      constexpr uint32_t idesc_s = idesc_bf16_f32(kT, kT, false, false);
      constexpr uint32_t idesc_acc = idesc_bf16_f32(kT, D, false, true);
      const uint32_t k_lo = desc_lo(smem_u32(sm.k), 16), v_lo = desc_lo(smem_u32(sm.v), 16),
                     q_lo = desc_lo(smem_u32(sm.q[0]), 16), do_lo = desc_lo(smem_u32(sm.dout[0]), 16),
                     q_mn = desc_lo(smem_u32(sm.q[0]), kChunkB), do_mn = desc_lo(smem_u32(sm.dout[0]), kChunkB);
      constexpr uint32_t kStep = S::kTile >> 4;
      auto waitq = [&](uint64_t* bar, uint32_t parity) -> bool {
        return quick_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
      };
      uint32_t nkv = 0, nt = 0;                   // key blocks, tiles
      uint32_t qs = 0, ds = 0, qn = 0, dn = 0;    // stages: of dK, dV; of S, dP
      bool ok = true;
      auto issue_s = [&]() {
        mma_nt<D>(0, k_lo, q_lo + qn * kStep, idesc_s);
        mma_commit_w(&sm.s_full);
        qn = qn + 1 == S::kQ ? 0 : qn + 1;
      };
      auto issue_dp = [&]() {
        mma_nt<D>(128, v_lo, do_lo + dn * kStep, idesc_s);
        mma_commit_w(&sm.dp_full);
        dn = dn + 1 == S::kDo ? 0 : dn + 1;
      };
      for (uint32_t n = 0;; ++n) {
        const uint32_t s = n % kKvSlots;
        if (!(ok = waitq(&sm.item_full[s], (n / kKvSlots) & 1))) break;
        const uint32_t tiles = warp_uniform((uint32_t)sm.item[s].tiles);
        uint32_t blocks = warp_uniform((uint32_t)sm.item[s].blocks);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.item_empty[s]);
        if (blocks == 0) break;
        for (; blocks > 0; --blocks) {
          if (!(ok = waitq(&sm.kv_full, nkv & 1))) break;
          if (!(ok = waitq(&sm.q_ready[nt & 3], (nt >> 2) & 1))) break;
          tc_fence_after();
          issue_s();
          if (!(ok = waitq(&sm.do_ready[nt & 3], (nt >> 2) & 1))) break;
          issue_dp();
          if (!(ok = waitq(&sm.acc_empty, (nkv & 1) ^ 1))) break;
#pragma unroll 1
          for (uint32_t t = 0; t < tiles; ++t, ++nt) {
            const bool more = t + 1 < tiles;
            if (more && !(ok = waitq(&sm.q_ready[(nt + 1) & 3], ((nt + 1) >> 2) & 1))) break;
            if (!(ok = waitq(&sm.p_full, nt & 1))) break;
            tc_fence_after();
            mma_tnh(256, 0, do_mn + ds * kStep, idesc_acc, t);
            mma_commit_w(&sm.do_empty[ds]);
            ds = ds + 1 == S::kDo ? 0 : ds + 1;
            if (more) issue_s();
            if (!(ok = waitq(&sm.ds_full, nt & 1))) break;
            tc_fence_after();
            mma_tnh(384, 128, q_mn + qs * kStep, idesc_acc, t);
            mma_commit_w(&sm.q_empty[qs]);
            qs = qs + 1 == S::kQ ? 0 : qs + 1;
            if (more) {
              if (!(ok = waitq(&sm.do_ready[(nt + 1) & 3], ((nt + 1) >> 2) & 1))) break;
              issue_dp();
            }
          }
          if (!ok) break;
          mma_commit_w(&sm.kv_empty);
          mma_commit_w(&sm.acc_full);
          ++nkv;
        }
        if (!ok) break;
      }
      mma_commit_w(&sm.mma_done);
      drain(&sm.mma_done, 0);
    } else {
      // ------- rows that must read as zero (warp 2: Q, warp 3: dO); dO loads;
      // warp 2 also brings LSE and D of the rows, four a lane, a tile ahead
      const bool is_q = warp == 2;
      const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kC;
      const uint64_t keep = policy_evict_last();
      uint32_t n = 0, nt = 0, sent = 0;  // items, tiles made ready, dO tiles asked for
      bool ok = true;
      Work w;
      while (ok && next_item(n, w, ok)) {
        int left = w.blocks * w.tiles, tok = w.tok0;  // dO tiles to ask for, the next one's token
        const int end = w.tok0 + w.tiles * prm.tpt;
        auto load_next = [&]() {
          if (left == 0) return;
          const uint32_t st = sent % S::kDo;
          if (!(ok = wait(&sm.do_empty[st], ((sent / S::kDo) & 1) ^ 1))) return;
          if (lane == 0) {
            mbar_expect_tx(&sm.do_full[st], bytes);
            for (int c = 0; c < S::kC; ++c)
              tma_load_3d(sm.dout[st] + c * kChunkB, &tm_do, &sm.do_full[st], c * 64, w.hk * p.G, tok, keep);
          }
          __syncwarp();
          ++sent;
          --left;
          tok += prm.tpt;
          if (tok == end) tok = w.tok0;  // again, for the next key block
        };
        // A stage's next load is only waited for once the tile kDo - 1 before it
        // has been made ready, so the wait always ends.
        if (!is_q)
          for (int x = 0; x < S::kDo - 1 && ok; ++x) load_next();
        float rl[4], rd[4];  // as loaded: arithmetic on them here would wait for the loads
        auto rows_load = [&](int t) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int col = (int)lane + 32 * i, rt = (int)(((uint32_t)col * prm.inv_g) >> 16), rg = col - rt * p.G;
            rl[i] = -INFINITY;
            rd[i] = 0.f;
            if (rt < min(prm.tpt, w.ntok - t * prm.tpt)) {
              const int64_t rv = (int64_t)(w.hk * p.G + rg) * p.nq + w.tok0 + t * prm.tpt + rt;
              rl[i] = p.lse[rv];
              rd[i] = p.dsum[rv];
            }
          }
        };
        if (is_q) rows_load(0);
        for (int j = 0; j < w.blocks && ok; ++j)
          for (int t = 0; t < w.tiles; ++t, ++nt) {
            const int rows = min(prm.tpt, w.ntok - t * prm.tpt) * p.G;
            const uint32_t nst = is_q ? S::kQ : S::kDo, st = nt % nst, f = nt / nst;
            if (!(ok = wait(is_q ? &sm.q_full[st] : &sm.do_full[st], f & 1))) break;
            if (rows < kT) {
              zero_tail(smem_u32(is_q ? sm.q[st] : sm.dout[st]), S::kC, rows, lane);
              fence_proxy_async_smem();
              __syncwarp();
            }
            if (is_q) {
              // once the rows of two tiles back have been read; -inf: no such row,
              // or a row without keys (P = 0)
              if (nt >= 2 && !(ok = wait(&sm.q_empty[(nt - 2) % S::kQ], ((nt - 2) / S::kQ) & 1))) break;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                sm.lse2[nt & 1][lane + 32 * i] = rl[i] == -INFINITY ? rl[i] : -rl[i] * kLog2e;
                sm.dsum[nt & 1][lane + 32 * i] = -rd[i];
              }
              __syncwarp();
            }
            if (lane == 0) mbar_arrive(is_q ? &sm.q_ready[nt & 3] : &sm.do_ready[nt & 3]);
            if (is_q) {
              if (t + 1 < w.tiles) rows_load(t + 1);
              else if (j + 1 < w.blocks) rows_load(0);
            } else {
              load_next();
              if (!ok) break;
            }
          }
      }
      if (!is_q && lane == 0)  // every copy it asked for has landed
        for (uint32_t x = sent > S::kDo ? sent - S::kDo : 0; x < sent; ++x)
          drain(&sm.do_full[x % S::kDo], (x / S::kDo) & 1);
    }
  } else {
    setmaxnreg_inc<kKvEw>();
    const uint32_t quarter = warp & 3, half = (warp - 4) >> 2;
    const uint32_t krow = quarter * 32 + lane;
    const uint32_t lane_base = (quarter * 32) << 16, ts = lane_base + half * 64;
    constexpr int HC = kT / 2, HD = D / 2;
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    uint32_t n = 0, nt = 0, ng = 0;
    bool ok = true;
    Work w;
    while (ok && next_item(n, w, ok)) {
      for (int b = 0; b < w.blocks && ok; ++b, ++ng) {
        const int j = w.block0 + b * prm.ks;
        const int key = j * kT + (int)krow;
        // P and dS of a masked key are zero: as a mask of the packed pairs
        const uint32_t on = key < w.keys && (!p.mask || p.mask[w.key0 + key]) ? 0xffffffffu : 0u;
        for (int t = 0; t < w.tiles; ++t, ++nt) {
          const uint32_t par = nt & 1;
          const float* ls = sm.lse2[par] + half * HC;
          const float* dv = sm.dsum[par] + half * HC;
          if (!(ok = wait(&sm.s_full, par))) break;
          tc_fence_after();
          uint32_t r[HC];
          tmem_ld32(ts, *reinterpret_cast<uint32_t(*)[32]>(r));
          tmem_ld32(ts + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
          ok = wait(&sm.q_ready[nt & 3], (nt >> 2) & 1);  // the rows' values
          tmem_wait_ld();
          if (!ok) break;
          uint32_t pk[32];
#pragma unroll
          for (int x = 0; x < HC; x += 4) {
            const ulonglong2 l4 = *reinterpret_cast<const ulonglong2*>(ls + x);
            float a, b, c, d;
            unpack_f32x2(fma_f32x2(pack_u32x2(r[x], r[x + 1]), c2, l4.x), a, b);
            unpack_f32x2(fma_f32x2(pack_u32x2(r[x + 2], r[x + 3]), c2, l4.y), c, d);
            a = ex2_approx(a);
            b = ex2_approx(b);
            c = ex2_approx(c);
            d = ex2_approx(d);
            r[x] = __float_as_uint(a);
            r[x + 1] = __float_as_uint(b);
            r[x + 2] = __float_as_uint(c);
            r[x + 3] = __float_as_uint(d);
            pk[x / 2] = pack_bf16x2(a, b) & on;
            pk[x / 2 + 1] = pack_bf16x2(c, d) & on;
          }
          tmem_st32(ts, pk);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.p_full);
          if (!(ok = wait(&sm.dp_full, par))) break;
          tc_fence_after();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t v[32];
            tmem_ld32(ts + 128 + h * 32, v);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; x += 4) {
              const ulonglong2 d4 = *reinterpret_cast<const ulonglong2*>(dv + h * 32 + x);
              float a, b, c, d;
              unpack_f32x2(mul_f32x2(pack_u32x2(r[h * 32 + x], r[h * 32 + x + 1]),
                                     add_f32x2(pack_u32x2(v[x], v[x + 1]), d4.x)),
                           a, b);
              unpack_f32x2(mul_f32x2(pack_u32x2(r[h * 32 + x + 2], r[h * 32 + x + 3]),
                                     add_f32x2(pack_u32x2(v[x + 2], v[x + 3]), d4.y)),
                           c, d);
              pk[h * 16 + x / 2] = pack_bf16x2(a, b) & on;
              pk[h * 16 + x / 2 + 1] = pack_bf16x2(c, d) & on;
            }
          }
          tmem_st32(ts + 128, pk);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.ds_full);
        }
        if (!ok) break;
        // this run's dV, dK of the key block
        if (!(ok = wait(&sm.acc_full, ng & 1))) break;
        tc_fence_after();
        const int64_t at =
            ((((int64_t)w.part * prm.kslots + w.kslot + j) * p.Hk + w.hk) * (D / 4) + half * (HD / 4)) * kT + krow;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          float* dst = (which ? p.part_dk : p.part_dv) + at * 4;
#pragma unroll
          for (int g = 0; g < HD / 32; ++g) {
            uint32_t r[32];
            tmem_ld32(lane_base + (which ? 384 : 256) + half * HD + g * 32, r);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 8; ++x)
              *reinterpret_cast<uint4*>(dst + (g * 8 + x) * kT * 4) =
                  make_uint4(r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.acc_empty);
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
// along the keys, all of a part in flight, written as rows through shared
// memory.
template <int D>
__global__ void __launch_bounds__(256) xattn_bwd_join_kernel(const BwdParams prm) {
  constexpr int kPer = D / 4 * kT / 256;
  __shared__ __align__(16) uint8_t rows[kT * (D * 2 + 16)];
  const XattnParams& p = prm.x;
  grid_wait();
  const Segment g = segment_of_slot(p.cu_k, p.B, p.nk, kT, blockIdx.x);
  const int keys = (int)min((int64_t)kT, g.n - g.tile * kT);
  if (keys <= 0) return;
  int64_t row, nq;
  segment_rows(p.cu_q, g.s, p.nq, row, nq);
  const int64_t tiles = (nq + prm.tpt - 1) / prm.tpt;
  const int parts = (int)((tiles + prm.R - 1) / prm.R);
  const int64_t kslot = min(g.row / kT + g.s + g.tile, prm.kslots - 1);
  const bool is_k = blockIdx.z == 0;
  const float* src = (is_k ? p.part_dk : p.part_dv) + (kslot * p.Hk + blockIdx.y) * (D * kT) + threadIdx.x * 4;
  const int64_t step = prm.kslots * p.Hk * (D * kT);
  const float f = is_k ? p.scale : 1.f;
  float4 a[kPer];
#pragma unroll
  for (int x = 0; x < kPer; ++x) a[x] = make_float4(0, 0, 0, 0);
#pragma unroll 1
  for (int i = 0; i < parts; ++i, src += step) {
    float4 b[kPer];
#pragma unroll
    for (int x = 0; x < kPer; ++x) b[x] = *reinterpret_cast<const float4*>(src + x * 1024);
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      a[x].x += b[x].x;
      a[x].y += b[x].y;
      a[x].z += b[x].z;
      a[x].w += b[x].w;
    }
  }
#pragma unroll
  for (int x = 0; x < kPer; ++x) {
    const int at = x * 256 + threadIdx.x;
    *reinterpret_cast<uint2*>(rows + (at % kT) * (D * 2 + 16) + (at / kT) * 8) =
        make_uint2(pack_bf16x2(a[x].x * f, a[x].y * f), pack_bf16x2(a[x].z * f, a[x].w * f));
  }
  __syncthreads();
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(is_k ? p.dk : p.dv) + (int64_t)blockIdx.y * D;
  const int64_t stride = is_k ? p.dks : p.dvs;
  for (int x = threadIdx.x; x < keys * (D / 8); x += 256) {
    const int r = x / (D / 8), e = x % (D / 8);
    const int64_t key = g.row + g.tile * kT + r;
    // a masked key's row is zero, also where a NaN or an infinity of Q or dO met its P and dS of 0
    const uint4 v = p.mask && !p.mask[key] ? make_uint4(0, 0, 0, 0)
                                           : *reinterpret_cast<const uint4*>(rows + r * (D * 2 + 16) + e * 16);
    *reinterpret_cast<uint4*>(out + key * stride + e * 8) = v;
  }
}

static_assert(sizeof(DqSmem<128>) <= 232448 && sizeof(KvSmem<128>) <= 232448 && sizeof(DqSmem<64>) <= 232448,
              "shared layout exceeds the block limit");

// The setmaxnreg split assumes exactly `regs` registers per thread at launch:
// with fewer, the increases would wait for registers that never come.
template <typename F>
cudaError_t launch(F kern, int64_t grid, int threads, size_t smem, int regs, const BwdParams& prm,
                   const CUtensorMap* tm, cudaStream_t s) {
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaFuncAttributes fa;
  e = cudaFuncGetAttributes(&fa, kern);
  if (e != cudaSuccess) return e;
  if (fa.numRegs != regs) return cudaErrorInvalidConfiguration;
  return launch_next(kern, dim3((unsigned)grid), dim3(threads), smem, s, tm[0], tm[1], tm[2], tm[3], prm);
}

// Items of a run along the keys: the blocks of a segment of mean length, so
// that CTAs side by side go over the same Q and dO tiles together and read
// them from L2.  (One CTA over all four blocks of 23,959 x 512 x 24 x 128: the
// runs of all CTAs pass L2, Q and dO came from DRAM four times, 237 us.)
int key_split(const XattnParams& p) {
  const int64_t mean = (p.nk / p.B + kT - 1) / kT;
  return (int)(mean < 1 ? 1 : (mean > 256 ? 256 : mean));
}

// Tiles of a run: the number of runs with the least modelled time, in cycles.
// An item of R tiles takes 2,200 each and 5,000; equal items run in whole waves,
// those of ragged segments (whose last runs are half full on average) end half
// an item apart.  And the partial sums of a segment's runs are written and read
// (3,400 bytes a cycle).  At most 1 GB of them.
int tiles_per_item(const XattnParams& p) {
  const int64_t tpt = kT / p.G, tiles = (p.nq + tpt - 1) / tpt, across = (int64_t)p.Hk * key_split(p);
  const int64_t part = 2 * segment_slots(p.nk, p.B, kT) * kT * p.Hk * p.d * (int64_t)sizeof(float);
  int64_t best = tiles;
  double least = 0;
  for (int64_t runs = 1; runs <= tiles && runs <= 256; ++runs) {
    if (runs > 1 && runs * part > ((int64_t)1 << 30)) break;
    const int64_t R = (tiles + runs - 1) / runs;
    const double item = R * 2200.0 + 5000.0;
    double t;
    if (p.B == 1) {
      t = (double)((runs * across + p.sms - 1) / p.sms) * item + (double)runs * (2 * part) / 3400.0;
    } else {
      const double waves = (runs + 0.5 * p.B) * (double)across / p.sms, each = (double)runs / p.B + 0.5;
      t = (waves < 1.0 ? 1.0 : waves + 0.5) * item + each * (2 * part) / 3400.0;
    }
    if (runs == 1 || t < least) {
      least = t;
      best = R;
    }
  }
  return (int)(best < 1 ? 1 : best);
}

// one of the two partial sums: [parts of a segment, key slots, kv heads, d / 4, 128, 4]
size_t part_bytes(const XattnParams& p, int R) {
  const int64_t tpt = kT / p.G, tiles = (p.nq + tpt - 1) / tpt;
  return (size_t)((tiles + R - 1) / R) * segment_slots(p.nk, p.B, kT) * p.Hk * p.d * kT * sizeof(float);
}

}  // namespace

int64_t xattn_bwd_tc_items(const XattnParams& p) { return segment_slots(p.nq, p.B, kT / p.G) * p.Hk; }

size_t xattn_bwd_tc_ws(const XattnParams& p) { return 2 * part_bytes(p, tiles_per_item(p)); }

cudaError_t launch_xattn_bwd_tc(const XattnParams& p, void* ws, cudaStream_t s) {
  BwdParams prm{};
  prm.x = p;
  prm.inv_g = (65536u + p.G - 1) / p.G;
  prm.tpt = kT / p.G;
  prm.R = tiles_per_item(p);
  prm.ks = key_split(p);
  prm.kslots = segment_slots(p.nk, p.B, kT);
  prm.x.part_dk = static_cast<float*>(ws);
  prm.x.part_dv = reinterpret_cast<float*>(static_cast<char*>(ws) + part_bytes(p, prm.R));
  prm.scale_log2 = p.scale * kLog2e;
  const bool few = p.nk <= kT || p.B > 1;  // a segment may have one block of keys
  // One segment of one block: the dQ kernel takes all of D, and there is no
  // prefix to check (85,202 x 77 x 24 x 128 takes 572 us; reading O and dO for D
  // would be another 155).
  cudaError_t e = few && !p.cu_q && p.nk > 0 ? cudaSuccess : launch_xattn_dsum(p, true, s);
  if (e != cudaSuccess) return e;
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
    prm.n_items = segment_slots(p.nq, p.B, prm.tpt) * p.Hk;
    const int64_t grid = prm.n_items < p.sms ? prm.n_items : p.sms;
    e = p.d == 64 ? launch(few ? xattn_dq_kernel<64, true> : xattn_dq_kernel<64, false>, grid, kDqThreads,
                           sizeof(DqSmem<64>), kDqLaunch, prm, tm, s)
                  : launch(few ? xattn_dq_kernel<128, true> : xattn_dq_kernel<128, false>, grid, kDqThreads,
                           sizeof(DqSmem<128>), kDqLaunch, prm, tm, s);
    if (e != cudaSuccess) return e;
    if (p.nk > 0) {
      prm.n_items = segment_slots(p.nq, p.B, prm.R * prm.tpt) * p.Hk * prm.ks;
      e = p.d == 64 ? launch(xattn_dkdv_kernel<64>, prm.n_items, kKvThreads, sizeof(KvSmem<64>), kKvLaunch, prm, tm, s)
                    : launch(xattn_dkdv_kernel<128>, prm.n_items, kKvThreads, sizeof(KvSmem<128>), kKvLaunch, prm, tm, s);
      if (e != cudaSuccess) return e;
    }
  }
  if (p.nk > 0) {
    const dim3 grid((unsigned)prm.kslots, p.Hk, 2);
    e = p.d == 64 ? launch_next(xattn_bwd_join_kernel<64>, grid, dim3(256), 0, s, prm)
                  : launch_next(xattn_bwd_join_kernel<128>, grid, dim3(256), 0, s, prm);
  }
  return e;
}

}  // namespace ut
