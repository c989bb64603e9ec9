// Windowed attention with visible first keys, forward, on the 5th-generation
// tensor cores (bf16 in, fp32 accumulate):
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
// over the keys j that query i sees (wattn.cuh) and whose mask is set.
//
// A query tile holds 128 rows: the G heads that share a kv head of 128 / G
// consecutive tokens of one segment (row = token * G + head; one TMA box).  A
// work item is a tile, a kv head and a range of the blocks of 128 keys that the
// tile sees: the blocks of its first keys, then those of its window, which begin
// at the window's first key, not at a multiple of 128, so that a tile of t
// tokens takes ceil((left + right + t) / 128) of them.
//
// CTAs take item after item (NextItem), the head fastest: CTAs in flight share
// the windows of neighbouring tiles in L2.  Roles:
//   warp 0      TMA: Q, K and V tiles, a ring each; which keys of a block the mask
//               leaves, a bit each
//   warp 1      TMEM owner and MMA issuer: S = Q K^T, O += P V.  The products
//               follow one another across items: the next item's first S is
//               computed while this one's last blocks are in the softmax.
//   warp 2      asks for the items and decodes them into a ring
//   warp 3      the rows of a V tile whose keys do not count become zero, so that
//               no value they hold (NaN, infinities) is multiplied
//   softmax     thread = row = TMEM lane; at d = 128 two warps share 32 rows and
//               take 64 columns each.  Pass 1: the maximum; where keys do not
//               count or a row of the warp has its limits in the block, S becomes
//               -inf there.  Pass 2: P as bf16 over S.  O is rescaled in TMEM
//               only where the maximum grew by more than 2^8, so the exponentials
//               stay bounded.
//   output      Q from shared memory to TMEM (d = 128), O / l and LSE, or the
//               split's partial result
// The passes are unrolled over 64 columns, or 32 (d = 64: then S is read again).
// Four warps unrolled over 128 columns (2048 canvas 1,481 us instead of 1,383 at
// that step, a third of a softmax warp's time without an instruction) and eight
// over 32 (1,532) were slower.  The two warps of 32 rows exchange their maxima at
// a hardware barrier: with an mbarrier, polled, 1,393 instead of 1,339.  Taking
// the exponentials with the old reference meanwhile gains nothing (1024 canvas
// 357 us instead of 347): the two share a scheduler, which has work either way.
// d = 128: one CTA an SM, two S buffers, Q in TMEM (S = Q K^T then reads only K
// from shared memory).  TMEM columns S0 [0,128), S1 [128,256), O [256,384), Q
// [384,448), the rows' maximum and sums [448,451).
// d = 64: two CTAs an SM, whose softmaxes and products overlap; one S buffer, Q
// in shared memory.  TMEM columns S [0,128), O [128,192), [192,194).
// Measured (two products of 128 x 128 x d a pair of tile and block): 85,714 rows,
// 24 heads of 128, 512 keys each side and 512 first ones 1,320 to 1,380 us (GPUs
// differ), 1.2 PFLOP/s, tensor pipe active 62%; 23,959 rows in 13 images, 24 heads
// of 64, 192 each side, masked 153 us.  Both are bound by the chain of waits, TMEM
// reads and arithmetic of a block's softmax between its products, and by what an
// item costs beside its blocks.  In SM cycles, of a line through windows of 8 to 64
// blocks (85,714 rows, no first keys): d = 128 3,800 an item and 1,350 a block, whose
// products need 1,024, so that of an item of 13 blocks 18% is its own; the card's
// power cap holds the clock at 1,720 to 1,770 MHz there.  d = 64 (two CTAs) 3,000 and
// 1,580, products 512, at 2,070 MHz.  13 rows over 40,000 keys of a cache and 512
// first ones, 24 heads of 128, split: 77 us, 6.5 TB/s, bound by DRAM.
// Rounding: P to bf16 for its product (the sum l is of the unrounded values),
// O once at the end.
// Every wait is bounded; on expiry the kernel records UT_ERR_TIMEOUT, drains
// its own copies and MMAs, frees TMEM and returns.
#include <float.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "wattn.cuh"
#include "xattn_tc.cuh"

namespace ut {

namespace {

constexpr int kM = 128, kN = 128;
constexpr uint32_t kChunkBytes = 128 * 128;  // 128 rows x 64 bf16
// Slots of key bits.  Those of block c are written when S of block c - 3 is done
// (K's stage is free), and S follows P of the block that had its buffer: of c - 5
// at the earliest, so that five are in use.
constexpr int kKeySlots = 8;
constexpr int kItemSlots = 3;                // no more are taken ahead: other CTAs may be idle

template <int D>
struct Form {
  static constexpr int kCtas = D == 128 ? 1 : 2;    // an SM
  static constexpr bool kQt = D == 128;             // Q in TMEM
  static constexpr int kS = D == 128 ? 2 : 1;       // S buffers
  static constexpr int kHalves = D == 128 ? 2 : 1;  // softmax warps of 32 rows
  static constexpr int kSoftmax = 4 * kHalves, kThreads = 32 * (8 + kSoftmax);
  static constexpr int kQ = D == 128 ? 1 : 2, kK = D == 128 ? 3 : 2, kV = kK;  // tiles in shared memory
  static constexpr uint32_t kCols = D == 128 ? 512 : 256;
  static constexpr uint32_t kO = D == 128 ? 256 : 128, kQc = 384, kMl = D == 128 ? 448 : 192;
  // registers per thread of the two-CTA form: launch and setmaxnreg split
  static constexpr int kRegLaunch = 80, kRegCtl = 64, kRegSoftmax = 112, kRegOut = 64;
  static_assert(kRegCtl + kRegSoftmax + kRegOut <= 3 * kRegLaunch, "the split must fit the launch");
};

struct Item {
  int32_t hk;          // kv head; -1: no more items
  int32_t blocks;      // its key blocks, at least one
  int32_t tok0, ntok;  // its tokens
  int32_t p0;          // position of the first
  int32_t key0;        // first key of the segment
  int32_t j0;          // first of the blocks of the tile's ranges
  int32_t split;
  WinRange rg;
};

template <int D>
struct Smem {
  using F = Form<D>;
  static constexpr int kChunks = D / 64;
  static constexpr uint32_t kTile = kM * D * 2;
  alignas(1024) uint8_t q[F::kQ][kTile];
  alignas(1024) uint8_t k[F::kK][kTile];
  alignas(1024) uint8_t v[F::kV][kTile];
  uint32_t keys[kKeySlots][4];     // masked keys: of a K tile, a bit set where it counts
  float most[2][F::kHalves][kM];   // of the halves of a row
  uint64_t q_full[F::kQ], q_empty[F::kQ], k_full[F::kK], k_empty[F::kK], v_full[F::kV], v_empty[F::kV], v_ready[F::kV];
  uint64_t qt_full, qt_empty, s_full[F::kS], p_full[F::kS], pv_done, ml_full, o_full, o_empty, mma_done;
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  Item item[kItemSlots];
  NextItem next;
  uint32_t tmem_base;
  int abort_flag;
};

// The two warps of 32 rows (hardware barriers 1 to 4)
UT_DEV void pair_sync(uint32_t id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }
UT_DEV void pair_arrive(uint32_t id) { asm volatile("barrier.cta.arrive %0, 64;" ::"r"(id) : "memory"); }

struct Params {
  WinParams w;
  uint32_t inv_g;   // ceil(2^16 / G): (r * inv_g) >> 16 = r / G for r < 128, G <= 64
  int tpt;          // tokens of a tile
  int slots;        // item slots along the query rows
  int64_t n_items;  // slots * Hk * nsplit
  float scale_log2;
  bool keep_kv;     // K and V are read by several items: keep them in L2
};

// The result of a tile without keys, or of a part without blocks: O = 0, LSE =
// -inf, or their partial results.  Whole warp.
template <int D>
UT_DEV void empty_rows(const XattnParams& p, int hk, int tok0, int ntok, int split, uint32_t lane) {
  for (int r = (int)lane / 8; r < ntok * p.G; r += 4) {
    const int tok = tok0 + r / p.G, h = hk * p.G + r % p.G;
    if (p.nsplit > 1) {
      const int64_t row = ((int64_t)split * p.nq + tok) * p.H + h;
      for (int c = (int)(lane & 7) * 4; c < D; c += 32) *reinterpret_cast<uint4*>(p.part_o + row * D + c) = make_uint4(0, 0, 0, 0);
      if ((lane & 7) == 0) p.part_ml[row] = make_float2(-1e30f, 0.f);
    } else {
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.o) + (int64_t)tok * p.os + (int64_t)h * D;
      for (int c = (int)(lane & 7) * 8; c < D; c += 64) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
      if ((lane & 7) == 0) p.lse[(int64_t)h * p.nq + tok] = -INFINITY;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(Form<D>::kThreads, Form<D>::kCtas)
    wattn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = Smem<D>;
  using F = Form<D>;
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const XattnParams& p = prm.w.x;
  const uint32_t warp = warp_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kQ; ++s) {
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_empty[s], F::kQt ? 4 : 1);  // the output warps have copied it / S is done
    }
    for (int s = 0; s < F::kK; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.k_empty[s], 1);
    }
    for (int s = 0; s < F::kV; ++s) {
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.v_empty[s], 1);
      mbar_init(&sm.v_ready[s], 1);
    }
    mbar_init(&sm.qt_full, 4);
    mbar_init(&sm.qt_empty, 1);
    for (int s = 0; s < F::kS; ++s) {
      mbar_init(&sm.s_full[s], 1);
      mbar_init(&sm.p_full[s], F::kSoftmax);
    }
    mbar_init(&sm.pv_done, 1);
    mbar_init(&sm.ml_full, F::kSoftmax);
    mbar_init(&sm.o_full, 1);
    mbar_init(&sm.o_empty, 4);
    mbar_init(&sm.mma_done, 1);
    for (int s = 0; s < kItemSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], 7 + F::kSoftmax);  // warps 0, 1, 3, 4, ...
    }
    next_item_init(sm.next);
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, F::kCols);
    tmem_relinquish();
  }
  grid_next();  // the kernel that joins the splits
  if (blockIdx.x == 0) {
    check_cu(p.cu_q, p.B, p.nq, p.status);
    check_cu(p.cu_k, p.B, p.nk, p.status);
    check_lens_of(p, prm.w.k_len);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(sm.tmem_base);

  auto wait = [&](uint64_t* bar, uint32_t parity) {  // whole warp, converged
    return warp_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto drain = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_drain(bar, parity, kDrainTimeoutNs)) set_status(p.status, UT_ERR_TIMEOUT);
  };
  // The next item; false at the end or on an abort (then ok = false).
  auto next_item = [&](uint32_t& n, Item& it, bool& ok) -> bool {
    const uint32_t s = n % kItemSlots;
    if (!(ok = wait(&sm.item_full[s], (n / kItemSlots) & 1))) return false;
    it = sm.item[s];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.item_empty[s]);
    ++n;
    return it.hk >= 0;
  };
  using Block = WinBlock<kN>;
  auto all_keys = [&](const Block& b) { return !p.mask && b.e - b.x >= kN; };

  // For the warps that read TMEM: thread = row = TMEM lane
  const uint32_t quarter = warp & 3, lane_base = tmem + ((quarter * 32) << 16), row = quarter * 32 + lane;
  auto token_of = [&](uint32_t r) -> int { return (int)((r * prm.inv_g) >> 16); };  // r / G

  if (warp < 4) {
    if constexpr (F::kCtas == 2) setmaxnreg_dec<F::kRegCtl>();
    if (warp == 0) {
      // ------------------------------------------------------ Q, K, V producer
      if (lane == 0) {
        tma_prefetch_desc(&tm_q);
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
      }
      const uint64_t pol = prm.keep_kv ? policy_evict_last() : policy_evict_first(), pol_q = policy_evict_first();
      const uint32_t q_bytes = (uint32_t)prm.tpt * p.G * 128 * S::kChunks;
      uint32_t n = 0, nq = 0, at = 0, sent = 0;  // items, Q tiles, K tiles, V tiles asked for
      bool ok = true;
      Item it;
      while (ok && next_item(n, it, ok)) {
        const uint32_t qs = nq % F::kQ;
        if (!(ok = wait(&sm.q_empty[qs], ((nq / F::kQ) & 1) ^ 1))) break;
        if (lane == 0) {
          mbar_expect_tx(&sm.q_full[qs], q_bytes);
          for (int c = 0; c < S::kChunks; ++c)
            tma_load_3d(sm.q[qs] + c * kChunkBytes, &tm_q, &sm.q_full[qs], c * 64, it.hk * p.G, it.tok0, pol_q);
        }
        __syncwarp();
        ++nq;
        uint32_t next[4];  // the mask of the keys lane, lane + 32, ..., a block ahead
        auto load_mask = [&](const Block& b) {
#pragma unroll
          for (int w = 0; w < 4; ++w)
            next[w] = b.x + w * 32 + (int)lane < b.e ? p.mask[(int64_t)it.key0 + b.x + w * 32 + lane] : 0u;
        };
        Block blk(it.rg, it.j0);
        if (p.mask) load_mask(blk);
        for (int t = 0; t < it.blocks; ++t) {
          const int x = blk.x;
          blk.next(it.rg);
          const uint32_t st = at % F::kK, ph = ((at / F::kK) & 1) ^ 1;
          if (!(ok = wait(&sm.k_empty[st], ph))) break;
          if (p.mask) {  // there before K is, and so before S
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              asm volatile("" : "+r"(next[w]));  // not looked at before
              const uint32_t word = __ballot_sync(0xffffffffu, next[w] != 0);
              if (lane == 0) sm.keys[at % kKeySlots][w] = word;
            }
            if (t + 1 < it.blocks) load_mask(blk);
          }
          if (lane == 0) {
            mbar_expect_tx(&sm.k_full[st], S::kTile);
            for (int c = 0; c < S::kChunks; ++c)
              tma_load_3d(sm.k[st] + c * kChunkBytes, &tm_k, &sm.k_full[st], c * 64, it.hk, it.key0 + x, pol);
          }
          __syncwarp();
          ++at;
          if (!(ok = wait(&sm.v_empty[st], ph))) break;
          if (lane == 0) {
            mbar_expect_tx(&sm.v_full[st], S::kTile);
            for (int c = 0; c < S::kChunks; ++c)
              tma_load_3d(sm.v[st] + c * kChunkBytes, &tm_v, &sm.v_full[st], c * 64, it.hk, it.key0 + x, pol);
          }
          __syncwarp();
          ++sent;
        }
      }
      if (lane == 0) {  // every copy has landed
        for (uint32_t x = nq > F::kQ ? nq - F::kQ : 0; x < nq; ++x) drain(&sm.q_full[x % F::kQ], (x / F::kQ) & 1);
        for (uint32_t x = at > F::kK ? at - F::kK : 0; x < at; ++x) drain(&sm.k_full[x % F::kK], (x / F::kK) & 1);
        for (uint32_t x = sent > F::kV ? sent - F::kV : 0; x < sent; ++x) drain(&sm.v_full[x % F::kV], (x / F::kV) & 1);
      }
    } else if (warp == 2) {
      // ----------------------------------------------------------- item decoder
      uint32_t n = 0, asked = 0;
      bool ok = true;
      for (int u = (int)blockIdx.x; ok;) {
        if (u >= 0) {
          if (lane == 0) next_item_ask(sm.next, asked);
          __syncwarp();
          ++asked;
        }
        Item it{};
        it.hk = -1;
        if (u >= 0) {
          const int at_q = u / p.Hk, split = at_q / prm.slots;
          const Segment g = warp_segment_of_slot(p.cu_q, p.B, p.nq, prm.tpt, at_q - split * prm.slots);
          const int64_t t0 = g.tile * prm.tpt;
          if (t0 < g.n) {  // else an idle slot
            int64_t k0, kn;
            win_keys(prm.w, g.s, k0, kn);
            it.hk = u - at_q * p.Hk;
            it.tok0 = (int)(g.row + t0);
            it.ntok = (int)min((int64_t)prm.tpt, g.n - t0);
            it.p0 = (int)(kn - g.n + t0);
            it.key0 = (int)k0;
            it.split = split;
            it.rg = win_range(it.p0, it.p0 + it.ntok - 1, (int)kn, prm.w.left, prm.w.right, prm.w.sinks);
            const int all = win_blocks<kN>(it.rg), per = (all + p.nsplit - 1) / p.nsplit;
            it.j0 = min(all, per * split);
            it.blocks = min(all, it.j0 + per) - it.j0;
            if (it.blocks == 0) {  // nothing to see: the result at once
              empty_rows<D>(p, it.hk, it.tok0, it.ntok, split, lane);
              it.hk = -1;
            }
          }
        }
        if (u < 0 || it.hk >= 0) {
          const uint32_t s = n % kItemSlots;
          if (!(ok = wait(&sm.item_empty[s], ((n / kItemSlots) & 1) ^ 1))) break;
          if (lane == 0) {
            sm.item[s] = it;
            mbar_arrive(&sm.item_full[s]);
          }
          __syncwarp();
          ++n;
          if (u < 0) break;  // no more items
        }
        if (!(ok = wait(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1))) break;
        u = (int)warp_uniform((uint32_t)next_item_answer(sm.next, asked - 1));
        fence_proxy_async_smem();  // the answer is read before its place is used again
        __syncwarp();
      }
      if (lane == 0 && asked > 0) drain(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1);
    } else if (warp == 3) {
      // ------------------------------------------------- the keys of the V tiles
      uint32_t n = 0, at = 0;
      bool ok = true;
      Item it;
      while (ok && next_item(n, it, ok)) {
        auto keys_of = [&](const Block& b) -> uint32_t {
          return all_keys(b) ? 15u : lane_keys(p.mask, (int64_t)it.key0 + b.x, b.e - b.x, lane);
        };
        Block blk(it.rg, it.j0);
        uint32_t next = keys_of(blk);
        for (int t = 0; t < it.blocks; ++t, ++at) {
          const uint32_t st = at % F::kV, keys = next;
          const bool whole = all_keys(blk);
          blk.next(it.rg);
          if (t + 1 < it.blocks) next = keys_of(blk);  // a block ahead
          if (!(ok = wait(&sm.v_full[st], (at / F::kV) & 1))) break;
          if (!whole) {
            if (!__all_sync(0xffffffffu, keys == 15u)) {
              const uint32_t base = smem_u32(sm.v[st]);
#pragma unroll
              for (int g = 0; g < 4; ++g)
                if (!((keys >> g) & 1u))
                  for (int c = 0; c < 8 * S::kChunks; ++c)
                    st_shared_v4(base + (c >> 3) * kChunkBytes + (g * 32 + lane) * 128 + (((c + lane) & 7) << 4), 0, 0, 0, 0);
              fence_proxy_async_smem();
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.v_ready[st]);
        }
      }
    } else {
      // -------------------------------------------------------------- MMA issuer
      // Converged, and uniform to the compiler: every branch depends on votes and
      // on values made uniform.  Step i issues P V of block i - kS, then S of block
      // i, over whose columns that P lay: the products run in this order.
      constexpr uint32_t idesc_s = idesc_bf16_f32(kM, kN, false, false);
      constexpr uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      constexpr uint32_t kStep = S::kTile >> 4, kFirst = 2, kLast = 4;
      const uint32_t q_lo = desc_lo(smem_u32(sm.q[0]), 16), k_lo = desc_lo(smem_u32(sm.k[0]), 16),
                     v_lo = desc_lo(smem_u32(sm.v[0]), kChunkBytes);
      auto waitq = [&](uint64_t* bar, uint32_t parity) -> bool {
        return quick_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
      };
      uint32_t n = 0, left = 0, qs = F::kQ - 1, qf = 1;           // items taken, blocks left of S's, Q stage
      uint32_t ks = 0, kf = 0, vs = 0, vf = 0, sb = 0, pf = 0, of = 1;  // stages and phases
      uint32_t f0 = 0, f1 = 0;                                    // flags of the blocks of P V; 0: none
      bool ok = true, end = false;
#pragma unroll 1
      do {
        const uint32_t f = F::kS == 2 ? f0 : f1;
        if (f) {
          if (!(ok = waitq(&sm.v_ready[vs], vf))) break;
          if (f & kFirst) {
            if (!(ok = waitq(&sm.o_empty, of))) break;
            of ^= 1;
          }
          if (!(ok = waitq(&sm.p_full[sb], pf))) break;
          tc_fence_after();
          mma_tnh(tmem + F::kO, tmem + sb * kN, v_lo + vs * kStep, idesc_o, (f & kFirst) ^ kFirst);
          mma_commit_w(&sm.pv_done);
          mma_commit_w(&sm.v_empty[vs]);
          if (f & kLast) mma_commit_w(&sm.o_full);
          if (++vs == F::kV) {
            vs = 0;
            vf ^= 1;
          }
          if (sb == F::kS - 1) pf ^= 1;
        }
        uint32_t fn = 0;
        if (left == 0 && !end) {
          const uint32_t s = n % kItemSlots;
          if (!(ok = waitq(&sm.item_full[s], (n / kItemSlots) & 1))) break;
          end = (int)warp_uniform((uint32_t)sm.item[s].hk) < 0;
          left = end ? 0u : warp_uniform((uint32_t)sm.item[s].blocks);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.item_empty[s]);
          ++n;
          if (!end) {
            fn = kFirst;
            if (++qs == F::kQ) {
              qs = 0;
              qf ^= 1;
            }
            if (!(ok = waitq(F::kQt ? &sm.qt_full : &sm.q_full[qs], qf))) break;
          }
        }
        if (left > 0) {
          --left;
          fn |= left == 0 ? 1u | kLast : 1u;
          if (!(ok = waitq(&sm.k_full[ks], kf))) break;
          tc_fence_after();
          if constexpr (F::kQt)
            mma_tk128(tmem + sb * kN, tmem + F::kQc, k_lo + ks * kStep, idesc_s);
          else
            mma_nt<D>(tmem + sb * kN, q_lo + qs * kStep, k_lo + ks * kStep, idesc_s);
          mma_commit_w(&sm.s_full[sb]);
          mma_commit_w(&sm.k_empty[ks]);
          if (left == 0) mma_commit_w(F::kQt ? &sm.qt_empty : &sm.q_empty[qs]);
          if (++ks == F::kK) {
            ks = 0;
            kf ^= 1;
          }
        }
        if (F::kS == 2) sb ^= 1;
        f0 = f1;
        f1 = fn;
      } while (f0 | f1);
      mma_commit_w(&sm.mma_done);  // every MMA has completed before TMEM is freed
      drain(&sm.mma_done, 0);
    }
  } else if (warp < 4 + F::kSoftmax) {
    // ------------------------------------------------------------------- softmax
    if constexpr (F::kCtas == 2) setmaxnreg_inc<F::kRegSoftmax>();
    constexpr int kCols = kN / F::kHalves, kC = F::kCtas == 2 ? 32 : 64;  // of a warp, of a step
    constexpr bool kReload = kC < kCols;
    const uint32_t half = F::kHalves == 2 ? (warp - 4) >> 2 : 0;
    const int rt = token_of(row), rt_first = token_of(quarter * 32), span = token_of(quarter * 32 + 31) - rt_first;
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    uint32_t n = 0, b = 0;  // items, blocks
    bool ok = true;
    Item it;
    while (ok && next_item(n, it, ok)) {
      const int right = it.p0 + rt + prm.w.right, left = it.p0 + rt - prm.w.left;  // last and first key of this row's
      const int right0 = right + rt_first - rt, left0 = left + rt_first - rt;      // and of the warp's first
      float m = -1e30f, l = 0.f, most = 0.f;  // most: what a row's maximum may grow to without a new reference
      Block blk(it.rg, it.j0);
#pragma unroll 1
      for (int t = 0; t < it.blocks; ++t, ++b) {
        const int e = blk.e, x = blk.x + (int)half * kCols;  // of this warp's first column
        blk.next(it.rg);
        const uint32_t sb = b % F::kS, ts = lane_base + sb * kN + half * kCols;
        if (!(ok = wait(&sm.s_full[sb], (b / F::kS) & 1))) break;
        tc_fence_after();
        bool whole = e - x >= kCols;  // every key of this warp's counts
        const uint32_t* const keys = &sm.keys[b % kKeySlots][half * (kCols / 32)];
        if (p.mask) {
          uint32_t all = keys[0];
#pragma unroll
          for (int w = 1; w < kCols / 32; ++w) all &= keys[w];
          whole = all == ~0u;
        }
        // Columns of steps with keys; behind them P is zero.  (d = 64: a causal batch
        // with four first keys 56 -> 48 us, whole blocks 0 to 2% more.  At d = 128 a
        // warp has one step.)  Uniform, and so the compiler's loops.
        const int live = kReload ? (int)warp_uniform((uint32_t)min(kCols, (e - x + kC - 1) / kC * kC)) : kCols;
        const bool limits = right0 - x < kCols - 1 || (left0 + span > x && x + kCols > prm.w.sinks);
        // ---- pass 1
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        uint32_t r[kC];
        auto load = [&](int g) {
#pragma unroll
          for (int y = 0; y < kC; y += 32) tmem_ld32(ts + g + y, *reinterpret_cast<uint32_t(*)[32]>(&r[y]));
        };
#pragma unroll 1
        for (int g = 0; g < live; g += kC) {
          load(g);
          tmem_wait_ld();
          if (!whole || limits) {
            // a bit for each column this row sees: lo .. hi and those below sink
            uint32_t on[kC / 32], some = ~0u;
#pragma unroll
            for (int w = 0; w < kC / 32; ++w) {
              const int first = g + 32 * w, hi = right - x - first, lo = left - x - first, sink = prm.w.sinks - x - first;
              on[w] = (p.mask ? keys[first / 32] : bits_to(e - 1 - x - first)) & bits_to(hi) & (bits_from(lo) | bits_to(sink - 1));
              some &= on[w];
            }
            if (__any_sync(0xffffffffu, some != ~0u)) {
#pragma unroll
              for (int y = 0; y < kC; ++y)
                if (!((on[y / 32] >> (y & 31)) & 1u)) r[y] = 0xff800000u;
              if (kReload) {
#pragma unroll
                for (int y = 0; y < kC; y += 32) tmem_st32(ts + g + y, *reinterpret_cast<uint32_t(*)[32]>(&r[y]));
              }
            }
          }
#pragma unroll
          for (int y = 0; y < kC; y += 8)
#pragma unroll
            for (int z = 0; z < 4; ++z) m4[z] = max3(m4[z], __uint_as_float(r[y + z]), __uint_as_float(r[y + z + 4]));
        }
        if (kReload && (!whole || limits)) tmem_wait_st();
        float mx = fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]) * prm.scale_log2;
        if constexpr (F::kHalves == 2) {
          sm.most[b & 1][half][row] = mx;  // both halves take the same reference
          pair_sync(1 + quarter);
          mx = fmaxf(mx, sm.most[b & 1][half ^ 1][row]);
        }
        mx = fmaxf(mx, -1e30f);  // finite where a row sees no key of the block
        // a partner that gave up leaves infinite maxima: both branches look
        auto given_up = [&]() -> bool { return F::kHalves == 2 && __any_sync(0xffffffffu, *abort_flag); };
        if (t == 0) {
          m = mx;
          most = fminf(m + 8.0f, FLT_MAX);  // two halves: an infinite maximum always asks for one
          if (!(ok = !given_up())) break;
        } else {
          const bool need = mx > (F::kHalves == 2 ? most : m + 8.0f);
          if (__any_sync(0xffffffffu, need)) {  // the same rows in both halves
            if (!(ok = !given_up())) break;
            const float alpha = need ? ex2_approx(m - mx) : 1.0f;
            if (need) {
              m = mx;
              most = fminf(m + 8.0f, FLT_MAX);
            }
            l *= alpha;
            if (!(ok = wait(&sm.pv_done, (b & 1) ^ 1))) break;  // O holds P V up to the block before
            tc_fence_after();
            const uint32_t to = lane_base + F::kO + half * (D / F::kHalves);
#pragma unroll 1
            for (int g = 0; g < D / F::kHalves; g += 16) {
              uint32_t o[16];
              tmem_ld16(to + g, o);
              tmem_wait_ld();
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * alpha);
              tmem_st16(to + g, o);
            }
          }
        }
        // ---- pass 2: loads run beside the exponentials of the columns before
        const uint64_t m2 = pack_f32x2(-m, -m);
        uint64_t sum[4] = {0, 0, 0, 0};
        if (kReload) load(0);
#pragma unroll 1
        for (int g = 0; g < live; g += kC) {
          if (kReload) tmem_wait_ld();
          float a[kC];
#pragma unroll
          for (int y = 0; y < kC; y += 2) unpack_f32x2(fma_f32x2(pack_u32x2(r[y], r[y + 1]), c2, m2), a[y], a[y + 1]);
          if (kReload && g + kC < live) load(g + kC);
          uint32_t pk[kC / 2];
#pragma unroll
          for (int y = 0; y < kC; y += 2) {
            a[y] = ex2_approx(a[y]);
            a[y + 1] = ex2_approx(a[y + 1]);
            sum[(y >> 1) & 3] = add_f32x2(sum[(y >> 1) & 3], pack_f32x2(a[y], a[y + 1]));
            pk[y / 2] = pack_bf16x2(a[y], a[y + 1]);
          }
          if constexpr (kC == 64)
            tmem_st32(ts + g, pk);
          else
            tmem_st16(ts + (g >> 6) * 64 + ((g >> 5) & 1) * 16, pk);
        }
        if constexpr (kReload) {
          const uint32_t none[16] = {};
#pragma unroll 1
          for (int g = live; g < kCols; g += kC) tmem_st16(ts + (g >> 6) * 64 + ((g >> 5) & 1) * 16, none);
        }
        float a0, a1;
        unpack_f32x2(add_f32x2(add_f32x2(sum[0], sum[1]), add_f32x2(sum[2], sum[3])), a0, a1);
        l += a0 + a1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[sb]);
      }
      if (!ok) break;
      // the rows' maximum and sum for the output warps, which have read the last ones
      if (!(ok = wait(&sm.o_empty, n & 1))) break;
      tc_fence_after();
      if (half == 0) tmem_st1(lane_base + F::kMl, __float_as_uint(m));
      tmem_st1(lane_base + F::kMl + 1 + half, __float_as_uint(l));
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.ml_full);
    }
    // A warp that gave up does not keep its partner waiting: it comes to their
    // barrier once more, and its infinite maxima, which are there before, send the
    // partner behind that barrier to the abort flag, not to another barrier.
    if (F::kHalves == 2 && !ok) {
      for (int x = 0; x < 2; ++x) sm.most[x][half][row] = INFINITY;
      __threadfence_block();
      __syncwarp();
      pair_arrive(1 + quarter);
    }
  } else {
    // ------------------------------------------------------------- Q in, O out
    if constexpr (F::kCtas == 2) setmaxnreg_dec<F::kRegOut>();
    const int rt = token_of(row);
    const uint32_t c = lane & 3;
    uint32_t n = 0, done = 0;
    bool ok = true;
    // Q of item i: shared memory (128B-swizzled, as TMA wrote it) -> TMEM, this
    // thread's row, bf16 pairs: the A operand of S = Q K^T
    auto load_q = [&](uint32_t i) -> bool {
      if constexpr (!F::kQt) return true;
      if (!wait(&sm.q_full[0], i & 1)) return false;
      if (!wait(&sm.qt_empty, (i & 1) ^ 1)) return false;
      tc_fence_after();
#pragma unroll 1
      for (int cc = 0; cc < S::kChunks; ++cc) {
        uint32_t qv[32];
        const uint32_t base = smem_u32(sm.q[0]) + cc * kChunkBytes + row * 128;
#pragma unroll
        for (int u = 0; u < 8; ++u)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(qv[4 * u]), "=r"(qv[4 * u + 1]), "=r"(qv[4 * u + 2]), "=r"(qv[4 * u + 3])
                       : "r"(base + ((u ^ (row & 7)) << 4)));
        tmem_st32(lane_base + F::kQc + cc * 32, qv);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sm.qt_full);
        mbar_arrive(&sm.q_empty[0]);
      }
      return true;
    };
    Item it, nx;
    bool more = next_item(n, nx, ok);
    if (more) ok = load_q(0);
    while (ok && more) {
      it = nx;
      more = next_item(n, nx, ok);
      if (!ok || (more && !(ok = load_q(n - 1)))) break;  // the next one's, once this one's last S is done
      if (!(ok = wait(&sm.ml_full, done & 1))) break;
      if (!(ok = wait(&sm.o_full, done & 1))) break;
      ++done;
      tc_fence_after();
      const int64_t tok0 = it.tok0;
      const int h = it.hk * p.G + (int)row - rt * p.G;
      const bool row_ok = rt < it.ntok;
      float m, l, l1 = 0.f;
      m = __uint_as_float(tmem_ld1(lane_base + F::kMl));
      l = __uint_as_float(tmem_ld1(lane_base + F::kMl + 1));
      if (F::kHalves == 2) l1 = __uint_as_float(tmem_ld1(lane_base + F::kMl + 2));
      tmem_wait_ld();
      l += l1;
      if (p.nsplit > 1) {
        const int64_t prow = ((int64_t)it.split * p.nq + tok0 + rt) * p.H + h;
#pragma unroll 1
        for (int g = 0; g < D / 32; ++g) {
          uint32_t r[32];
          tmem_ld32(lane_base + F::kO + g * 32, r);
          tmem_wait_ld();
          if (row_ok) {
#pragma unroll
            for (int x = 0; x < 32; x += 4)
              *reinterpret_cast<uint4*>(p.part_o + prow * D + g * 32 + x) = make_uint4(r[x], r[x + 1], r[x + 2], r[x + 3]);
          }
          __syncwarp();
        }
        if (row_ok) p.part_ml[prow] = make_float2(m, l);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.o_empty);
        continue;
      }
      // A thread holds a row; the four lanes of a quad exchange 16-byte units so
      // that lane c holds unit c of each of the quad's rows, and a store covers 64
      // contiguous bytes of eight rows instead of 16 of 32.
      const float f = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
      uint32_t o[D / 2];
#pragma unroll
      for (int g = 0; g < D / 32; ++g) {  // all of O first: the next item's first P V waits for it
        uint32_t r[32];
        tmem_ld32(lane_base + F::kO + g * 32, r);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; ++x)
          o[g * 16 + x] = pack_bf16x2(__uint_as_float(r[2 * x]) * f, __uint_as_float(r[2 * x + 1]) * f);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.o_empty);
      if (row_ok) p.lse[(int64_t)h * p.nq + tok0 + rt] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      __nv_bfloat16* out[4];
      __nv_bfloat16* const base = static_cast<__nv_bfloat16*>(p.o) + tok0 * p.os + (int64_t)it.hk * p.G * D + c * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = quarter * 32 + (lane & ~3u) + i;
        const int yt = token_of(y);
        out[i] = yt < it.ntok ? base + (int64_t)yt * p.os + (y - yt * p.G) * D : nullptr;
      }
#pragma unroll
      for (int g = 0; g < D / 32; ++g) {
        uint32_t u[4][4];
#pragma unroll
        for (int x = 0; x < 16; ++x) u[x >> 2][x & 3] = o[g * 16 + x];
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
  if (warp == 1) tmem_dealloc(sm.tmem_base, F::kCols);
}

static_assert(sizeof(Smem<128>) <= 232448 && sizeof(Smem<64>) <= 114 * 1024, "shared layout exceeds the block limit");

template <int D>
cudaError_t launch_d(const Params& prm, const CUtensorMap* tm, cudaStream_t s) {
  const size_t smem = sizeof(Smem<D>);
  cudaError_t e = cudaFuncSetAttribute(wattn_fwd_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // the setmaxnreg split assumes exactly kRegLaunch registers per thread at
  // launch: with fewer, the increases would wait for registers that never come
  if (Form<D>::kCtas == 2) {
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, wattn_fwd_tc_kernel<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs != Form<D>::kRegLaunch) return cudaErrorInvalidConfiguration;
  }
  wattn_fwd_tc_kernel<D><<<(unsigned)prm.n_items, Form<D>::kThreads, smem, s>>>(tm[0], tm[1], tm[2], prm);
  return cudaGetLastError();
}

}  // namespace

int64_t wattn_fwd_tc_items(const WinParams& w) { return segment_slots(w.x.nq, w.x.B, kM / w.x.G) * w.x.Hk; }

// Parts of the keys of a tile: of one, of as many as fill one to four waves of CTAs,
// and of fewer and longer ones, what takes least by this count: a wave lasts as long
// as an item's blocks and two more, joining n parts as long as 4 + n / 2.  (4 queries of 24 heads of
// 128 over 1,024 keys each: 28 us in three parts, 24 whole; of 24 / 8 heads of 64:
// 20 in parts, 24 whole.)  The blocks are those of n_k / n_seg rows, as far as a
// tile sees them: of caches their capacity, for how far they are filled is not
// known on the host.
int wattn_fwd_tc_splits(const WinParams& w) {
  const XattnParams& p = w.x;
  const int64_t items = wattn_fwd_tc_items(w), ctas = (int64_t)p.sms * (p.d == 64 ? Form<64>::kCtas : Form<128>::kCtas);
  const int64_t near = (int64_t)w.left + w.right + w.sinks + kM / p.G, rows = p.nk / p.B;
  const int64_t blocks = std::max<int64_t>(1, (std::min(near, rows) + kN - 1) / kN);
  int64_t least = 2 * ((items + ctas - 1) / ctas * (blocks + 2)), want = 1;
  for (int v = 1; v <= 4; ++v) {
    const int64_t most = std::min<int64_t>(std::min<int64_t>(v * ctas / items, blocks), 1024);
    if (most < 2) continue;
    for (int64_t each = (blocks + most - 1) / most; each < blocks; each += (each + 1) / 2) {
      const int64_t n = (blocks + each - 1) / each;  // the fewest parts of that length
      const int64_t time = 2 * ((n * items + ctas - 1) / ctas * (each + 2) + 4) + n;
      if (time >= least) continue;
      least = time;
      want = n;
    }
  }
  return (int)want;
}

cudaError_t launch_wattn_fwd_tc(const WinParams& w, cudaStream_t s) {
  const XattnParams& p = w.x;
  Params prm{};
  prm.w = w;
  prm.inv_g = (65536u + p.G - 1) / p.G;
  prm.tpt = kM / p.G;
  prm.slots = (int)segment_slots(p.nq, p.B, prm.tpt);
  prm.n_items = (int64_t)prm.slots * p.Hk * p.nsplit;
  prm.scale_log2 = p.scale * kLog2e;
  prm.keep_kv = prm.slots > p.B;
  CUtensorMap tm[3];
  // an empty side has no tensor to describe: its map is never used
  const void* k = p.nk > 0 ? p.k : p.q;
  const void* v = p.nk > 0 ? p.v : p.q;
  const int64_t ks = p.nk > 0 ? p.ks : p.qs, vs = p.nk > 0 ? p.vs : p.qs, nk = p.nk > 0 ? p.nk : 1;
  if (!encode_tmap_heads_bf16(&tm[0], p.q, p.d, p.H, p.nq, p.qs * 2, p.G, prm.tpt) ||
      !encode_tmap_heads_bf16(&tm[1], k, p.d, p.Hk, nk, ks * 2, 1, kN) ||
      !encode_tmap_heads_bf16(&tm[2], v, p.d, p.Hk, nk, vs * 2, 1, kN))
    return cudaErrorInvalidValue;
  return p.d == 64 ? launch_d<64>(prm, tm, s) : launch_d<128>(prm, tm, s);
}

}  // namespace ut
