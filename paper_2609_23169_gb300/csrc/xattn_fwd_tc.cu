// Cross attention to an encoder's states, forward, on the 5th-generation
// tensor cores (bf16 in, fp32 accumulate):
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
// over the keys j of query i's segment whose mask is set.
//
// A query tile holds 128 rows: the G heads that share a kv head of 128 / G
// consecutive tokens of one segment (row = token * G + head; one TMA box), so
// that K and V are read once for the group.  A work item is T such tiles, one
// kv head and one range of key blocks; the tiles share every K and V tile in
// shared memory, and while one tile's softmax runs the others' products do.
// T = 2 and blocks of 128 keys at d = 128, T = 4 and 64 keys at d = 64: either
// fills tensor memory with S and O.  (Two tiles at d = 64 too: 89 us instead of
// 71 for 23,959 x 257 x 24, the softmax warps wait for products 1,000 of 2,700
// cycles a block.)
//
// One CTA per SM, which takes item after item (NextItem); items with the head
// fastest, so that CTAs in flight read neighbouring 256-byte pieces of the same
// rows and share K and V in L2.  Roles (128 + 128 T threads; with T = 2
// registers rebalanced with setmaxnreg):
//   warp 0      TMA: the K and V tiles, one ring (K0 V0 K1 V1 ...); leaves
//               beside a V tile which of its keys count
//   warp 2      asks for the items and decodes them (segment search, key
//               range) into a ring; TMA: the query tiles, a ring of their own
//   warp 1      TMEM owner and MMA issuer of the even tiles, warp 3 of the odd
//               ones: per block S = Q K^T, then, as P is written over S in TMEM,
//               O += P V.  With T = 2 that product begins with the first 96
//               keys while P of the last 32 is being written, and the issuers
//               take turns (P V and the next S of one tile together), else the
//               tensor core mixes the two tiles' instructions, both finish late,
//               and both softmaxes then run at once with the tensor core idle.
//               Their code is fetched anew each time and kept short for that:
//               the part of a wait that spins is called (431 -> 400 us for
//               85,202 x 512 x 24 x 128).
//   warps 4...  softmax, four warps a tile: thread = row = TMEM lane.  Read S
//               from TMEM, mask, keep a running maximum (O is rescaled in TMEM
//               only where it grew by more than 2^8, so the exponentials stay
//               bounded), write P as bf16 over S; after the last block O / l and
//               LSE, or the split's partial result.
// Masked keys and the rows of other segments: S there becomes -inf, the
// smaller of S and a bias of +-inf that warp 0 leaves in shared memory (the
// min of NaN and -inf is -inf; selecting by bits of the mask took 900 to 1,300
// cycles a block, this takes 400), and those rows of the V tile become zero
// before its products (by warp 0 or the softmax warps), so that no value they
// hold (NaN, infinities) is multiplied.
// Rounding: P to bf16 for its product (the sum l is of the unrounded values),
// O once at the end.
// Measured: 85,202 x 512 x 24 x 128 430 us a pass among others, 1,250 TFLOP/s,
// 0.66 of the card's bf16 rate (390 us for the first twenty, before the power
// cap holds), bound by the softmax between the products (tensor pipe active
// 58%); 23,959 x 257 x 24 x 64 66 us; one query over 85,202 keys, 24 heads of
// 128, 155 us, 6.7 TB/s.
// Every wait is bounded; on expiry the kernel records UT_ERR_TIMEOUT, drains
// its own copies and MMAs, frees TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "xattn_tc.cuh"

namespace ut {

namespace {

constexpr int kM = 128;  // rows of a query tile
// Registers of the two-tile form (384 threads)
constexpr int kRegLaunch = 168, kRegCtl = 120, kRegSoftmax = 192;  // per thread; setmaxnreg split
static_assert(kRegCtl + 2 * kRegSoftmax <= 3 * kRegLaunch, "the split must fit the launch's registers");
constexpr uint32_t kChunkBytes = kM * 128;  // 128 rows x 64 bf16
constexpr int kItemSlots = 3;  // no more are taken ahead: other CTAs may be idle

// Two tiles and blocks of 128 keys at d = 128, four and 64 at d = 64: the
// tiles' S and O fill tensor memory either way.
template <int D>
struct Form {
  static constexpr int kTiles = D == 128 ? 2 : 4;
  static constexpr int kN = D == 128 ? 128 : 64;       // keys of a block
  static constexpr int kThreads = 128 + 128 * kTiles;
};

struct Item {
  int32_t hk;      // kv head; -1: no more items
  int32_t blocks;  // key blocks of this item (0: write the empty result)
  int32_t tok0;    // first token of tile 0
  int32_t ntok;    // tokens of all tiles (the last ones may be empty)
  int32_t key0;    // first key
  int32_t left;    // keys from key0 to the end of the segment
  int32_t split;
};

template <int D>
struct Smem {
  static constexpr int kChunks = D / 64, T = Form<D>::kTiles, kN = Form<D>::kN;
  static constexpr uint32_t kTile = kM * D * 2, kKvTile = kN * D * 2, kKvChunk = kN * 128;
  static constexpr int kQ = D == 128 ? 3 : 8;   // query tiles in flight
  static constexpr int kKv = D == 128 ? 4 : 8;  // K and V tiles in flight
  alignas(1024) uint8_t q[kQ][kTile];
  alignas(1024) uint8_t kv[kKv][kKvTile];
  float bias[kKv / 2][kN];                // of the keys of a V tile: 0 < bias = attend
  alignas(16) uint32_t keys[kKv / 2][4];  // and as bits
  uint64_t q_full[kQ], q_empty[kQ], kv_full[kKv], kv_empty[kKv], keys_full[kKv / 2], v_ready[kKv / 2];
  uint64_t s_full[T], p_most[T], p_full[T], o_full[T], o_empty[T], turn[2], mma_done;
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  Item item[kItemSlots];
  NextItem next;
  uint32_t tmem_base;
  int abort_flag;
};

struct Params {
  XattnParams x;
  uint32_t inv_g;    // ceil(2^16 / G): (r * inv_g) >> 16 = r / G for r < 128, G <= 64
  int tpt;           // tokens of a tile
  int slots;         // item slots along the query rows
  int64_t n_items;   // slots * Hk * nsplit
  float scale_log2;
  bool keep_kv;      // K and V are read by several items: keep them in L2
};

template <int D>
__global__ void __launch_bounds__(Form<D>::kThreads, 1)
    xattn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const Params prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
  using S = Smem<D>;
  constexpr int T = S::T, kN = S::kN, kGroups = kN / 32;
  // who zeroes rows of V: warp 0, two blocks behind its loads, where four blocks
  // are in flight (four tiles); else the softmax warps
  constexpr bool kZeroes = T == 4;
  // TMEM columns of tile t: S and P at t kN, O at 256 + t D
  static_assert(T * kN <= 256 && 256 + T * D <= 512, "tensor memory");
  const XattnParams& p = prm.x;
  const uint32_t warp = warp_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, UT_ERR_INVALID_ARG);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kQ; ++s) {
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_empty[s], 1);
    }
    for (int s = 0; s < S::kKv; ++s) {
      mbar_init(&sm.kv_full[s], 1);
      mbar_init(&sm.kv_empty[s], 2);  // both issuers' products
      if (s % 2 == 0) {
        mbar_init(&sm.keys_full[s / 2], 1);
        mbar_init(&sm.v_ready[s / 2], 1);
      }
    }
    for (int w = 0; w < 2; ++w) mbar_init(&sm.turn[w], 1);
    for (int w = 0; w < T; ++w) {
      mbar_init(&sm.s_full[w], 1);
      mbar_init(&sm.p_most[w], 4);
      mbar_init(&sm.p_full[w], 4);
      mbar_init(&sm.o_full[w], 1);
      mbar_init(&sm.o_empty[w], 4);
    }
    mbar_init(&sm.mma_done, 2);
    for (int s = 0; s < kItemSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], 3 + 4 * T);  // warps 0, 1, 3 and the softmax warps
    }
    next_item_init(sm.next);
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  if (blockIdx.x == 0) {
    check_cu(p.cu_q, p.B, p.nq, p.status);
    check_cu(p.cu_k, p.B, p.nk, p.status);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // all 512 columns are this CTA's, so they start at address 0, a constant in
  // the instructions below
  if (sm.tmem_base != 0 && threadIdx.x == 0) {
    set_status(p.status, UT_ERR_CUDA);
    sm.abort_flag = 1;
  }

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

  // whether a block with `left` keys to the end of its segment needs no masking
  auto all_keys = [&](int left) { return !p.mask && left >= kN; };

  if (warp < 4) {
    if constexpr (T == 2) setmaxnreg_dec<kRegCtl>();
    if (warp == 0) {
      // ------------------------------------------------------- K, V producer
      if (lane == 0) {
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
      }
      const uint64_t pol = prm.keep_kv ? policy_evict_last() : policy_evict_first();
      uint32_t n = 0, at = 0, ready = 0;         // tiles asked for, V tiles made ready
      uint32_t waiting = 0, older = 0, newer = 0;  // V tiles to be made ready (two at most), their keys
      bool ok = true;
      Item it;
      auto make_ready = [&]() {  // the next V tile, once it is there
        const uint32_t st = (2 * ready + 1) % S::kKv;
        if (!(ok = wait(&sm.kv_full[st], (2 * ready / S::kKv) & 1))) return;
        const uint32_t keys = waiting == 2 ? older : newer;
        if (!__all_sync(0xffffffffu, keys == 15u)) {
          const uint32_t base = smem_u32(sm.kv[st]);
#pragma unroll
          for (int g = 0; g < kGroups; ++g)
            if (!((keys >> g) & 1u))
              for (int x = 0; x < 8 * S::kChunks; ++x)
                st_shared_v4(base + (x >> 3) * S::kKvChunk + (g * 32 + lane) * 128 + (((x + lane) & 7) << 4), 0, 0, 0, 0);
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(&sm.v_ready[st / 2]);
        ++ready;
        --waiting;
      };
      while (ok && next_item(n, it, ok)) {
        auto keys_of = [&](int j) -> uint32_t {
          if (all_keys(it.left - j * kN)) return 15u;
          return lane_keys(p.mask, (int64_t)it.key0 + j * kN, it.left - j * kN, lane);
        };
        uint32_t next = it.blocks > 0 ? keys_of(0) : 0;
        for (int j = 0; j < it.blocks && ok; ++j) {
          const bool plain = all_keys(it.left - j * kN);
          const uint32_t keys = next;
          if (j + 1 < it.blocks) next = keys_of(j + 1);  // a block ahead
#pragma unroll 1
          for (int which = 0; which < 2; ++which, ++at) {
            const uint32_t st = at % S::kKv;
            if (which && waiting == 2) make_ready();
            if (!ok || !(ok = wait(&sm.kv_empty[st], ((at / S::kKv) & 1) ^ 1))) break;
            if (which && !plain) {
#pragma unroll
              for (int g = 0; g < kGroups; ++g) {
                const bool on = (keys >> g) & 1u;
                const uint32_t word = __ballot_sync(0xffffffffu, on);
                sm.bias[st / 2][g * 32 + lane] = on ? INFINITY : -INFINITY;
                if (lane == 0) sm.keys[st / 2][g] = word;
              }
              __syncwarp();
            }
            if (lane == 0) {
              if (which) mbar_arrive(&sm.keys_full[st / 2]);
              mbar_expect_tx(&sm.kv_full[st], S::kKvTile);
              const void* tm = which ? static_cast<const void*>(&tm_v) : static_cast<const void*>(&tm_k);
              for (int c = 0; c < S::kChunks; ++c)
                tma_load_3d(sm.kv[st] + c * S::kKvChunk, tm, &sm.kv_full[st], c * 64, it.hk, it.key0 + j * kN, pol);
            }
            __syncwarp();
          }
          older = newer;
          newer = keys;
          if constexpr (kZeroes) ++waiting;
        }
        while (ok && waiting > 0) make_ready();  // nothing may be left waiting for the next item
      }
      if (lane == 0)
        for (uint32_t x = at > S::kKv ? at - S::kKv : 0; x < at; ++x) drain(&sm.kv_full[x % S::kKv], (x / S::kKv) & 1);
    } else if (warp == 2) {
      // ------------------------------------------- item decoder, Q producer
      if (lane == 0) tma_prefetch_desc(&tm_q);
      const uint64_t pol = policy_evict_first();
      const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kChunks;
      uint32_t n = 0, at = 0, asked = 0;
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
          const Segment g = warp_segment_of_slot(p.cu_q, p.B, p.nq, T * prm.tpt, at_q - split * prm.slots);
          const int64_t t0 = g.tile * T * prm.tpt;
          int64_t k0, kn;
          segment_rows(p.cu_k, g.s, p.nk, k0, kn);
          const int nblk = (int)((kn + kN - 1) / kN), per = (nblk + p.nsplit - 1) / p.nsplit;
          const int b0 = min(nblk, per * split), b1 = min(nblk, b0 + per);
          it.split = split;
          if (t0 < g.n) it.hk = u - at_q * p.Hk;  // else an idle slot
          it.blocks = b1 - b0;
          it.tok0 = (int)(g.row + t0);
          it.ntok = (int)min((int64_t)T * prm.tpt, g.n - t0);
          it.key0 = (int)(k0 + (int64_t)b0 * kN);
          it.left = (int)(kn - (int64_t)b0 * kN);
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
          const int tiles = it.blocks == 0 ? 0 : (it.ntok + prm.tpt - 1) / prm.tpt;
          for (int w = 0; w < tiles; ++w, ++at) {
            const uint32_t st = at % S::kQ;
            if (!(ok = wait(&sm.q_empty[st], ((at / S::kQ) & 1) ^ 1))) break;
            if (lane == 0) {
              mbar_expect_tx(&sm.q_full[st], bytes);
              for (int c = 0; c < S::kChunks; ++c)
                tma_load_3d(sm.q[st] + c * kChunkBytes, &tm_q, &sm.q_full[st], c * 64, it.hk * p.G,
                            it.tok0 + w * prm.tpt, pol);
            }
            __syncwarp();
          }
          if (!ok) break;
        }
        if (!(ok = wait(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1))) break;
        u = (int)warp_uniform((uint32_t)next_item_answer(sm.next, asked - 1));
        fence_proxy_async_smem();  // the answer is read before its place is used again
        __syncwarp();
      }
      if (lane == 0 && asked > 0) drain(&sm.next.full[(asked - 1) & 1], ((asked - 1) >> 1) & 1);
      if (lane == 0)
        for (uint32_t x = at > S::kQ ? at - S::kQ : 0; x < at; ++x) drain(&sm.q_full[x % S::kQ], (x / S::kQ) & 1);
    } else if (warp == 1 || warp == 3) {
      // ------------------- MMA issuer of the even tiles (warp 1) / the odd ones
      // Converged, and uniform to the compiler: every branch depends on votes
      // and on item fields made uniform.
      constexpr uint32_t idesc_s = idesc_bf16_f32(kM, kN, false, false);
      constexpr uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      constexpr uint32_t kQStep = S::kTile >> 4, kKvStep = S::kKvTile >> 4;
      const uint32_t q_lo = desc_lo(smem_u32(sm.q[0]), 16), k_lo = desc_lo(smem_u32(sm.kv[0]), 16),
                     v_lo = desc_lo(smem_u32(sm.kv[0]), S::kKvChunk);
      auto waitq = [&](uint64_t* bar, uint32_t parity) -> bool {
        return quick_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
      };
      const uint32_t w = warp >> 1;
      uint32_t n = 0, qat = 0, kvat = 0, np = 0, no = 0, turns = 0;  // np, no: phases, a bit per tile
      bool ok = true;
      for (;; ++n) {
        const uint32_t slot = n % kItemSlots;
        if (!(ok = waitq(&sm.item_full[slot], (n / kItemSlots) & 1))) break;
        const int hk = (int)warp_uniform((uint32_t)sm.item[slot].hk);
        const int blocks = (int)warp_uniform((uint32_t)sm.item[slot].blocks);
        const uint32_t tiles = warp_uniform((uint32_t)((sm.item[slot].ntok + prm.tpt - 1) / prm.tpt));
        if (hk < 0) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
        if (blocks == 0) continue;
        if (w >= tiles) {  // nothing for this warp's tiles: pass the K and V tiles on
#pragma unroll 1
          for (int x = 0; x < 2 * blocks && ok; ++x, ++kvat) {
            ok = waitq((x & 1) && kZeroes ? &sm.v_ready[kvat % S::kKv / 2] : &sm.kv_full[kvat % S::kKv],
                       (kvat / S::kKv) & 1);
            if (ok && lane == 0) mbar_arrive(&sm.kv_empty[kvat % S::kKv]);
          }
          if (!ok) break;
          qat += tiles;
          continue;
        }
        const uint32_t q0 = (qat + w) % S::kQ, q0_phase = (qat + w) / S::kQ & 1;  // of the first of its tiles
        // step j: O += P V of block j - 1, S = Q K^T of block j
#pragma unroll 1
        for (int j = 0; j <= blocks; ++j) {
          const uint32_t ks = kvat % S::kKv, vs = (kvat - 1) % S::kKv;
          if (j < blocks && !(ok = waitq(&sm.kv_full[ks], (kvat / S::kKv) & 1))) break;
          if (j > 0 && !(ok = waitq(kZeroes ? &sm.v_ready[vs / 2] : &sm.kv_full[vs], ((kvat - 1) / S::kKv) & 1))) break;
#pragma unroll 1
          for (uint32_t t = w; t < tiles; t += 2) {
            const uint32_t ts = t * kN, to = 256 + t * D, qs = T == 2 ? q0 : (qat + t) % S::kQ;
            const bool last = T == 2 || t + 2 >= tiles;  // of this warp's tiles
            if (j == 0 && !(ok = waitq(&sm.q_full[qs], T == 2 ? q0_phase : ((qat + t) / S::kQ) & 1))) break;
            if (j == 1) {
              if (!(ok = waitq(&sm.o_empty[t], ((no >> t) & 1) ^ 1))) break;
              no ^= 1u << t;
            }
            if (j > 0 && !(ok = waitq(T == 2 ? &sm.p_most[t] : &sm.p_full[t], (np >> t) & 1))) break;
            // an item's first S and its last P V wait for no turn: the tiles need
            // not start or end together
            const bool turn = T == 2 && tiles == 2 && j > 0 && j < blocks;
            if (turn) {
              if (!(ok = waitq(&sm.turn[w], (turns & 1) ^ (w ^ 1)))) break;
              ++turns;
            }
            tc_fence_after();
            if (j > 0) {
              const uint32_t v_b = v_lo + vs * kKvStep;
              if constexpr (T == 2) {
                mma_tn<96>(to, ts, v_b, idesc_o, j > 1);
                if (!(ok = waitq(&sm.p_full[t], (np >> t) & 1))) break;
                tc_fence_after();
                mma_tn<32>(to, ts + 48, v_b + 768, idesc_o, 1);
              } else {
                mma_tn<64>(to, ts, v_b, idesc_o, j > 1);
              }
              np ^= 1u << t;
              if (last) mma_commit_w(&sm.kv_empty[vs]);
              if (j == blocks) mma_commit_w(&sm.o_full[t]);
            }
            if (j < blocks) {
              mma_nt<D>(ts, q_lo + qs * kQStep, k_lo + ks * kKvStep, idesc_s);
              mma_commit_w(&sm.s_full[t]);
              if (last) mma_commit_w(&sm.kv_empty[ks]);
              if (j == blocks - 1) mma_commit_w(&sm.q_empty[qs]);
            }
            if (turn) {
              __syncwarp();
              if (lane == 0) mbar_arrive(&sm.turn[w ^ 1]);
            }
            if constexpr (T == 2) break;
          }
          if (!ok) break;
          if (j < blocks) kvat += 2;
        }
        if (!ok) break;
        qat += tiles;
      }
      mma_commit_w(&sm.mma_done);  // every MMA has completed before TMEM is freed
      drain(&sm.mma_done, 0);
    }
  } else {
    // ----------------------------------------------------------------- softmax
    if constexpr (T == 2) setmaxnreg_inc<kRegSoftmax>();
    const int w = (int)(warp >> 2) - 1;  // its tile
    const uint32_t quarter = warp & 3, lane_base = (quarter * 32) << 16;
    const uint32_t ts = lane_base + w * kN, to = lane_base + 256 + w * D;
    auto token_of = [&](uint32_t r) -> uint32_t { return (r * prm.inv_g) >> 16; };  // r / G
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    const uint32_t row = quarter * 32 + lane, rt = token_of(row);  // this thread's row and its token
    uint32_t n = 0, ns = 0, no = 0, kvat = 0;
    bool ok = true;
    for (;; ++n) {
      // the item stays in its slot until this tile is done with it
      const uint32_t slot = n % kItemSlots;
      if (!(ok = wait(&sm.item_full[slot], (n / kItemSlots) & 1))) break;
      const volatile Item* it = &sm.item[slot];
      if (it->hk < 0) break;
      const int ntok = min(prm.tpt, it->ntok - w * prm.tpt);  // of this tile
      const int blocks = ntok > 0 ? it->blocks : 0;
      float m = -1e30f, l = 0.f;
      for (int j = 0; j < blocks; ++j) {
        const bool plain = all_keys(it->left - j * kN);
        const uint32_t vat = kvat + 2 * j + 1, vst = vat % S::kKv;
        if (!(ok = wait(&sm.s_full[w], ns & 1))) break;
        ++ns;
        tc_fence_after();
        uint32_t r[kN];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) tmem_ld32(ts + g * 32, *reinterpret_cast<uint32_t(*)[32]>(&r[g * 32]));
        if (!plain) {
          ok = wait(kZeroes ? &sm.keys_full[vst / 2] : &sm.kv_full[vst], (vat / S::kKv) & 1);
          if constexpr (!kZeroes) {  // thread = row; the other tile's warps may write the same zeros
            if (ok && !((sm.keys[vst / 2][quarter] >> lane) & 1u)) {
              const uint32_t v_row = smem_u32(sm.kv[vst]) + (quarter * 32 + lane) * 128;
#pragma unroll
              for (int x = 0; x < 8 * S::kChunks; ++x)
                st_shared_v4(v_row + (x >> 3) * S::kKvChunk + (((x + lane) & 7) << 4), 0, 0, 0, 0);
            }
            fence_proxy_async_smem();
          }
        }
        tmem_wait_ld();
        if (!ok) break;
        if (!plain) {
          const uint4 word = *reinterpret_cast<const uint4*>(sm.keys[vst / 2]);
          if ((word.x & word.y & (kGroups == 4 ? word.z & word.w : ~0u)) != 0xffffffffu) {
#pragma unroll
            for (int x = 0; x < kN; x += 4) {
              const float4 b = *reinterpret_cast<const float4*>(sm.bias[vst / 2] + x);
              r[x] = __float_as_uint(fminf(__uint_as_float(r[x]), b.x));
              r[x + 1] = __float_as_uint(fminf(__uint_as_float(r[x + 1]), b.y));
              r[x + 2] = __float_as_uint(fminf(__uint_as_float(r[x + 2]), b.z));
              r[x + 3] = __float_as_uint(fminf(__uint_as_float(r[x + 3]), b.w));
            }
          }
        }
        float m8[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) m8[x] = fmaxf(__uint_as_float(r[x]), __uint_as_float(r[x + 8]));
#pragma unroll
        for (int x = 16; x < kN; x += 16)
#pragma unroll
          for (int y = 0; y < 8; ++y) m8[y] = max3(m8[y], __uint_as_float(r[x + y]), __uint_as_float(r[x + y + 8]));
        float mx = max3(max3(m8[0], m8[1], m8[2]), max3(m8[3], m8[4], m8[5]), fmaxf(m8[6], m8[7]));
        mx = fmaxf(mx * prm.scale_log2, -1e30f);  // finite where a row sees no key of the block
        const bool need = j > 0 && mx > m + 8.0f;
        if (j == 0) m = mx;
        if (__any_sync(0xffffffffu, need)) {
          // S of this block was issued after O += P V of the previous one, so
          // that product has completed
          const float alpha = need ? ex2_approx(m - mx) : 1.0f;
          if (need) m = mx;
          l *= alpha;
#pragma unroll 1
          for (int g = 0; g < D / 16; ++g) {
            uint32_t o[16];
            tmem_ld16(to + g * 16, o);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
            tmem_st16(to + g * 16, o);
          }
        }
        const uint64_t m2 = pack_f32x2(-m, -m);
        uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          uint32_t pk[16];
#pragma unroll
          for (int x = 0; x < 32; x += 2) {
            float p0, p1;
            unpack_f32x2(fma_f32x2(pack_u32x2(r[g * 32 + x], r[g * 32 + x + 1]), c2, m2), p0, p1);
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
            sum[(x >> 1) & 3] = add_f32x2(sum[(x >> 1) & 3], pack_f32x2(p0, p1));
            pk[x / 2] = pack_bf16x2(p0, p1);
          }
          tmem_st16(ts + g * 16, pk);
          if (T == 2 && g == 2) {  // three quarters of P: its product may begin
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.p_most[w]);
          }
        }
        float a0, a1;
        unpack_f32x2(add_f32x2(add_f32x2(sum[0], sum[1]), add_f32x2(sum[2], sum[3])), a0, a1);
        l += a0 + a1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[w]);
      }
      if (!ok) break;
      if (blocks > 0) {
        if (!(ok = wait(&sm.o_full[w], no & 1))) break;
        ++no;
        tc_fence_after();
      }
      const int hk = it->hk, split = it->split;
      const int64_t tok0 = (int64_t)it->tok0 + w * prm.tpt;
      kvat += 2 * it->blocks;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
      if (ntok <= 0) continue;
      const int h = hk * p.G + (int)(row - rt * p.G);
      const bool row_ok = (int)rt < ntok;
      if (p.nsplit > 1) {
        const int64_t prow = ((int64_t)split * p.nq + tok0 + rt) * p.H + h;
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
          uint32_t r[32];
          if (blocks > 0) {
            tmem_ld32(to + g * 32, r);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) r[x] = 0;
          }
          if (!row_ok) continue;
#pragma unroll
          for (int x = 0; x < 32; x += 4)
            *reinterpret_cast<uint4*>(p.part_o + prow * D + g * 32 + x) =
                make_uint4(r[x], r[x + 1], r[x + 2], r[x + 3]);
        }
        if (row_ok) p.part_ml[prow] = make_float2(m, l);
        tc_fence_before();
        __syncwarp();
        if (blocks > 0 && lane == 0) mbar_arrive(&sm.o_empty[w]);
        continue;
      }
      if (row_ok) p.lse[(int64_t)h * p.nq + tok0 + rt] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      // O / l in bf16.  A thread holds a row; the four lanes of a quad exchange
      // 16-byte units so that lane c holds unit c of each of the quad's rows, and
      // a store covers 64 contiguous bytes of eight rows instead of 16 of 32.
      const float f = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
      const uint32_t c = lane & 3;
      __nv_bfloat16* out[4];
      __nv_bfloat16* const base = static_cast<__nv_bfloat16*>(p.o) + tok0 * p.os + (int64_t)hk * p.G * D + c * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = quarter * 32 + (lane & ~3u) + i, yt = token_of(y);
        out[i] = (int)yt < ntok ? base + (int64_t)yt * p.os + (y - yt * p.G) * D : nullptr;
      }
#pragma unroll 1
      for (int g = 0; g < D / 32; ++g) {
        uint32_t u[4][4];
        if (blocks > 0) {
          uint32_t r[32];
          tmem_ld32(to + g * 32, r);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 16; ++x)
            u[x >> 2][x & 3] = pack_bf16x2(__uint_as_float(r[2 * x]) * f, __uint_as_float(r[2 * x + 1]) * f);
        } else {
#pragma unroll
          for (int x = 0; x < 16; ++x) u[x >> 2][x & 3] = 0;
        }
        if (g == D / 32 - 1) {
          tc_fence_before();
          __syncwarp();
          if (blocks > 0 && lane == 0) mbar_arrive(&sm.o_empty[w]);
        }
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

static_assert(sizeof(Smem<128>) <= 232448 && sizeof(Smem<64>) <= 232448, "shared layout exceeds the block limit");

template <int D>
cudaError_t launch_d(const Params& prm, const CUtensorMap* tm, cudaStream_t s) {
  const size_t smem = sizeof(Smem<D>);
  cudaError_t e = cudaFuncSetAttribute(xattn_fwd_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // the setmaxnreg split assumes exactly kRegLaunch registers per thread at
  // launch: with fewer, the increases would wait for registers that never come
  if (Form<D>::kTiles == 2) {
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, xattn_fwd_tc_kernel<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs != kRegLaunch) return cudaErrorInvalidConfiguration;
  }
  xattn_fwd_tc_kernel<D><<<(unsigned)prm.n_items, Form<D>::kThreads, smem, s>>>(tm[0], tm[1], tm[2], prm);
  return cudaGetLastError();
}

}  // namespace

static int tiles_of_item(int d) { return d == 64 ? Form<64>::kTiles : Form<128>::kTiles; }

int64_t xattn_fwd_tc_items(const XattnParams& p) {
  return segment_slots(p.nq, p.B, tiles_of_item(p.d) * (kM / p.G)) * p.Hk;
}

cudaError_t launch_xattn_fwd_tc(const XattnParams& p, cudaStream_t s) {
  Params prm{};
  prm.x = p;
  prm.inv_g = (65536u + p.G - 1) / p.G;
  prm.tpt = kM / p.G;
  prm.slots = (int)segment_slots(p.nq, p.B, tiles_of_item(p.d) * prm.tpt);
  prm.n_items = (int64_t)prm.slots * p.Hk * p.nsplit;
  prm.scale_log2 = p.scale * kLog2e;
  prm.keep_kv = prm.slots > p.B;
  CUtensorMap tm[3];
  // an empty side has no tensor to describe: its map is never used
  const void* k = p.nk > 0 ? p.k : p.q;
  const void* v = p.nk > 0 ? p.v : p.q;
  const int64_t ks = p.nk > 0 ? p.ks : p.qs, vs = p.nk > 0 ? p.vs : p.qs, nk = p.nk > 0 ? p.nk : 1;
  const int kN = p.d == 64 ? Form<64>::kN : Form<128>::kN;
  if (!encode_tmap_heads_bf16(&tm[0], p.q, p.d, p.H, p.nq, p.qs * 2, p.G, prm.tpt) ||
      !encode_tmap_heads_bf16(&tm[1], k, p.d, p.Hk, nk, ks * 2, 1, kN) ||
      !encode_tmap_heads_bf16(&tm[2], v, p.d, p.Hk, nk, vs * 2, 1, kN))
    return cudaErrorInvalidValue;
  return p.d == 64 ? launch_d<64>(prm, tm, s) : launch_d<128>(prm, tm, s);
}

}  // namespace ut
