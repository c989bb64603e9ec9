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
// the windows of neighbouring tiles in L2.  Roles (256 threads):
//   warp 0      TMA: Q, K and V tiles, a ring each
//   warp 1      TMEM owner and MMA issuer: S = Q K^T, O += P V.  The products
//               follow one another across items: the next item's first S is
//               computed while this one's last blocks are in the softmax.
//   warp 2      asks for the items and decodes them into a ring
//   warp 3      which keys of a block count: a bias for S, and the rows of the V
//               tile that do not become zero, so that no value they hold (NaN,
//               infinities) is multiplied
//   warps 4-7   softmax: thread = row = TMEM lane.  Read S, apply the keys' bias
//               and the row's own limits (only in blocks where some row of the
//               warp has one), keep a running maximum (O is rescaled in TMEM only
//               where it grew by more than 2^8, so the exponentials stay
//               bounded), write P as bf16; O / l and LSE (or the split's partial
//               result) of an item are written after the first block of the next.
// d = 128: one CTA an SM, two S buffers, Q copied to TMEM by the softmax warps
// (S = Q K^T then reads only K from shared memory).  TMEM columns S0 [0,128),
// S1 [128,256), O [256,384), P [384,448), Q [448,512).
// d = 64: two CTAs an SM, whose softmaxes and products overlap; one S buffer, Q
// in shared memory.  TMEM columns S [0,128), O [128,192), P [192,256).
// Rounding: P to bf16 for its product (the sum l is of the unrounded values),
// O once at the end.
// Every wait is bounded; on expiry the kernel records UT_ERR_TIMEOUT, drains
// its own copies and MMAs, frees TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "wattn.cuh"
#include "xattn_tc.cuh"

namespace ut {

namespace {

constexpr int kM = 128, kN = 128, kThreads = 256;
constexpr uint32_t kChunkBytes = 128 * 128;  // 128 rows x 64 bf16
constexpr int kItemSlots = 3;                // no more are taken ahead: other CTAs may be idle

template <int D>
struct Form {
  static constexpr int kCtas = D == 128 ? 1 : 2;    // an SM
  static constexpr bool kQt = D == 128;             // Q in TMEM
  static constexpr int kS = D == 128 ? 2 : 1;       // S buffers
  static constexpr int kQ = D == 128 ? 1 : 2, kK = D == 128 ? 3 : 2, kV = kK;  // tiles in shared memory
  static constexpr uint32_t kCols = D == 128 ? 512 : 256;
  static constexpr uint32_t kO = D == 128 ? 256 : 128, kP = D == 128 ? 384 : 192, kQc = 448;
  // registers of the two-CTA form: per thread, launch and setmaxnreg split
  static constexpr int kRegLaunch = 128, kRegCtl = 64, kRegSoftmax = 192;
};
static_assert(Form<64>::kRegCtl + Form<64>::kRegSoftmax <= 2 * Form<64>::kRegLaunch, "the split must fit the launch");

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
  alignas(16) float bias[F::kV][kN];  // of the keys of a V tile: 0 < bias = attend
  uint64_t q_full[F::kQ], q_empty[F::kQ], k_full[F::kK], k_empty[F::kK], v_full[F::kV], v_empty[F::kV], v_ready[F::kV];
  uint64_t qt_full, qt_empty, s_full[F::kS], s_empty[F::kS], p_full, pv_done, o_empty, mma_done;
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  Item item[kItemSlots];
  NextItem next;
  uint32_t tmem_base;
  int abort_flag;
};

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
__global__ void __launch_bounds__(kThreads, Form<D>::kCtas)
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
      mbar_init(&sm.q_empty[s], F::kQt ? 4 : 1);  // the softmax warps have copied it / S is done
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
      mbar_init(&sm.s_empty[s], 4);
    }
    mbar_init(&sm.p_full, 4);
    mbar_init(&sm.pv_done, 1);
    mbar_init(&sm.o_empty, 4);
    mbar_init(&sm.mma_done, 1);
    for (int s = 0; s < kItemSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], 7);  // warps 0, 1, 3 and the softmax warps
    }
    next_item_init(sm.next);
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, F::kCols);
    tmem_relinquish();
  }
  if (blockIdx.x == 0) {
    check_cu(p.cu_q, p.B, p.nq, p.status);
    check_cu(p.cu_k, p.B, p.nk, p.status);
    check_lens_of(prm.w);
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
  // Block t of an item holds the keys x .. x + 127 of the segment, those below e.
  auto block_of = [&](const Item& it, int t, int& x, int& e) { win_block<kN>(it.rg, it.j0 + t, x, e); };
  auto all_keys = [&](int x, int e) { return !p.mask && e - x >= kN; };

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
        for (int t = 0; t < it.blocks; ++t) {
          int x, e;
          block_of(it, t, x, e);
          const uint32_t st = at % F::kK, ph = ((at / F::kK) & 1) ^ 1;
          if (!(ok = wait(&sm.k_empty[st], ph))) break;
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
        auto keys_of = [&](int t) -> uint32_t {
          int x, e;
          block_of(it, t, x, e);
          return all_keys(x, e) ? 15u : lane_keys(p.mask, (int64_t)it.key0 + x, e - x, lane);
        };
        uint32_t next = keys_of(0);
        for (int t = 0; t < it.blocks; ++t, ++at) {
          const uint32_t st = at % F::kV, keys = next;
          int x, e;
          block_of(it, t, x, e);
          if (t + 1 < it.blocks) next = keys_of(t + 1);  // a block ahead
          if (!(ok = wait(&sm.v_full[st], (at / F::kV) & 1))) break;
          if (!all_keys(x, e)) {
#pragma unroll
            for (int g = 0; g < 4; ++g) sm.bias[st][g * 32 + lane] = (keys >> g) & 1u ? INFINITY : -INFINITY;
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
      // on values made uniform.  Step i issues S of block i and P V of block i -
      // kS; at an item's first block P V comes first, as Q arrives in TMEM late.
      constexpr uint32_t idesc_s = idesc_bf16_f32(kM, kN, false, false);
      constexpr uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      constexpr uint32_t kStep = S::kTile >> 4, kFirst = 2;
      const uint32_t q_lo = desc_lo(smem_u32(sm.q[0]), 16), k_lo = desc_lo(smem_u32(sm.k[0]), 16),
                     v_lo = desc_lo(smem_u32(sm.v[0]), kChunkBytes);
      auto waitq = [&](uint64_t* bar, uint32_t parity) -> bool {
        return quick_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
      };
      uint32_t n = 0, left = 0, nq = 0;      // items taken, blocks left of S's, Q tiles
      uint32_t ks = 0, kf = 0, vs = 0, vf = 0, sb = 0, sf = 1, pf = 0, of = 1;  // stages and phases
      uint32_t f0 = 0, f1 = 0;               // flags of the blocks of P V; 0: none
      bool ok = true, end = false;
      auto pv = [&](uint32_t f) -> bool {
        if (!waitq(&sm.v_ready[vs], vf)) return false;
        if (f & kFirst) {
          if (!waitq(&sm.o_empty, of)) return false;
          of ^= 1;
        }
        if (!waitq(&sm.p_full, pf)) return false;
        tc_fence_after();
        mma_tn<128>(tmem + F::kO, tmem + F::kP, v_lo + vs * kStep, idesc_o, (f & kFirst) ^ kFirst);
        mma_commit_w(&sm.pv_done);
        mma_commit_w(&sm.v_empty[vs]);
        pf ^= 1;
        if (++vs == F::kV) {
          vs = 0;
          vf ^= 1;
        }
        return true;
      };
#pragma unroll 1
      do {
        uint32_t fn = 0;
        if (left == 0 && !end) {
          const uint32_t s = n % kItemSlots;
          if (!(ok = waitq(&sm.item_full[s], (n / kItemSlots) & 1))) break;
          end = (int)warp_uniform((uint32_t)sm.item[s].hk) < 0;
          left = end ? 0u : warp_uniform((uint32_t)sm.item[s].blocks);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.item_empty[s]);
          ++n;
          if (!end) fn = kFirst;
        }
        const bool early = F::kQt && (fn & kFirst);  // P V first
        if (early && f0 && !(ok = pv(f0))) break;
        if (left > 0) {
          fn |= 1u;
          --left;
          if (fn & kFirst) {
            if (!(ok = F::kQt ? waitq(&sm.qt_full, nq & 1) : waitq(&sm.q_full[nq % F::kQ], (nq / F::kQ) & 1))) break;
            ++nq;
          }
          if (!(ok = waitq(&sm.k_full[ks], kf))) break;
          if (!(ok = waitq(&sm.s_empty[sb], sf))) break;
          tc_fence_after();
          if constexpr (F::kQt)
            mma_tk128(tmem + sb * kN, tmem + F::kQc, k_lo + ks * kStep, idesc_s);
          else
            mma_nt<D>(tmem + sb * kN, q_lo + ((nq - 1) % F::kQ) * kStep, k_lo + ks * kStep, idesc_s);
          mma_commit_w(&sm.s_full[sb]);
          mma_commit_w(&sm.k_empty[ks]);
          if (left == 0) mma_commit_w(F::kQt ? &sm.qt_empty : &sm.q_empty[(nq - 1) % F::kQ]);
          if (++ks == F::kK) {
            ks = 0;
            kf ^= 1;
          }
          if (++sb == F::kS) {
            sb = 0;
            sf ^= 1;
          }
        }
        const uint32_t f = F::kS == 2 ? f0 : f1;
        if (!early && f && !(ok = pv(f))) break;
        f0 = f1;
        f1 = fn;
      } while (f0 | f1);
      mma_commit_w(&sm.mma_done);  // every MMA has completed before TMEM is freed
      drain(&sm.mma_done, 0);
    }
  } else {
    // ------------------------------------------------------------------- softmax
    if constexpr (F::kCtas == 2) setmaxnreg_inc<F::kRegSoftmax>();
    const uint32_t quarter = warp & 3, lane_base = tmem + ((quarter * 32) << 16), row = quarter * 32 + lane;
    auto token_of = [&](uint32_t r) -> int { return (int)((r * prm.inv_g) >> 16); };  // r / G
    const int rt = token_of(row), rt_first = token_of(quarter * 32), rt_last = token_of(quarter * 32 + 31);
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    uint32_t n = 0, nq = 0, b = 0, vst = 0, vf = 0;  // items, Q tiles copied, blocks; V stage and phase
    bool ok = true, pend = false;
    Item it{}, nx{};
    float m = -1e30f, l = 0.f;
    // what the pending item's rows need
    int e_hk = 0, e_tok0 = 0, e_ntok = 0, e_split = 0;
    float e_m = 0.f, e_l = 0.f;

    // O / l in bf16 and LSE, or the partial result
    auto write_rows = [&](int hk, int tok0, int ntok, int split, float em, float el) {
      const int h = hk * p.G + (int)(row - rt * p.G);
      const bool row_ok = rt < ntok;
      if (p.nsplit > 1) {
        const int64_t prow = ((int64_t)split * p.nq + tok0 + rt) * p.H + h;
#pragma unroll 1
        for (int g = 0; g < D / 32; ++g) {
          uint32_t r[32];
          tmem_ld32(lane_base + F::kO + g * 32, r);
          tmem_wait_ld();
          if (!row_ok) continue;
#pragma unroll
          for (int x = 0; x < 32; x += 4)
            *reinterpret_cast<uint4*>(p.part_o + prow * D + g * 32 + x) = make_uint4(r[x], r[x + 1], r[x + 2], r[x + 3]);
        }
        if (row_ok) p.part_ml[prow] = make_float2(em, el);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.o_empty);
        return;
      }
      if (row_ok) p.lse[(int64_t)h * p.nq + tok0 + rt] = el == 0.f ? -INFINITY : (em + log2f(el)) * kLn2;
      // A thread holds a row; the four lanes of a quad exchange 16-byte units so
      // that lane c holds unit c of each of the quad's rows, and a store covers 64
      // contiguous bytes of eight rows instead of 16 of 32.
      const float f = el > 0.f ? 1.f / el : (el == 0.f ? 0.f : el);
      const uint32_t c = lane & 3;
      __nv_bfloat16* out[4];
      __nv_bfloat16* const base = static_cast<__nv_bfloat16*>(p.o) + (int64_t)tok0 * p.os + (int64_t)hk * p.G * D + c * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = quarter * 32 + (lane & ~3u) + i;
        const int yt = token_of(y);
        out[i] = yt < ntok ? base + (int64_t)yt * p.os + (y - yt * p.G) * D : nullptr;
      }
#pragma unroll 1
      for (int g = 0; g < D / 32; ++g) {
        uint32_t r[32], u[4][4];
        tmem_ld32(lane_base + F::kO + g * 32, r);
        tmem_wait_ld();
        if (g == D / 32 - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.o_empty);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x)
          u[x >> 2][x & 3] = pack_bf16x2(__uint_as_float(r[2 * x]) * f, __uint_as_float(r[2 * x + 1]) * f);
        exchange_units<1>(u, c & 1, 0, 1);
        exchange_units<1>(u, c & 1, 2, 3);
        exchange_units<2>(u, c >> 1, 0, 2);
        exchange_units<2>(u, c >> 1, 1, 3);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (out[i]) *reinterpret_cast<uint4*>(out[i] + g * 32) = make_uint4(u[i][0], u[i][1], u[i][2], u[i][3]);
      }
    };
    // nx's Q tile: shared memory (128B-swizzled, as TMA wrote it) -> TMEM, this
    // thread's row, bf16 pairs: the A operand of S = Q K^T
    auto load_q = [&]() -> bool {
      if (!wait(&sm.q_full[0], nq & 1)) return false;
      if (!wait(&sm.qt_empty, (nq & 1) ^ 1)) return false;
      tc_fence_after();
#pragma unroll
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
      ++nq;
      return true;
    };

    bool more = next_item(n, nx, ok), first = true;
    if (F::kQt && more) ok = load_q();
    int t = 0, pos = 0;
    // A block a round; the last round only writes the last item's rows.
#pragma unroll 1
    while (ok && (more || pend)) {
      bool last = false;
      if (more) {
        if (first) {
          it = nx;
          pos = it.p0 + rt;  // of this row's token
          t = 0;
        }
        int x, e;
        block_of(it, t, x, e);
        const uint32_t sb = b % F::kS, ts = lane_base + sb * kN;
        const bool whole = all_keys(x, e);
        last = t == it.blocks - 1;
        if (!(ok = wait(&sm.s_full[sb], (b / F::kS) & 1))) break;
        if (!whole && !(ok = wait(&sm.v_ready[vst], vf))) break;
        tc_fence_after();
        // The rows' own limits, where some row of the warp has one in this block:
        // S there becomes -inf in TMEM, 32 columns at a time.  (In the code below,
        // unrolled over 128 columns, they cost every block 1,500 cycles: the code
        // no longer fits the instruction cache.)
        const bool lim_r = it.p0 + rt_first + prm.w.right - x < kN - 1,
                   lim_l = it.p0 + rt_last - prm.w.left > x && x + kN > prm.w.sinks;
        if (lim_r || lim_l) {
          const int hi = pos + prm.w.right - x, lo = pos - prm.w.left - x, sink = prm.w.sinks - x;
#pragma unroll 1
          for (int g = 0; g < kN; g += 32) {
            const bool cut = (g + 31 > it.p0 + rt_first + prm.w.right - x) ||
                             (g < it.p0 + rt_last - prm.w.left - x && g + 31 >= sink);
            if (!cut) continue;
            uint32_t r[32];
            tmem_ld32(ts + g, r);
            tmem_wait_ld();
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (y > hi - g || (y < lo - g && y >= sink - g)) r[y] = 0xff800000u;
            tmem_st32(ts + g, r);
          }
          tmem_wait_st();
        }
        uint32_t r[kN];
#pragma unroll
        for (int g = 0; g < 4; ++g) tmem_ld32(ts + g * 32, *reinterpret_cast<uint32_t(*)[32]>(&r[g * 32]));
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.s_empty[sb]);
        if (last) {  // the next item's Q: its first S is computed while this block is in the softmax
          more = next_item(n, nx, ok);
          if (F::kQt && more) ok = load_q();
          if (!ok) break;
        }
        if (!whole) {
          asm volatile("" ::: "memory");  // a branch, not a choice between 128 values
#pragma unroll
          for (int y = 0; y < kN; y += 4) {
            const float4 v = *reinterpret_cast<const float4*>(sm.bias[vst] + y);
            r[y] = __float_as_uint(fminf(__uint_as_float(r[y]), v.x));
            r[y + 1] = __float_as_uint(fminf(__uint_as_float(r[y + 1]), v.y));
            r[y + 2] = __float_as_uint(fminf(__uint_as_float(r[y + 2]), v.z));
            r[y + 3] = __float_as_uint(fminf(__uint_as_float(r[y + 3]), v.w));
          }
        }
        if (++vst == F::kV) {
          vst = 0;
          vf ^= 1;
        }
        float m8[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) m8[y] = fmaxf(__uint_as_float(r[y]), __uint_as_float(r[y + 8]));
#pragma unroll
        for (int y = 16; y < kN; y += 16)
#pragma unroll
          for (int z = 0; z < 8; ++z) m8[z] = max3(m8[z], __uint_as_float(r[y + z]), __uint_as_float(r[y + z + 8]));
        float mx = max3(max3(m8[0], m8[1], m8[2]), max3(m8[3], m8[4], m8[5]), fmaxf(m8[6], m8[7]));
        mx = fmaxf(mx * prm.scale_log2, -1e30f);  // finite where a row sees no key of the block
        const bool need = !first && mx > m + 8.0f;
        const bool any = __any_sync(0xffffffffu, need);
        float alpha = 1.f;
        if (first) {
          m = mx;
          l = 0.f;
        } else if (need) {
          alpha = ex2_approx(m - mx);
          m = mx;
          l *= alpha;
        }
        const uint64_t m2 = pack_f32x2(-m, -m);
        uint64_t sum[4] = {0, 0, 0, 0};
        uint32_t pk[kN / 2];
#pragma unroll
        for (int y = 0; y < kN; y += 2) {
          float p0, p1;
          unpack_f32x2(fma_f32x2(pack_u32x2(r[y], r[y + 1]), c2, m2), p0, p1);
          p0 = ex2_approx(p0);
          p1 = ex2_approx(p1);
          sum[(y >> 1) & 3] = add_f32x2(sum[(y >> 1) & 3], pack_f32x2(p0, p1));
          pk[y / 2] = pack_bf16x2(p0, p1);
        }
        float a0, a1;
        unpack_f32x2(add_f32x2(add_f32x2(sum[0], sum[1]), add_f32x2(sum[2], sum[3])), a0, a1);
        l += a0 + a1;
        // P's columns are free, and O holds P V up to the block before, once its
        // product is done
        if (!(ok = wait(&sm.pv_done, (b & 1) ^ 1))) break;
        tc_fence_after();
        if (any) {
#pragma unroll 1
          for (int g = 0; g < D / 16; ++g) {
            uint32_t o[16];
            tmem_ld16(lane_base + F::kO + g * 16, o);
            tmem_wait_ld();
#pragma unroll
            for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * alpha);
            tmem_st16(lane_base + F::kO + g * 16, o);
          }
        }
        tmem_st32(lane_base + F::kP, *reinterpret_cast<uint32_t(*)[32]>(&pk[0]));
        tmem_st32(lane_base + F::kP + 32, *reinterpret_cast<uint32_t(*)[32]>(&pk[32]));
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full);
        ++b;
        ++t;
      } else {
        if (!(ok = wait(&sm.pv_done, (b & 1) ^ 1))) break;
        tc_fence_after();
      }
      if (first && pend) write_rows(e_hk, e_tok0, e_ntok, e_split, e_m, e_l);
      if (first) pend = false;
      first = last;
      if (last) {
        pend = true;
        e_hk = it.hk;
        e_tok0 = it.tok0;
        e_ntok = it.ntok;
        e_split = it.split;
        e_m = m;
        e_l = l;
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
  wattn_fwd_tc_kernel<D><<<(unsigned)prm.n_items, kThreads, smem, s>>>(tm[0], tm[1], tm[2], prm);
  return cudaGetLastError();
}

}  // namespace

int64_t wattn_fwd_tc_items(const WinParams& w) { return segment_slots(w.x.nq, w.x.B, kM / w.x.G) * w.x.Hk; }

// Parts of the keys of a tile: the fewest whole waves of items that fill the SMs
// (to a tenth of the best of four), none shorter than two blocks of a mean
// segment's keys, as far as a tile sees them.
int wattn_fwd_tc_splits(const WinParams& w) {
  const XattnParams& p = w.x;
  const int64_t items = wattn_fwd_tc_items(w), ctas = (int64_t)p.sms * (p.d == 64 ? Form<64>::kCtas : Form<128>::kCtas);
  double best = 0;
  int64_t want = 1;
  for (int v = 1; v <= 4; ++v) {
    const int64_t n = v * ctas / items;
    const double use = (double)(n * items) / ((double)v * ctas);
    if (n >= 1 && use > best + 0.1) {
      best = use;
      want = n;
    }
  }
  const int64_t near = (int64_t)w.left + w.right + w.sinks + kM / p.G, rows = p.nk / p.B;
  const int64_t most = ((near < rows ? near : rows) + kN - 1) / kN / 2;
  const int64_t n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
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
