// Cross attention to an encoder's states, forward, on the 5th-generation
// tensor cores (bf16 in, fp32 accumulate):
//   O_i = softmax_j(scale q_i . k_j) v_j,   LSE_i = ln sum_j exp(scale q_i . k_j)
// over the keys j of query i's segment whose mask is set.
//
// A query tile holds 128 rows: the G heads that share a kv head of 128 / G
// consecutive tokens of one segment (row = token * G + head; one TMA box), so
// that K and V are read once for the group.  A work item is two such tiles,
// one kv head and one range of key blocks (128 keys each); its tiles take
// turns on the tensor cores, so that one tile's products run while the other
// tile's softmax does, and share every K and V tile in shared memory.
//
// Persistent CTAs, one per SM; items with the head fastest, so that CTAs in
// flight read neighbouring 256-byte pieces of the same rows and share K and V
// in L2.  Roles (384 threads, registers rebalanced with setmaxnreg):
//   warp 0      TMA: the K and V tiles, one ring (K0 V0 K1 V1 ...)
//   warp 1      TMEM owner and MMA issuer.  Over the blocks of all items in
//               one stream, for each tile w: O_w += P_w V of the previous
//               block, then S_w = Q_w K^T of this one (P_w overwrote S_w in
//               TMEM, so this order needs no second buffer).
//   warp 2      TMA: the query tiles, a ring of their own
//   warp 3      decodes the items (segment search, key range) into a ring
//   warps 4-7   softmax of tile 0, warps 8-11 of tile 1: thread = row = TMEM
//               lane.  Read S from TMEM, mask, keep a running maximum (O is
//               rescaled in TMEM only where it grew by more than 2^8, so the
//               exponentials stay bounded), write P as bf16 over S; after the
//               last block O / l and LSE, or the split's partial result.
// Masked keys and the rows of other segments: S there is replaced by -inf,
// and the MMA warp zeroes those rows of the V tile before its products, so
// that no value they hold (NaN, infinities) is multiplied.
// TMEM columns: S_0 / P_0 [0,128), S_1 / P_1 [128,256), O_0 [256,256+d), O_1
// [384,384+d).
// Every wait is bounded; on expiry the kernel records UT_ERR_TIMEOUT, drains
// its own copies and MMAs, frees TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "segments.cuh"
#include "xattn.cuh"

namespace ut {

namespace {

constexpr int kM = 128;  // rows of a query tile
constexpr int kN = 128;  // keys of a block
constexpr int kThreads = 384;
constexpr int kRegLaunch = 168, kRegCtl = 120, kRegSoftmax = 192;  // per thread; setmaxnreg split
static_assert(kRegCtl + 2 * kRegSoftmax <= 3 * kRegLaunch, "the split must fit the launch's registers");
constexpr uint32_t kChunkBytes = 128 * 128;  // 128 rows x 64 bf16
constexpr int kItemSlots = 4, kItemReaders = 11;

struct Item {
  int32_t hk;      // kv head; -1: no more items
  int32_t blocks;  // key blocks of this item (0: write the empty result)
  int32_t tok0;    // first token of tile 0
  int32_t ntok[2]; // tokens of the tiles (tile 1 may be empty)
  int32_t key0;    // first key
  int32_t left;    // keys from key0 to the end of the segment
  int32_t split;
};

template <int D>
struct Smem {
  static constexpr int kChunks = D / 64;
  static constexpr uint32_t kTile = 128 * D * 2;
  static constexpr int kQ = D == 128 ? 3 : 4;   // query tiles in flight
  static constexpr int kKv = D == 128 ? 4 : 8;  // K and V tiles in flight
  alignas(1024) uint8_t q[kQ][kTile];
  alignas(1024) uint8_t kv[kKv][kTile];
  uint64_t q_full[kQ], q_empty[kQ], kv_full[kKv], kv_empty[kKv];
  uint64_t s_full[2], p_full[2], o_full[2], o_empty[2], mma_done;
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  Item item[kItemSlots];
  uint32_t tmem_base;
  int abort_flag;
};

struct Params {
  XattnParams x;
  int tpt;           // tokens of a tile
  int slots;         // item slots along the query rows (two tiles each)
  int64_t n_items;   // slots * Hk * nsplit
  float scale_log2;
  bool keep_kv;      // K and V are read by several items: keep them in L2
};

UT_DEV void tma_load_3d(void* dst, const void* tmap, uint64_t* bar, int32_t x, int32_t y, int32_t z, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(smem_u32(dst)),
      "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

// This lane's four keys of a block (lane + 32 g): bit g set where the key
// exists and is not masked.
UT_DEV uint32_t lane_keys(const uint8_t* mask, int64_t key, int left, uint32_t lane) {
  uint32_t b = 0;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int x = (int)lane + 32 * g;
    if (x < left && (!mask || mask[key + x])) b |= 1u << g;
  }
  return b;
}

// Pairs of fp32 values in one 64-bit register: one instruction for two.
UT_DEV uint64_t pack_u32x2(uint32_t a, uint32_t b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
  return r;
}
UT_DEV uint64_t pack_f32x2(float a, float b) { return pack_u32x2(__float_as_uint(a), __float_as_uint(b)); }
UT_DEV void unpack_f32x2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
UT_DEV uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
UT_DEV uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 32 lanes x 32 bit, 16 consecutive columns per thread
UT_DEV void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
UT_DEV void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    xattn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const Params prm) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
  using S = Smem<D>;
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
      mbar_init(&sm.kv_empty[s], 1);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(&sm.s_full[w], 1);
      mbar_init(&sm.p_full[w], 4);
      mbar_init(&sm.o_full[w], 1);
      mbar_init(&sm.o_empty[w], 4);
    }
    mbar_init(&sm.mma_done, 1);
    for (int s = 0; s < kItemSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], kItemReaders);
    }
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
  const uint32_t tmem = sm.tmem_base;

  auto wait = [&](uint64_t* bar, uint32_t parity) {  // whole warp, converged
    return warp_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto wait1 = [&](uint64_t* bar, uint32_t parity) {  // one thread
    return mbar_wait(bar, parity, abort_flag, p.status, p.timeout_ns);
  };
  auto drain = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_drain(bar, parity, kDrainTimeoutNs)) set_status(p.status, UT_ERR_TIMEOUT);
  };
  // The next item; false at the end or on an abort (then ok = false).  Whole
  // warp, or a single thread with one = true.
  auto next_item = [&](uint32_t& n, Item& it, bool& ok, bool one) -> bool {
    const uint32_t s = n % kItemSlots, f = (n / kItemSlots) & 1;
    ok = one ? wait1(&sm.item_full[s], f) : wait(&sm.item_full[s], f);
    if (!ok) return false;
    it = sm.item[s];
    if (!one) __syncwarp();
    if (one || lane == 0) mbar_arrive(&sm.item_empty[s]);
    ++n;
    return it.hk >= 0;
  };

  if (warp < 4) {
    setmaxnreg_dec<kRegCtl>();
    if (warp == 0 && lane == 0) {
      // ------------------------------------------------------- K, V producer
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
      const uint64_t pol = prm.keep_kv ? policy_evict_last() : policy_evict_first();
      uint32_t n = 0, at = 0;
      bool ok = true;
      Item it;
      while (ok && next_item(n, it, ok, true)) {
        for (int j = 0; j < it.blocks && ok; ++j) {
#pragma unroll 1
          for (int which = 0; which < 2; ++which) {
            const uint32_t st = at % S::kKv, f = at / S::kKv;
            if (!(ok = wait1(&sm.kv_empty[st], (f & 1) ^ 1))) break;
            mbar_expect_tx(&sm.kv_full[st], S::kTile);
            const void* tm = which ? static_cast<const void*>(&tm_v) : static_cast<const void*>(&tm_k);
            for (int c = 0; c < S::kChunks; ++c)
              tma_load_3d(sm.kv[st] + c * kChunkBytes, tm, &sm.kv_full[st], c * 64, it.hk, it.key0 + j * kN, pol);
            ++at;
          }
        }
      }
      for (uint32_t x = at > S::kKv ? at - S::kKv : 0; x < at; ++x) drain(&sm.kv_full[x % S::kKv], (x / S::kKv) & 1);
    } else if (warp == 2 && lane == 0) {
      // ---------------------------------------------------------- Q producer
      tma_prefetch_desc(&tm_q);
      const uint64_t pol = policy_evict_first();
      const uint32_t bytes = (uint32_t)prm.tpt * p.G * 128 * S::kChunks;
      uint32_t n = 0, at = 0;
      bool ok = true;
      Item it;
      while (ok && next_item(n, it, ok, true)) {
        if (it.blocks == 0) continue;
        for (int w = 0; w < 2 && ok; ++w) {
          if (it.ntok[w] == 0) continue;
          const uint32_t st = at % S::kQ, f = at / S::kQ;
          if (!(ok = wait1(&sm.q_empty[st], (f & 1) ^ 1))) break;
          mbar_expect_tx(&sm.q_full[st], bytes);
          for (int c = 0; c < S::kChunks; ++c)
            tma_load_3d(sm.q[st] + c * kChunkBytes, &tm_q, &sm.q_full[st], c * 64, it.hk * p.G, it.tok0 + w * prm.tpt,
                        pol);
          ++at;
        }
      }
      for (uint32_t x = at > S::kQ ? at - S::kQ : 0; x < at; ++x) drain(&sm.q_full[x % S::kQ], (x / S::kQ) & 1);
    } else if (warp == 3 && lane == 0) {
      // -------------------------------------------------------- item decoder
      uint32_t n = 0;
      bool ok = true;
      for (int64_t w = blockIdx.x; ok; w += gridDim.x) {
        Item it{};
        it.hk = -1;
        if (w < prm.n_items) {
          const int64_t u = w / p.Hk;
          const Segment g = segment_of_slot(p.cu_q, p.B, p.nq, 2 * prm.tpt, u % prm.slots);
          const int64_t t0 = g.tile * 2 * prm.tpt;
          if (t0 >= g.n) continue;  // an idle slot
          int64_t k0, kn;
          segment_rows(p.cu_k, g.s, p.nk, k0, kn);
          const int64_t nblk = (kn + kN - 1) / kN, per = (nblk + p.nsplit - 1) / p.nsplit;
          it.split = (int)(u / prm.slots);
          const int64_t b0 = min(nblk, per * it.split), b1 = min(nblk, b0 + per);
          it.hk = (int)(w % p.Hk);
          it.blocks = (int)(b1 - b0);
          it.tok0 = (int)(g.row + t0);
          it.ntok[0] = (int)min((int64_t)prm.tpt, g.n - t0);
          it.ntok[1] = (int)max((int64_t)0, min((int64_t)prm.tpt, g.n - t0 - prm.tpt));
          it.key0 = (int)(k0 + b0 * kN);
          it.left = (int)(kn - b0 * kN);
        }
        const uint32_t s = n % kItemSlots, f = n / kItemSlots;
        if (!(ok = wait1(&sm.item_empty[s], (f & 1) ^ 1))) break;
        sm.item[s] = it;
        mbar_arrive(&sm.item_full[s]);
        ++n;
        if (it.hk < 0) break;
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------- MMA issuer
      constexpr uint32_t idesc_s = idesc_bf16_f32(kM, kN, false, false);
      constexpr uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      uint32_t n = 0, qat = 0, kvat = 0;
      uint32_t nps[2] = {0, 0}, noe[2] = {0, 0};  // P tiles consumed, O accumulators begun
      bool ok = true;
      // the previous block: its V stage, which tiles it has, and its place in its item
      bool have = false, first = false, last = false, on[2] = {false, false};
      uint32_t v_st = 0;
      auto pv = [&](int w) -> bool {  // O_w (+)= P_w V of the previous block
        if (!wait(&sm.p_full[w], nps[w] & 1)) return false;
        ++nps[w];
        if (first) {
          if (!wait(&sm.o_empty[w], (noe[w] & 1) ^ 1)) return false;
          ++noe[w];
        }
        tc_fence_after();
        const uint32_t va = smem_u32(sm.kv[v_st]);
#pragma unroll
        for (int kk = 0; kk < kN / 16; ++kk)
          mma_bf16_ts_w(tmem + 256 + w * 128, tmem + w * 128 + kk * 8, sdesc_sw128(va + kk * 2048, kChunkBytes, 1024),
                        idesc_o, !first || kk > 0);
        if (last) mma_commit_w(&sm.o_full[w]);
        return true;
      };
      Item it;
      while (ok && next_item(n, it, ok, false)) {
        if (it.blocks == 0) continue;
        const bool tile[2] = {true, it.ntok[1] > 0};
        for (int j = 0; j < it.blocks && ok; ++j) {
          const uint32_t k_st = kvat % S::kKv, kf = kvat / S::kKv;
          const uint32_t vn = kvat + 1, vs = vn % S::kKv, vf = vn / S::kKv;
          kvat += 2;
          const int left = it.left - j * kN;
          const bool full = !p.mask && left >= kN;
          uint32_t keys = 15u;
          if (!full) keys = lane_keys(p.mask, (int64_t)it.key0 + j * kN, left, lane);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (!ok) break;
            if (have && on[w] && !(ok = pv(w))) break;
            if (have && w == 1) mma_commit_w(&sm.kv_empty[v_st]);
            if (!tile[w]) continue;
            if (w == 0 && !(ok = wait(&sm.kv_full[k_st], kf & 1))) break;
            const uint32_t q_st = (qat + w) % S::kQ, qf = (qat + w) / S::kQ;
            if (j == 0 && !(ok = wait(&sm.q_full[q_st], qf & 1))) break;
            tc_fence_after();
            const uint32_t qa = smem_u32(sm.q[q_st]), ka = smem_u32(sm.kv[k_st]);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = (kk >> 2) * kChunkBytes + (kk & 3) * 32;
              mma_bf16_ss_w(tmem + w * 128, sdesc_sw128(qa + off, 16, 1024), sdesc_sw128(ka + off, 16, 1024), idesc_s,
                            kk > 0);
            }
            mma_commit_w(&sm.s_full[w]);
            if (j == it.blocks - 1) mma_commit_w(&sm.q_empty[q_st]);
          }
          if (!ok) break;
          mma_commit_w(&sm.kv_empty[k_st]);
          // V of this block, needed by the next step's products: zero the rows
          // that must not enter them while the softmax works
          if (!(ok = wait(&sm.kv_full[vs], vf & 1))) break;
          if (__any_sync(0xffffffffu, keys != 15u)) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
              if (!((keys >> g) & 1u)) {
                const uint32_t row = smem_u32(sm.kv[vs]) + (lane + 32 * g) * 128;
#pragma unroll
                for (int c = 0; c < S::kChunks; ++c)
#pragma unroll
                  for (int x = 0; x < 8; ++x)
                    st_shared_v4(row + c * kChunkBytes + (((x + lane) & 7) << 4), 0, 0, 0, 0);
              }
            fence_proxy_async_smem();
            __syncwarp();
          }
          v_st = vs;
          have = true;
          first = j == 0;
          last = j == it.blocks - 1;
          on[0] = true;
          on[1] = tile[1];
        }
        qat += tile[1] ? 2 : 1;
      }
      if (ok && have) {
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (ok && on[w]) ok = pv(w);
      }
      mma_commit_w(&sm.mma_done);  // every MMA has completed before TMEM is freed
      drain(&sm.mma_done, 0);
    }
  } else {
    // ----------------------------------------------------------------- softmax
    setmaxnreg_inc<kRegSoftmax>();
    const int w = warp < 8 ? 0 : 1;
    const uint32_t quarter = warp & 3, lane_base = (quarter * 32) << 16;
    const uint32_t ts = tmem + lane_base + w * 128, to = tmem + lane_base + 256 + w * 128;
    const uint64_t c2 = pack_f32x2(prm.scale_log2, prm.scale_log2);
    uint32_t n = 0, ns = 0, no = 0;
    bool ok = true;
    for (;; ++n) {
      // the item stays in its slot until this tile is done with it
      const uint32_t slot = n % kItemSlots;
      if (!(ok = wait(&sm.item_full[slot], (n / kItemSlots) & 1))) break;
      const volatile Item* it = &sm.item[slot];
      if (it->hk < 0) break;
      const int blocks = it->ntok[w] > 0 ? it->blocks : 0;
      float m = -1e30f, l = 0.f;
      uint32_t keys = blocks > 0 ? lane_keys(p.mask, it->key0, it->left, lane) : 0;
      for (int j = 0; j < blocks; ++j) {
        const uint32_t now = keys;
        if (j + 1 < blocks)  // the next block's, fetched a block ahead
          keys = lane_keys(p.mask, (int64_t)it->key0 + (j + 1) * kN, it->left - (j + 1) * kN, lane);
        if (!(ok = wait(&sm.s_full[w], ns & 1))) break;
        ++ns;
        tc_fence_after();
        uint32_t r[kN];
#pragma unroll
        for (int g = 0; g < 4; ++g) tmem_ld32(ts + g * 32, *reinterpret_cast<uint32_t(*)[32]>(&r[g * 32]));
        tmem_wait_ld();
        if (!__all_sync(0xffffffffu, now == 15u)) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint32_t word = __ballot_sync(0xffffffffu, (now >> g) & 1u);
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (!((word >> x) & 1u)) r[g * 32 + x] = 0xff800000u;  // -inf
          }
        }
        float m8[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) m8[x] = __uint_as_float(r[x]);
#pragma unroll
        for (int x = 8; x < kN; x += 16) {
#pragma unroll
          for (int y = 0; y < 8; ++y)
            m8[y] = x + 8 + y < kN ? fmaxf(fmaxf(m8[y], __uint_as_float(r[x + y])), __uint_as_float(r[x + 8 + y < kN ? x + 8 + y : 0]))
                                   : fmaxf(m8[y], __uint_as_float(r[x + y]));
        }
        float mx = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])),
                         fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7])));
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
        for (int g = 0; g < 4; ++g) {
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
      // O / l and LSE, or the split's partial result
      if (blocks > 0) {
        if (!(ok = wait(&sm.o_full[w], no & 1))) break;
        ++no;
        tc_fence_after();
      }
      const int row = (int)(quarter * 32 + lane), rt = row / p.G;  // this row's token of the tile
      const int h = it->hk * p.G + row % p.G, ntok = it->ntok[w], split = it->split;
      const int64_t tok = (int64_t)it->tok0 + w * prm.tpt + rt;
      const bool row_ok = rt < ntok;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
      const bool part = p.nsplit > 1;
      const float f = part ? 1.f : (l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l));
      const int64_t prow = ((int64_t)split * p.nq + tok) * p.H + h;
      __nv_bfloat16* orow = static_cast<__nv_bfloat16*>(p.o) + tok * p.os + (int64_t)h * D;
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
        if (part) {
#pragma unroll
          for (int x = 0; x < 32; x += 4)
            *reinterpret_cast<uint4*>(p.part_o + prow * D + g * 32 + x) =
                make_uint4(r[x], r[x + 1], r[x + 2], r[x + 3]);
        } else {
#pragma unroll
          for (int x = 0; x < 32; x += 8) {
            uint4 v;
            v.x = pack_bf16x2(__uint_as_float(r[x + 0]) * f, __uint_as_float(r[x + 1]) * f);
            v.y = pack_bf16x2(__uint_as_float(r[x + 2]) * f, __uint_as_float(r[x + 3]) * f);
            v.z = pack_bf16x2(__uint_as_float(r[x + 4]) * f, __uint_as_float(r[x + 5]) * f);
            v.w = pack_bf16x2(__uint_as_float(r[x + 6]) * f, __uint_as_float(r[x + 7]) * f);
            *reinterpret_cast<uint4*>(orow + g * 32 + x) = v;
          }
        }
      }
      if (blocks > 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.o_empty[w]);
      }
      if (row_ok) {
        if (part) p.part_ml[prow] = make_float2(m, l);
        else p.lse[(int64_t)h * p.nq + tok] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

static_assert(sizeof(Smem<128>) <= 232448 && sizeof(Smem<64>) <= 232448, "shared layout exceeds the block limit");

template <int D>
cudaError_t launch_d(const Params& prm, const CUtensorMap* tm, cudaStream_t s) {
  const size_t smem = sizeof(Smem<D>);
  cudaError_t e = cudaFuncSetAttribute(xattn_fwd_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // the setmaxnreg split assumes exactly kRegLaunch registers per thread at
  // launch: with fewer, the increases would wait for registers that never come
  cudaFuncAttributes fa;
  e = cudaFuncGetAttributes(&fa, xattn_fwd_tc_kernel<D>);
  if (e != cudaSuccess) return e;
  if (fa.numRegs != kRegLaunch) return cudaErrorInvalidConfiguration;
  const int grid = (int)(prm.n_items < prm.x.sms ? prm.n_items : prm.x.sms);
  xattn_fwd_tc_kernel<D><<<grid, kThreads, smem, s>>>(tm[0], tm[1], tm[2], prm);
  return cudaGetLastError();
}

}  // namespace

int64_t xattn_fwd_tc_items(const XattnParams& p) { return segment_slots(p.nq, p.B, 2 * (kM / p.G)) * p.Hk; }

cudaError_t launch_xattn_fwd_tc(const XattnParams& p, cudaStream_t s) {
  Params prm{};
  prm.x = p;
  prm.tpt = kM / p.G;
  prm.slots = (int)segment_slots(p.nq, p.B, 2 * prm.tpt);
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
