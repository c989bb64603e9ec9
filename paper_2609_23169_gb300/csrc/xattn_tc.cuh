// Device helpers of the cross-attention tensor-core kernels.
#pragma once
#include "common.cuh"
#include "pairs.cuh"
#include "xattn.cuh"

namespace ut {

UT_DEV void tma_load_3d(void* dst, const void* tmap, uint64_t* bar, int32_t x, int32_t y, int32_t z, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(smem_u32(dst)),
      "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

// A whole product of tcgen05.mma instructions, executed by a converged warp
// and issued by one elected lane, with the shared-memory descriptors split
// into a constant high word and a low word that only needs additions.  The
// operands have to be the same in every lane, and are kept in uniform
// registers where the warp's control flow is provably uniform (votes,
// warp_uniform below): a product then costs its issue and little else.  With
// operands in ordinary registers (one thread in a divergent branch) an
// instruction took 80-130 cycles to issue, more than it takes to run.
//   kDescHi: 128-byte swizzle, 1024 bytes between groups of eight 128-byte
//   rows; desc_lo: start address and leading byte offset, in units of 16 bytes
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
UT_DEV uint32_t desc_lo(uint32_t addr, uint32_t lbo_bytes) { return ((addr & 0x3FFFFu) >> 4) | ((lbo_bytes >> 4) << 16); }
UT_DEV uint32_t warp_uniform(uint32_t x) { return __reduce_or_sync(0xffffffffu, x); }

#define UT_SS_STEP(off, acc)                                             \
  "add.u32 x, %1, " off ";\n\tadd.u32 y, %2, " off ";\n\t"              \
  "mov.b64 a, {x, %4};\n\tmov.b64 b, {y, %4};\n\t"                     \
  "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, " acc ";\n\t"
#define UT_SS_HEAD                                                                     \
  "{\n\t.reg .pred e, f, t;\n\t.reg .b64 a, b;\n\t.reg .b32 x, y;\n\t"              \
  "setp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
// d = A B^T over D columns of two K-major tiles (128-row sub-tiles of 64 columns)
template <int D>
UT_DEV void mma_nt(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  if constexpr (D == 64)
    asm volatile(UT_SS_HEAD UT_SS_STEP("0", "f") UT_SS_STEP("2", "t") UT_SS_STEP("4", "t") UT_SS_STEP("6", "t") "}" ::"r"(d),
                 "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(kDescHi)
                 : "memory");
  else
    asm volatile(UT_SS_HEAD UT_SS_STEP("0", "f") UT_SS_STEP("2", "t") UT_SS_STEP("4", "t") UT_SS_STEP("6", "t")
                     UT_SS_STEP("1024", "t") UT_SS_STEP("1026", "t") UT_SS_STEP("1028", "t") UT_SS_STEP("1030", "t") "}" ::"r"(d),
                 "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(kDescHi)
                 : "memory");
}
#define UT_TS_STEP(acol, boff, acc)                                     \
  "add.u32 x, %1, " acol ";\n\tadd.u32 y, %2, " boff ";\n\t"           \
  "mov.b64 b, {y, %5};\n\t"                                            \
  "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, " acc ";\n\t"
// d (+)= A B over N rows of B: A in TMEM (bf16 pairs, 8 columns a step), B
// row-major (MN-major operand, 16 rows of 128 bytes a step)
#define UT_TS_HEAD                                                  \
  "{\n\t.reg .pred e, p, t;\n\t.reg .b64 b;\n\t.reg .b32 x, y;\n\t" \
  "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
template <int N>
UT_DEV void mma_tn(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  if constexpr (N == 96)
    asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "128", "t") UT_TS_STEP("16", "256", "t")
                     UT_TS_STEP("24", "384", "t") UT_TS_STEP("32", "512", "t") UT_TS_STEP("40", "640", "t") "}" ::"r"(d),
                 "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
  else if constexpr (N == 64)
    asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "128", "t") UT_TS_STEP("16", "256", "t")
                     UT_TS_STEP("24", "384", "t") "}" ::"r"(d),
                 "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
  else if constexpr (N == 128)
    asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "128", "t") UT_TS_STEP("16", "256", "t")
                     UT_TS_STEP("24", "384", "t") UT_TS_STEP("32", "512", "t") UT_TS_STEP("40", "640", "t")
                         UT_TS_STEP("48", "768", "t") UT_TS_STEP("56", "896", "t") "}" ::"r"(d),
                 "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
  else
    asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "128", "t") "}" ::"r"(d), "r"(a), "r"(b_lo),
                 "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
}

// d = A B^T over 128 columns: A in TMEM (bf16 pairs), B a K-major tile
UT_DEV void mma_tk128(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc) {
  const uint32_t accumulate = 0;
  asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "2", "t") UT_TS_STEP("16", "4", "t")
                   UT_TS_STEP("24", "6", "t") UT_TS_STEP("32", "1024", "t") UT_TS_STEP("40", "1026", "t")
                       UT_TS_STEP("48", "1028", "t") UT_TS_STEP("56", "1030", "t") "}" ::"r"(d),
               "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
               : "memory");
}

// d (+)= A B over 128 rows of B, A in TMEM as two halves of 64 columns, each in
// the first 32 of the 64 columns that it replaced
UT_DEV void mma_tnh(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(UT_TS_HEAD UT_TS_STEP("0", "0", "p") UT_TS_STEP("8", "128", "t") UT_TS_STEP("16", "256", "t")
                   UT_TS_STEP("24", "384", "t") UT_TS_STEP("64", "512", "t") UT_TS_STEP("72", "640", "t")
                       UT_TS_STEP("80", "768", "t") UT_TS_STEP("88", "896", "t") "}" ::"r"(d),
               "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
               : "memory");
}

// warp_wait for warps whose code has to stay short: one try, and the loop that
// spins (bounded as always) out of line.
static __device__ __noinline__ bool spin_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                       uint64_t timeout_ns) {
  return warp_wait(bar, parity, abort_flag, status, timeout_ns);
}
UT_DEV bool quick_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status, uint64_t timeout_ns) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  if (__builtin_expect(__all_sync(0xffffffffu, r), 1)) return true;
  return warp_uniform(spin_wait(bar, parity, abort_flag, status, timeout_ns));
}

// ------------------------------------------------------------- next item
// The grid has a block for each item; the blocks that run take the items of
// those that have not started, one after another, until none is left (a block
// is asked for an item ahead).  So segments of unequal lengths fill the SMs
// evenly: with a fixed share of the items each, the longest of 152 shares was
// 1.42 times the mean for 13 ragged images.
struct NextItem {
  alignas(16) uint8_t answer[2][16];
  uint64_t full[2];
};
UT_DEV void next_item_init(NextItem& x) {
  mbar_init(&x.full[0], 1);
  mbar_init(&x.full[1], 1);
}
UT_DEV void next_item_ask(NextItem& x, uint32_t i) {  // request i, by one thread
  mbar_expect_tx(&x.full[i & 1], 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                   smem_u32(x.answer[i & 1])),
               "r"(smem_u32(&x.full[i & 1]))
               : "memory");
}
// the answer to request i (its barrier waited for): an item, or -1
UT_DEV int next_item_answer(NextItem& x, uint32_t i) {
  int item;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t.reg .b32 c, y, z, w;\n\t"
      "ld.shared.b128 h, [%1];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "mov.b32 %0, -1;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {c, y, z, w}, h;\n\t"
      "@p mov.b32 %0, c;\n\t}"
      : "=r"(item)
      : "r"(smem_u32(x.answer[i & 1]))
      : "memory");
  return item;
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

UT_DEV float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// the smaller of two, NaN where either is
UT_DEV float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Lanes whose number differs in bit kBit exchange unit b of the lower one (bit =
// 0) for unit a of the upper one (bit = 1).
template <int kBit>
UT_DEV void exchange_units(uint32_t (&u)[4][4], uint32_t bit, int a, int b) {
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const uint32_t got = __shfl_xor_sync(0xffffffffu, bit ? u[a][x] : u[b][x], kBit);
    u[a][x] = bit ? got : u[a][x];
    u[b][x] = bit ? u[b][x] : got;
  }
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

// one column
UT_DEV uint32_t tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr));
  return r;
}
UT_DEV void tmem_st1(uint32_t taddr, uint32_t r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(r) : "memory");
}

}  // namespace ut
