// Parameters of the cross-attention kernels and the launchers of their forms.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ultratex.h"

namespace ut {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

struct XattnParams {
  const void* q; const void* k; const void* v;
  void* o; float* lse;                   // outputs of the forward, inputs of the backward
  const void* dout; void* dq; void* dk; void* dv;
  const int32_t* cu_q; const int32_t* cu_k; const uint8_t* mask;
  int32_t* status;
  int64_t nq, nk;
  int B, H, Hk, G, d;                    // segments, query heads, kv heads, H / Hk, head dimension
  int64_t qs, ks, vs, os, dos, dqs, dks, dvs;  // elements between rows
  float scale;
  uint64_t timeout_ns;
  int sms;
  // Work split over the long axis: keys in the forward (part_o [nsplit, nq,
  // H, d] unnormalised, part_ml [nsplit, nq, H] the running maximum in the
  // base-2 domain and the sum), query rows in the fp32 backward (part_dk,
  // part_dv [nsplit, nk, Hk, d]).
  int nsplit;
  float* part_o; float2* part_ml;
  float* dsum;                           // [H, nq] D = dO . O
  float* part_dk; float* part_dv;
};

// Checks of a shape and of the pointers (api_cond.cu); the rest of p is filled
// in between.
ut_status xattn_shape(const ut_xattn_shape* s, bool backward, XattnParams* p);
ut_status xattn_pointers(const ut_xattn_shape* s, const XattnParams& p);

// Work items of a pass without splits, and how many parts its long axis is
// split into.
int64_t xattn_items(const XattnParams& p, bool bf16, bool backward);
int xattn_splits(const XattnParams& p, bool bf16, bool backward);
int64_t xattn_fwd_tc_items(const XattnParams& p);
cudaError_t launch_xattn_fwd_simt(const XattnParams& p, cudaStream_t s);  // fp32
cudaError_t launch_xattn_fwd_tc(const XattnParams& p, cudaStream_t s);    // bf16
cudaError_t launch_xattn_join(const XattnParams& p, bool bf16, cudaStream_t s);  // of the forward's key splits
cudaError_t launch_xattn_dkdv_join(const XattnParams& p, cudaStream_t s);  // of the fp32 backward's splits
int64_t xattn_bwd_tc_items(const XattnParams& p);
size_t xattn_bwd_tc_ws(const XattnParams& p);
cudaError_t launch_xattn_dsum(const XattnParams& p, bool bf16, cudaStream_t s);  // D, and the check of the prefixes
cudaError_t launch_xattn_bwd_simt(const XattnParams& p, cudaStream_t s);         // fp32
cudaError_t launch_xattn_bwd_tc(const XattnParams& p, void* ws, cudaStream_t s); // bf16

// The kernels of a backward pass follow one another without a gap: each says
// at once that the next may be launched, and the next does what needs no
// result (barriers, TMEM, its own decoding) and then waits for the whole grid
// before it.
__device__ __forceinline__ void grid_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename F, typename... A>
cudaError_t launch_next(F kern, dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace ut
