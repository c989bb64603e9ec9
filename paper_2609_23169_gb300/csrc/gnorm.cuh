// Parameters of the group-norm kernels and their launchers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace ut {

struct GnormParams {
  const void* x; void* y; const void* dy; void* dx;
  const float* gamma; const float* beta;   // [C], or null: 1 and 0
  float* mean; float* rstd;                // [B, G]
  float* dgamma; float* dbeta;             // [C], or null
  const int32_t* cu;
  int32_t* status;
  int64_t n;                               // rows
  int64_t xs, ys, dys, dxs;                // elements between rows
  int B, C, G, act;
  float eps;
  int group_lanes;                         // threads that sum a group
  int slots, slot_bytes, ring_at;          // the ring in shared memory
  uint64_t timeout_ns;
  void* ws;
  int sms;
};

constexpr int kGnMaxChannels = 8192, kGnMaxBoth = 12288;  // channels; channels + groups (shared memory)

size_t gnorm_ws(const GnormParams& p, bool backward);
cudaError_t launch_gnorm_fwd(const GnormParams& p, bool bf16, cudaStream_t s);
cudaError_t launch_gnorm_bwd(const GnormParams& p, bool bf16, cudaStream_t s);

}  // namespace ut
