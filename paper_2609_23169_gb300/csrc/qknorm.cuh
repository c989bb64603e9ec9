// Parameters of the query / key norm kernels (qknorm.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace ut {

struct QkNormParams {
  const void* q; const void* k; const void* v;
  const float* wq; const float* wk;              // [d] or NULL (ones)
  const int32_t* pos;                            // [n] or NULL (0, 1, ...)
  const int32_t* rows;                           // [n] rows of ko, vo, or NULL (0, 1, ...)
  void* qo; void* ko; void* vo;                  // forward: outputs; backward: dq, dk
  const void* dqo; const void* dko;
  float* dwq; float* dwk;                        // [d] or NULL
  float* part;                                   // [blocks, 2, d]: partial dwq, dwk
  int32_t* status;
  int64_t n, cache_rows;
  int H, Hk, d;
  int64_t qs, ks, vs, qos, kos, vos, dqos, dkos; // elements between rows
  float eps;
  // RoPE: a pair's angle in turns per unit of its coordinate, as a fraction of
  // 2^64, and its coordinate (0 image, 1 y, 2 x)
  uint64_t turn[64];
  uint8_t axis[64];
  uint32_t side, area;                           // tokens of an image's side, of an image (at most 2^31)
  int32_t prefix;
  int sms;
};

// Blocks an SM (4 and 3, with fewer registers each: 2048 canvas 387 us instead of
// 335, training step of a 1024 canvas 282 instead of 250); the backward's leave
// partial sums.
constexpr int kQnFwdBlocksPerSm = 3, kQnBlocksPerSm = 2;
inline int64_t qknorm_bwd_blocks(int64_t n, int sms) {
  const int64_t want = (n + 7) / 8, most = (int64_t)sms * kQnBlocksPerSm;
  return want < most ? want : most;
}
cudaError_t launch_qknorm_fwd(const QkNormParams& p, bool bf16, cudaStream_t s);
cudaError_t launch_qknorm_bwd(const QkNormParams& p, bool bf16, cudaStream_t s);

}  // namespace ut
