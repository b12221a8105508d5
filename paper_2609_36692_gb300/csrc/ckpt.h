// 8-bit activation checkpoints: storage arithmetic shared by the kernels that
// write and read them (ckpt.cu, ckpt_wgrad.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

namespace normpre {

constexpr int kCkptBlock = 32;    // elements that share a step
constexpr int kCkptPanel = 128;   // features whose four steps form one 32-bit word per row

inline int64_t ckpt_ld(int64_t features) { return (features + kCkptBlock - 1) / kCkptBlock * kCkptBlock; }
inline int64_t ckpt_panels(int64_t features) { return (features + kCkptPanel - 1) / kCkptPanel; }

struct CkptView {
  const int8_t* codes;     // [tokens][ld]
  const uint32_t* steps;   // [panels][tokens]
};

// The step of byte b of a panel word: the byte is the biased exponent of an
// fp32 power of two.  255 gives infinity, and the codes of such a block are
// zero, so that code * step is NaN without a test.
__device__ __forceinline__ float ckpt_step(uint32_t word, int b) {
  return __uint_as_float(((word >> (8 * b)) & 0xFFu) << 23);
}

struct WgradArgs {
  const void* dy;
  int64_t dy_ld;
  CkptView x;
  int64_t x_ld;
  void* dw;
  int64_t dw_ld;
  int64_t tokens;
  int n, k;                // dW is n x k
  int accumulate;
  int* flags;
};
// bf16 dY whose base and rows are on 16-byte boundaries; at least one token.
cudaError_t launch_ckpt_wgrad_tc(const WgradArgs& a, int dw_dtype, cudaStream_t s, std::string* err);
cudaError_t launch_ckpt_wgrad_simt(const WgradArgs& a, int dy_dtype, int dw_dtype, cudaStream_t s);

}  // namespace normpre
