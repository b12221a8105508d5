// Weight gradient of a linear layer from its input's 8-bit checkpoint:
// dW = dY^T xhat, summed over the tokens.
//
// k_wgrad_simt: fp32 arithmetic, one CTA of 256 threads per 64 x 64 piece of
// dW, 16 tokens at a time through shared memory, a 4 x 4 piece per thread; any
// dtype, stride and size.  Bound by the fp32 FMA pipe.
#include "ckpt.h"
#include "common.cuh"
#include "internal.h"

namespace normpre {
namespace {

template <typename TY, typename TW>
__global__ void __launch_bounds__(256) k_wgrad_simt(const __grid_constant__ WgradArgs a) {
  __shared__ float Y[16][64], X[16][64];
  const int n0 = blockIdx.y * 64, k0 = blockIdx.x * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const TY* dy = static_cast<const TY*>(a.dy);
  float acc[4][4] = {};
  for (int64_t t0 = 0; t0 < a.tokens; t0 += 16) {
    for (int e = threadIdx.x; e < 16 * 64; e += 256) {
      const int64_t t = t0 + (e >> 6);
      const int c = e & 63, n = n0 + c, k = k0 + c;
      Y[e >> 6][c] = t < a.tokens && n < a.n ? to_f32(dy[t * a.dy_ld + n]) : 0.f;
      float x = 0.f;
      if (t < a.tokens && k < a.k)
        x = static_cast<float>(a.x.codes[t * a.x_ld + k]) *
            ckpt_step(a.x.steps[(k / kCkptPanel) * a.tokens + t], (k % kCkptPanel) / kCkptBlock);
      X[e >> 6][c] = x;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const float4 y = *reinterpret_cast<const float4*>(&Y[t][4 * ty]);
      const float4 x = *reinterpret_cast<const float4*>(&X[t][4 * tx]);
      const float yv[4] = {y.x, y.y, y.z, y.w}, xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][c] = fmaf(yv[r], xv[c], acc[r][c]);
    }
    __syncthreads();
  }
  TW* dw = static_cast<TW*>(a.dw);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = n0 + 4 * ty + r, k = k0 + 4 * tx + c;
      if (n < a.n && k < a.k) {
        TW* p = dw + n * a.dw_ld + k;
        *p = from_f32<TW>(a.accumulate ? to_f32(*p) + acc[r][c] : acc[r][c]);
      }
    }
}

}  // namespace

cudaError_t launch_ckpt_wgrad_simt(const WgradArgs& a, int dy_dtype, int dw_dtype, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(cdiv(a.k, 64)), static_cast<unsigned>(cdiv(a.n, 64)));
  if (dy_dtype == 0) {
    if (dw_dtype == 0) k_wgrad_simt<float, float><<<grid, 256, 0, s>>>(a);
    else k_wgrad_simt<float, bf16><<<grid, 256, 0, s>>>(a);
  } else {
    if (dw_dtype == 0) k_wgrad_simt<bf16, float><<<grid, 256, 0, s>>>(a);
    else k_wgrad_simt<bf16, bf16><<<grid, 256, 0, s>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace normpre
