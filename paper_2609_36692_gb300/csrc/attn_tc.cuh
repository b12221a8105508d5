// What the tensor-core attention kernels share: tile addressing, the walk over
// the work list, and the host side's tensor maps.
#pragma once

#include <cudaTypedefs.h>

#include <string>

#include "attn.h"
#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace normpre {

constexpr int kTile = 128;                 // rows and keys of a tile
constexpr int kChunk = kTile * 128;        // bytes of 128 rows of 64 bf16: one TMA box, 128-byte swizzle
constexpr float kLog2e = 1.4426950408889634f;

// The r-th item of this CTA, -1 past its last.  With a plan's lists: ids from
// walk[gridDim.x + 1 + walk[c]] up to walk[gridDim.x + 1 + walk[c + 1]].  Without
// (many items per CTA): the items in falling order of cost, back and forth over
// the CTAs.
__device__ __forceinline__ int64_t walk_item(const int* walk, int64_t r, int64_t items) {
  const int64_t g = gridDim.x, c = blockIdx.x;
  if (walk) {
    const int64_t i = walk[c] + r;
    return i < walk[c + 1] ? walk[g + 1 + i] : -1;
  }
  const int64_t i = r * g + ((r & 1) ? g - 1 - c : c);
  return i < items ? i : -1;
}

// One tile of `chunks` 64-wide column chunks: 128 rows from `row` of a head.
// Rows past the tensor and columns past head_dim arrive as zeros.
__device__ __forceinline__ void load_rows(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int64_t row, int head,
                                          int chunks) {
  for (int c = 0; c < chunks; ++c)
    tc::tma_load_3d(dst + c * kChunk, map, bar, 64 * c, static_cast<int>(row), head);
}

// Descriptor of a tile read along its columns (K = head dimension: K-major) or
// along its rows (K = tokens: MN-major); step kk of 16 adds to the address.
__device__ __forceinline__ uint64_t desc_cols(uint32_t tile) { return tc::sdesc(tile, 16, 1024); }
__device__ __forceinline__ uint64_t desc_rows(uint32_t tile) { return tc::sdesc(tile, kChunk, 1024); }
__host__ __device__ constexpr uint64_t cols_step(int kk) { return ((kk >> 2) * kChunk + (kk & 3) * 32) >> 4; }
__host__ __device__ constexpr uint64_t rows_step(int kk) { return (kk * 2048) >> 4; }

// D = A B^T over columns 16 K0 .. 16 K1 of the head dimension: both tiles in
// shared memory.
template <int DP, int K0 = 0, int K1 = DP / 16>
__device__ __forceinline__ void product_ss(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t idesc = tc::idesc_bf16(kTile, kTile, 0, 0);
  const uint64_t ad = desc_cols(a), bd = desc_cols(b);
#pragma unroll
  for (int kk = K0; kk < K1; ++kk) tc::mma_bf16(d, ad + cols_step(kk), bd + cols_step(kk), idesc, kk != 0);
}
// D (+)= A B over rows 16 K0 .. 16 K1 of B: A in TMEM, its columns 64 .. 127
// `gap` columns further on.
template <int DP, int K0 = 0, int K1 = 8>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, bool first, int gap) {
  constexpr uint32_t idesc = tc::idesc_bf16(kTile, DP, 0, 1);
  const uint64_t bd = desc_rows(b);
#pragma unroll
  for (int kk = K0; kk < K1; ++kk)
    tc::mma_bf16_ta(d, a + kk * 8 + (kk >= 4 ? gap : 0), bd + rows_step(kk), idesc, !first || kk != K0);
}

// Zeroes rows [rows, 128) of a tile in shared memory (one warp): what follows
// a sequence in the pack, which may hold anything, must not meet a zero
// probability in a product.
__device__ __forceinline__ void zero_tail(uint8_t* tile, int rows, int chunks, int lane) {
  for (int c = 0; c < chunks; ++c)
    for (int b = rows * 128 + lane * 16; b < kChunk; b += 32 * 16)
      *reinterpret_cast<uint4*>(tile + c * kChunk + b) = make_uint4(0, 0, 0, 0);
  tc::fence_smem_async();
  __syncwarp();
}

// Zeroes rows [total, tokens) of a tensor: warp w of n.
__device__ __forceinline__ void zero_padding(const AttnArgs& a, const AttnTensor& t, int heads, int64_t w, int64_t n,
                                             int lane) {
  const int64_t rows = static_cast<int64_t>(a.tokens - a.total) * heads;
  for (int64_t i = w; i < rows; i += n) {
    const int64_t r = a.total + i / heads;
    bf16* p = static_cast<bf16*>(t.p) + r * t.ts + (i % heads) * t.hs;
    for (int c = lane * 8; c < a.dim; c += 256) *reinterpret_cast<uint4*>(p + c) = make_uint4(0, 0, 0, 0);
  }
}

// 32 fp32 columns of a thread's row, scaled, as bf16 at p (columns c .. of `dim`).
__device__ __forceinline__ void store_row32(bf16* p, const uint32_t* r, float w, int c, int dim) {
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = pack_bf16x2(__uint_as_float(r[i + 2 * e]) * w, __uint_as_float(r[i + 2 * e + 1]) * w);
    if (c + i < dim) *reinterpret_cast<uint4*>(p + c + i) = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

// Map of a [tokens][heads][dim] bf16 tensor for boxes of 128 rows x 64 columns.
inline bool rows_map(CUtensorMap* m, const AttnTensor& t, int tokens, int heads, int dim, std::string* err) {
  const uint64_t dims[3] = {static_cast<uint64_t>(dim), static_cast<uint64_t>(tokens), static_cast<uint64_t>(heads)};
  const uint64_t strides[2] = {static_cast<uint64_t>(t.ts) * 2, static_cast<uint64_t>(t.hs) * 2};
  const uint32_t box[3] = {64, kTile, 1};
  return driver_encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, t.p, dims, strides, box, err);
}

}  // namespace normpre
