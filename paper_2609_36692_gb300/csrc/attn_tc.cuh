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
// the CTAs.  What does not fit the call (see block_fits) is flagged and ends the
// CTA's walk.
__device__ __forceinline__ int64_t walk_item(const int* walk, int64_t r, int64_t items, int* flags) {
  const int64_t g = gridDim.x, c = blockIdx.x;
  if (walk) {
    const int64_t i = walk[c] + r, end = walk[c + 1];
    if (i >= 0 && end <= items) {
      if (i >= end) return -1;
      const int64_t id = walk[g + 1 + i];
      if (id >= 0 && id < items) return id;
    }
    raise_host_flag(flags, kFlagLists);
    return -1;
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
// D (+)= A B over rows 16 K0 .. 16 K1 of B: A in TMEM as bf16, two a column;
// `spread` (1, 2, 4): its columns lie in that many parts, each at the start of
// its share of 128 columns.
template <int DP, int spread, int K0 = 0, int K1 = 8>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, bool first) {
  constexpr uint32_t idesc = tc::idesc_bf16(kTile, DP, 0, 1);
  const uint64_t bd = desc_rows(b);
#pragma unroll
  for (int kk = K0; kk < K1; ++kk)
    tc::mma_bf16_ta(d, a + 8 * kk + (kk * spread / 8) * (spread == 1 ? 0 : 64 / spread), bd + rows_step(kk), idesc,
                    !first || kk != K0);
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

// A warp's 32 rows x N (16 or 32) fp32 columns, one row a thread, scaled, to
// global memory as bf16: columns c .. of rows row0 .. of a tile whose first
// `rows` exist.  The lanes of 2 or 4 rows exchange their 16-byte pieces first,
// so that a row's piece of 2 N bytes leaves in one instruction: scattered
// 16-byte stores took several microseconds a tile.
template <int N>
__device__ __forceinline__ void store_rows(bf16* tile, int64_t ts, const uint32_t* r, float w, int row0, int rows, int c,
                                           int dim, int lane) {
  constexpr int kPieces = N / 8;
  static_assert(kPieces == 2 || kPieces == 4, "pieces");
  uint32_t v[kPieces][4];
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[i][e] = pack_bf16x2(__uint_as_float(r[8 * i + 2 * e]) * w, __uint_as_float(r[8 * i + 2 * e + 1]) * w);
  // piece i of row (lane & ~(kPieces - 1)) + k comes to lane i of the group, as its v[k]
#pragma unroll
  for (int o = 1; o < kPieces; o <<= 1)
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (!(i & o)) {
        const bool up = lane & o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t give = up ? v[i][e] : v[i | o][e];
          const uint32_t got = __shfl_xor_sync(0xffffffffu, give, o);
          if (up) v[i][e] = got; else v[i | o][e] = got;
        }
      }
  const int piece = lane & (kPieces - 1), first = row0 + (lane & ~(kPieces - 1));
  bf16* p = tile + first * ts + c + 8 * piece;
#pragma unroll
  for (int k = 0; k < kPieces; ++k)
    if (first + k < rows && c + 8 * piece < dim)
      *reinterpret_cast<uint4*>(p + k * ts) = make_uint4(v[k][0], v[k][1], v[k][2], v[k][3]);
}

// The first items of a CTA, resolved once into shared memory: looking one up
// is two dependent global loads, a microsecond between two items otherwise.
struct ItemRef {
  int start, len, blk, head;   // blk -1: no item
};

// The r-th item of this CTA from a list of blocks with `per` items each.
__device__ __forceinline__ ItemRef list_item(const AttnArgs& a, const AttnBlock* list, int blocks, const int* walk, int per,
                                             int64_t r) {
  const ItemRef none = {0, 0, -1, 0};
  const int64_t i = walk_item(walk, r, static_cast<int64_t>(blocks) * per, a.flags);
  if (i < 0) return none;
  const AttnBlock b = list[i / per];
  if (!block_fits(b, a.total)) {
    raise_host_flag(a.flags, kFlagLists);
    return none;
  }
  return ItemRef{b.start, b.len, b.blk, static_cast<int>(i % per)};
}

// Map of a [tokens][heads][dim] bf16 tensor for boxes of 128 rows x 64 columns.
inline bool rows_map(CUtensorMap* m, const AttnTensor& t, int tokens, int heads, int dim, std::string* err) {
  const uint64_t dims[3] = {static_cast<uint64_t>(dim), static_cast<uint64_t>(tokens), static_cast<uint64_t>(heads)};
  const uint64_t strides[2] = {static_cast<uint64_t>(t.ts) * 2, static_cast<uint64_t>(t.hs) * 2};
  const uint32_t box[3] = {64, kTile, 1};
  return driver_encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, t.p, dims, strides, box, err);
}

}  // namespace normpre
