// Packed causal attention: what the host side (attn.cu) and the kernels share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

#include "internal.h"

namespace normpre {

// 128 rows of one sequence: rows start + 128 blk .. of the pack, of which the
// sequence holds min(128, len - 128 blk).
struct AttnBlock {
  int start;   // the sequence's first row
  int len;     // the sequence's rows
  int blk;     // index of the block in the sequence
  int pad;
};

// Whether an entry of the lists fits into `total` rows.  The lists are rebuilt for
// other lengths in place, and a call that was captured before then walks them
// with counts of its own: every entry is checked before anything is addressed
// by it, so that such a call ends with a flag and not out of range.
__host__ __device__ inline bool block_fits(const AttnBlock& b, int total) {
  return b.start >= 0 && b.start <= total && b.len > 0 && b.len <= total - b.start && b.blk >= 0 &&
         b.blk <= (b.len - 1) / 128;
}

// A [tokens][heads][head_dim] tensor, strides in elements.
struct AttnTensor {
  void* p;
  int64_t ts, hs;
};

struct AttnArgs {
  AttnTensor q, k, v, o, dout, dq, dk, dv;
  float* lse;                // [heads][tokens]
  float* delta;              // [heads][tokens] <do_i, o_i>
  const AttnBlock* by_query; // blocks, the ones that see the most keys first
  const AttnBlock* by_key;   // blocks, the ones seen by the most queries first
  const AttnBlock* by_pair;  // the blocks of even index, in by_query's order
  int n_blocks, n_pairs;
  // items of each CTA of the tensor-core kernels (null: see walk_item)
  const int *walk_fwd, *walk_dkdv, *walk_dq;
  int total;                 // rows that belong to sequences
  int tokens;
  int heads, kv_heads, group, dim;
  float scale;               // c
  float scale_log2;          // c log2(e): exp(c x) = exp2(scale_log2 x)
  int* flags;                // pinned host memory
  int test_stall;
};

// The forward kernel's two query tiles are two heads of a group; otherwise two
// neighbouring tiles of one head.
inline bool attn_pair_heads(int group) { return group % 2 == 0; }

// CTAs of a tensor-core kernel.
inline int walk_grid(int64_t items) {
  return static_cast<int>(items < 1 ? 1 : items < device_sm_count() ? items : device_sm_count());
}

// fp32 kernels, one CTA per 64 rows and head (attn_simt.cu).
cudaError_t launch_attn_forward_simt(const AttnArgs& a, cudaStream_t s);
cudaError_t launch_attn_backward_simt(const AttnArgs& a, cudaStream_t s);
// Tensor-core kernels, bf16 (attn_fwd.cu, attn_bwd.cu).
cudaError_t launch_attn_forward_tc(const AttnArgs& a, cudaStream_t s, std::string* err);
cudaError_t launch_attn_backward_tc(const AttnArgs& a, cudaStream_t s, std::string* err);
// delta_i = <do_i, o_i>; zero for rows outside the sequences.
cudaError_t launch_attn_delta(const AttnArgs& a, int dtype, cudaStream_t s);

}  // namespace normpre
