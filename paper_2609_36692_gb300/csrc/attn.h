// Packed causal attention: what the host side (attn.cu) and the kernels share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

#include "heads.h"
#include "internal.h"

namespace normpre {

// 128 rows of one sequence: rows start + 128 blk .. of the pack, of which the
// sequence holds min(128, len - 128 blk).
struct AttnBlock {
  int start;   // the sequence's first row
  int len;     // the sequence's rows
  int blk;     // index of the block in the sequence
  int part;    // of a key block whose queries are split: its place (see KeyPart); by_split: the first place
};

// Whether an entry of the lists fits into `total` rows.  The lists are rebuilt for
// other lengths in place, and a call that was captured before then walks them
// with counts of its own: every entry is checked before anything is addressed
// by it, so that such a call ends with a flag and not out of range.
__host__ __device__ inline bool block_fits(const AttnBlock& b, int total) {
  return b.start >= 0 && b.start <= total && b.len > 0 && b.len <= total - b.start && b.blk >= 0 &&
         b.blk <= (b.len - 1) / 128;
}

// Which blocks of 128 keys a block of 128 queries meets, and the other way
// round.  Row i sees keys j <= i with i - j < window or j < sinks: a query block
// meets the sinks' blocks [0, sink) and then [lo, blk] (sink <= lo), a key block
// the query blocks blk .. last.  Without a window (kNoWindow): all up to blk.
constexpr int kNoWindow = 1 << 25;   // beyond every distance of two rows
struct KeySpan {
  int lo, sink;
  __host__ __device__ int count(int blk) const { return blk - lo + 1 + sink; }
  // the block before j, on the way down; -1: none
  __host__ __device__ int down(int j) const { return j > lo || j <= sink ? j - 1 : sink - 1; }
  // the block after j, on the way up
  __host__ __device__ int up(int j) const { return j + 1 == sink ? lo : j + 1; }
  __host__ __device__ int first() const { return sink ? 0 : lo; }
  // the block of which only the first 32 keys or fewer are seen, as sinks; -1: none
  __host__ __device__ int narrow(int sinks) const { return sink && sinks - 128 * (sink - 1) <= 32 ? sink - 1 : -1; }
};
__host__ __device__ inline KeySpan key_span(int blk, int window, int sinks) {
  KeySpan s;
  const int below = 128 * blk - window + 1, ends = (sinks + 127) / 128;
  s.lo = below > 0 ? below / 128 : 0;
  s.sink = ends < s.lo ? ends : s.lo;
  return s;
}
__host__ __device__ inline int last_query(int blk, int len, int window, int sinks) {
  const int last = (len - 1) / 128, in = (128 * blk + 126 + window) / 128;
  return 128 * blk < sinks || last < in ? last : in;
}

// Whether every row sees itself alone: then p = 1 whatever the scores, and ds = 0
// is written as such, where the difference of two equal sums would leave noise.
__host__ __device__ inline bool sees_itself(int window, int sinks) { return window == 1 && sinks == 0; }

// The sinks' key blocks meet all later query blocks, however short the window.
// They are split into parts of about `chunk` query blocks, each an item of its
// own, whose sums over queries (dk, dv in fp32) lie in a slot of the workspace
// until they are added up in the parts' order.  part = index of the part * 2^12 +
// slot + 1; 0: not split.
constexpr int kMaxSlots = 4000;
__host__ __device__ inline int key_parts(int count, int chunk) { return (count + chunk - 1) / chunk; }
struct KeyPart {
  int first, end;    // query blocks
  int slot;          // -1: not split
  bool fits;         // whether the entry is one of this call's (see block_fits)
};
__host__ __device__ inline KeyPart key_part(const AttnBlock& b, int window, int sinks, int chunk, int slots) {
  KeyPart p;
  const int count = last_query(b.blk, b.len, window, sinks) - b.blk + 1;
  p.first = b.blk;
  p.end = b.blk + count;
  p.slot = (b.part & 4095) - 1;
  p.fits = true;
  if (b.part) {
    const int n = chunk > 0 ? key_parts(count, chunk) : 0, i = b.part >> 12;
    p.fits = i >= 0 && i < n && n < 4096 && p.slot >= 0 && p.slot < slots;
    if (p.fits) {
      p.first = b.blk + static_cast<int>(static_cast<int64_t>(count) * i / n);
      p.end = b.blk + static_cast<int>(static_cast<int64_t>(count) * (i + 1) / n);
    }
  }
  return p;
}

typedef HeadsView AttnTensor;

struct AttnArgs {
  AttnTensor q, k, v, o, dout, dq, dk, dv;
  float* lse;                // [heads][tokens]
  float* delta;              // [heads][tokens] <do_i, o_i>
  const AttnBlock* by_query; // blocks, the ones that see the most keys first
  const AttnBlock* by_key;   // blocks, the ones seen by the most queries first
  const AttnBlock* by_pair;  // the blocks of even index, in by_query's order
  const AttnBlock* by_split; // key blocks whose queries are split
  int n_blocks, n_pairs;
  int n_keys, n_split;       // entries of by_key (a split block has several), of by_split
  int chunk, slots;          // see KeyPart
  float* partial;            // [slots][kv_heads][dk, dv][128][dim]
  // items of each CTA of the tensor-core kernels (null: see walk_item)
  const int *walk_fwd, *walk_dkdv, *walk_dq;
  int total;                 // rows that belong to sequences
  int tokens;
  int heads, kv_heads, group, dim;
  int window, sinks;         // kNoWindow, 0: none, or none that the lengths reach
  float scale;               // c
  float scale_log2;          // c log2(e): exp(c x) = exp2(scale_log2 x)
  int* flags;                // pinned host memory
  int test_stall;
};

// The forward kernel's two query tiles are two heads of a group; otherwise two
// neighbouring tiles of one head.
inline bool attn_pair_heads(int group) { return group % 2 == 0; }

// Kinds of tensor-core kernels: no window; one; one whose narrow sink block (see
// KeySpan::narrow) has a path of its own.  That path pays where it is a good part of
// the walk, and its code costs up to 4 % everywhere, so that only short windows take
// it.  Forward, without and with it: window 256, 4 sinks 39.6 and 38.7 us (8192 tokens
// in seven sequences, 16 / 8 heads of 128), 62.7 and 58.6 (8 x 2432, 12 heads of 64);
// window 1024 54.0 and 55.0, 88.9 and 90.1.
enum WindowKind { kWhole = 0, kWindow = 1, kWindowNarrow = 2 };
inline int window_kind(const AttnArgs& a) {
  if (a.window >= kNoWindow) return kWhole;
  return a.window <= 512 && a.sinks > 0 && (a.sinks - 1) % 128 < 32 ? kWindowNarrow : kWindow;
}

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
// Adds up the parts of split key blocks, if there are any.
cudaError_t launch_attn_join(const AttnArgs& a, int dtype, cudaStream_t s);
// delta_i = <do_i, o_i>; zero for rows outside the sequences.
cudaError_t launch_attn_delta(const AttnArgs& a, int dtype, cudaStream_t s);

}  // namespace normpre
