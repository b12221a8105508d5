// Packed causal attention in fp32 arithmetic: one CTA of 256 threads per 64
// rows of one sequence and head.
//
// With a window both walk only the tiles that the rows see: the window's, and
// those of the sequence's first rows that stay visible.
//
// Forward: the CTA's 64 query rows meet the sequence's keys 64 at a time,
// starting with the block on the diagonal (where every row sees at least
// itself, so the running maximum is finite from the first block on), with the
// running maximum and sum of the softmax; one pass over K and V.
// Backward: P is formed again from the log-sum.  Half of the CTAs own 64 keys
// (dK, dV summed over the query heads of the group and the later query blocks),
// half 64 queries (dQ): each output is summed by one CTA in a fixed order, at
// the price of forming the scores twice.
// Differences of scores are taken before the factor log2(e) of the exponentials:
// that factor's rounding then is one of the difference, not of the score.
//
// A thread holds a 4 x 4 piece of a 64 x 64 score tile (rows ty + 16 r, columns
// tx + 16 c) and a 4 x (D / 16) piece of a 64 x D product; tiles lie in shared
// memory with rows padded by 4 floats, which spreads the 16-byte reads of 8
// consecutive rows over all banks.
// Bound by the fp32 FMA pipe (8 16-byte reads feed 64 FMAs of a 4 x 4 piece) and,
// at few rows, by the longest sequence's CTAs; not by HBM.  1000 tokens in three
// sequences, 12 heads of 64: forward 0.062 ms (14 TFLOP/s), backward 0.127 ms (16),
// where the longest CTAs pass ten tiles of 8200 FMA cycles each, two CTAs an SM.
// 8 x 1024 tokens: 0.39 ms (33 TFLOP/s) and 1.27 ms (25).  With a window of 100 and
// 3 sinks the three sequences take 0.088 to 0.094 ms backward: 64 x 64 tiles of which 45 % is
// visible, 600 CTAs of two to four tiles in two rounds.  Sinks take a fourth of a
// tile's products where 16 keys or fewer are visible (forward, 2000 tokens 63 -> 55 us).
#include <type_traits>

#include "attn.h"
#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace normpre {
namespace {

constexpr int kB = 64;              // rows and keys of a tile
constexpr int kThreads = 256;
constexpr int kPs = kB + 4;         // row stride of a score tile
constexpr float kLog2e = 1.4426950408889634f;

template <int DP> __host__ __device__ constexpr int ld() { return DP + 4; }

// Groups of 16 keys of a tile: four, or one where no more than 16 are visible, as
// sinks.
template <int N> using Groups = std::integral_constant<int, N>;

// 64 rows from `row0` of a head into shared memory; rows at or past `rows` and
// columns at or past `dim` are zero.
template <typename T, int DP> struct Tile {
  static constexpr int kEach = kB * (DP / 8) / kThreads;   // groups of 8 elements of a thread
  float v[kEach][8];
  __device__ __forceinline__ void fetch(const AttnTensor& t, int64_t row0, int rows, int head, int dim) {
    const T* src = static_cast<const T*>(t.p) + row0 * t.ts + head * t.hs;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = threadIdx.x + kThreads * i, r = e / (DP / 8), c = (e % (DP / 8)) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
      if (r < rows && c < dim) load8(src + r * t.ts + c, v[i]);
    }
  }
  __device__ __forceinline__ void put(float* dst) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = threadIdx.x + kThreads * i, r = e / (DP / 8), c = (e % (DP / 8)) * 8;
#pragma unroll
      for (int k = 0; k < 8; k += 4)
        *reinterpret_cast<float4*>(dst + r * ld<DP>() + c + k) = make_float4(v[i][k], v[i][k + 1], v[i][k + 2], v[i][k + 3]);
    }
  }
};
template <typename T, int DP>
__device__ __forceinline__ void load_tile(float* dst, const AttnTensor& t, int64_t row0, int rows, int head, int dim) {
  Tile<T, DP> x;
  x.fetch(t, row0, rows, head, dim);
  x.put(dst);
}
// Two tiles of the same rows, their reads in flight together.
template <typename T, int DP>
__device__ __forceinline__ void load_tiles(float* dst0, const AttnTensor& t0, float* dst1, const AttnTensor& t1,
                                           int64_t row0, int rows, int head, int dim) {
  Tile<T, DP> x, y;
  x.fetch(t0, row0, rows, head, dim);
  y.fetch(t1, row0, rows, head, dim);
  x.put(dst0);
  y.put(dst1);
}

// s[r][c] = <A row ty + 16 r, B row tx + 16 c>, of the first 16 NC rows of B
template <int DP, int NC = 4>
__device__ __forceinline__ void scores(const float* A, const float* B, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) s[r][c] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 a[4], b[NC];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * ld<DP>() + d);
      if (i < NC) b[i] = *reinterpret_cast<const float4*>(B + (tx + 16 * i) * ld<DP>() + d);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        s[r][c] = fmaf(a[r].x, b[c].x, s[r][c]);
        s[r][c] = fmaf(a[r].y, b[c].y, s[r][c]);
        s[r][c] = fmaf(a[r].z, b[c].z, s[r][c]);
        s[r][c] = fmaf(a[r].w, b[c].w, s[r][c]);
      }
  }
}

// acc[r] (row ty + 16 r, columns 4 tx + 64 k ..) += sum_j P[ty + 16 r][j] V[j][...], j < 16 NC
template <int DP, int NC = 4>
__device__ __forceinline__ void accumulate(const float* P, const float* V, int ty, int tx, float4 (&acc)[4][DP / 64]) {
#pragma unroll 2
  for (int j = 0; j < 16 * NC; j += 4) {
    float4 p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = *reinterpret_cast<const float4*>(P + (ty + 16 * r) * kPs + j);
#pragma unroll
    for (int jj = 0; jj < 4; ++jj)
#pragma unroll
      for (int k = 0; k < DP / 64; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(V + (j + jj) * ld<DP>() + 4 * tx + 64 * k);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float w = jj == 0 ? p[r].x : jj == 1 ? p[r].y : jj == 2 ? p[r].z : p[r].w;
          acc[r][k].x = fmaf(w, v.x, acc[r][k].x);
          acc[r][k].y = fmaf(w, v.y, acc[r][k].y);
          acc[r][k].z = fmaf(w, v.z, acc[r][k].z);
          acc[r][k].w = fmaf(w, v.w, acc[r][k].w);
        }
      }
  }
}

template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v, float w) {
  if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<float4*>(p) = make_float4(v.x * w, v.y * w, v.z * w, v.w * w);
  } else {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x * w, v.y * w), pack_bf16x2(v.z * w, v.w * w));
  }
}

template <typename T, int DP>
__device__ __forceinline__ void store_tile(const AttnTensor& t, int64_t row0, int rows, int head, int dim, int ty,
                                           int tx, const float4 (&acc)[4][DP / 64], const float (&w)[4]) {
  T* dst = static_cast<T*>(t.p) + row0 * t.ts + head * t.hs;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) {
      const int row = ty + 16 * r, c = 4 * tx + 64 * k;
      if (row < rows && c < dim) store4(dst + row * t.ts + c, acc[r][k], w[r]);
    }
}

// Zeroes 64 rows from `row0` of a head.
template <typename T>
__device__ __forceinline__ void zero_rows(const AttnTensor& t, int64_t row0, int rows, int head, int dim) {
  T* dst = static_cast<T*>(t.p) + row0 * t.ts + head * t.hs;
  const float z[8] = {};
  for (int e = threadIdx.x; e < rows * (dim / 8); e += kThreads)
    store8(dst + (e / (dim / 8)) * t.ts + (e % (dim / 8)) * 8, z);
}

// What a CTA works on: 64 rows of a sequence, or 64 rows past the last one.
struct Rows {
  int64_t seq;     // the sequence's first row
  int first;       // this CTA's first row in the sequence
  int len;         // the sequence's rows; 0: rows that belong to no sequence
  AttnBlock block;
};
__device__ __forceinline__ bool rows_of(const AttnArgs& a, const AttnBlock* list, int blocks, int64_t i, Rows& w) {
  if (i < 2 * static_cast<int64_t>(blocks)) {
    const AttnBlock b = w.block = list[i >> 1];
    if (!block_fits(b, a.total)) {
      if (threadIdx.x == 0) raise_host_flag(a.flags, kFlagLists);
      return false;
    }
    w.seq = b.start;
    w.first = 128 * b.blk + 64 * static_cast<int>(i & 1);
    w.len = b.len;
    return w.first < w.len;
  }
  w.seq = a.total + 64 * (i - 2 * static_cast<int64_t>(blocks));
  w.first = w.len = 0;
  return w.seq < a.tokens;
}

// WIN: the rows have a window.  The kernels without one are kernels of their own:
// its tests in every pair of rows and its second kind of tile cost them 3 to 11 %
// forward, 1 to 3 % backward.
template <typename T, int DP, bool WIN>
__global__ void __launch_bounds__(kThreads) k_attn_fwd(const __grid_constant__ AttnArgs a) {
  extern __shared__ float sm[];
  float* Q = sm;
  float* KV = Q + kB * ld<DP>();
  float* P = KV + kB * ld<DP>();
  const int head = static_cast<int>(blockIdx.x % a.heads), kvh = head / a.group;
  Rows w;
  if (!rows_of(a, a.by_query, a.n_blocks, blockIdx.x / a.heads, w)) return;
  const int64_t row0 = w.seq + w.first;
  float* lse = a.lse + static_cast<int64_t>(head) * a.tokens + row0;
  if (!w.len) {
    const int rows = static_cast<int>(min(static_cast<int64_t>(kB), a.tokens - row0));
    zero_rows<T>(a.o, row0, rows, head, a.dim);
    if (threadIdx.x < rows) lse[threadIdx.x] = -INFINITY;
    return;
  }
  const int rows = min(kB, w.len - w.first);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_tile<T, DP>(Q, a.q, row0, rows, head, a.dim);
  float4 acc[4][DP / 64];
  float m[4], l[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) acc[r][k] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const int diag = w.first / kB;
  // keys of a tile, NC groups of 16
  auto tile = [&](int jb, auto groups) {
    constexpr int NC = decltype(groups)::value;
    const int krows = min(16 * NC, w.len - jb * kB);
    __syncthreads();
    load_tile<T, DP>(KV, a.k, w.seq + jb * kB, krows, kvh, a.dim);
    __syncthreads();
    float s[4][4];
    scores<DP, NC>(Q, KV, ty, tx, s);
    const int up = kB * (diag - jb);
    auto hidden = [&](int r, int c) {
      if constexpr (!WIN) return jb == diag && tx + 16 * c > ty + 16 * r;
      const int far = up + ty + 16 * r - tx - 16 * c;        // rows between the two
      return far < 0 || (far >= a.window && kB * jb + tx + 16 * c >= a.sinks);
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        s[r][c] = hidden(r, c) ? -INFINITY : s[r][c] * a.scale;
        mx = fmaxf(mx, s[r][c]);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      mx = fmaxf(mx, m[r]);
      const float keep = exp2f((m[r] - mx) * kLog2e);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float p = hidden(r, c) ? 0.f : exp2f((s[r][c] - mx) * kLog2e);
        P[(ty + 16 * r) * kPs + tx + 16 * c] = p;
        sum += p;
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l[r] = l[r] * keep + sum;
      m[r] = mx;
#pragma unroll
      for (int k = 0; k < DP / 64; ++k) {
        acc[r][k].x *= keep; acc[r][k].y *= keep; acc[r][k].z *= keep; acc[r][k].w *= keep;
      }
    }
    __syncthreads();
    load_tile<T, DP>(KV, a.v, w.seq + jb * kB, krows, kvh, a.dim);
    __syncthreads();
    accumulate<DP, NC>(P, KV, ty, tx, acc);
  };
  if constexpr (WIN) {
    const int lo = max(0, w.first - a.window + 1) / kB, sink = min(lo, (a.sinks + kB - 1) / kB);
    for (int jb = diag; jb >= 0; jb = jb > lo || jb <= sink ? jb - 1 : sink - 1) {
      if (jb < sink && a.sinks - jb * kB <= 16) tile(jb, Groups<1>());
      else tile(jb, Groups<4>());
    }
  } else {
    for (int jb = diag; jb >= 0; --jb) tile(jb, Groups<4>());
  }
  float inv[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    inv[r] = 1.f / l[r];
    if (tx == 0 && ty + 16 * r < rows) lse[ty + 16 * r] = fmaf(log2f(l[r]), 0.6931471805599453f, m[r]);
  }
  store_tile<T, DP>(a.o, row0, rows, head, a.dim, ty, tx, acc, inv);
}

// P and dS of query rows i0 .. and key rows j0 .. of a sequence, from tiles in
// shared memory; zero where i < j or past the sequence's end.  s holds
// ds / c on return, p the probabilities.
template <int DP, bool WIN, int NC = 4>
__device__ __forceinline__ void grad_scores(const AttnArgs& a, const float* Q, const float* K, const float* dO,
                                            const float* V, const float* lse, const float* delta, int i0, int j0,
                                            int len, int ty, int tx, float (&p)[4][4], float (&s)[4][4]) {
  float t[4][4];
  scores<DP, NC>(Q, K, ty, tx, t);
  scores<DP, NC>(dO, V, ty, tx, s);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = i0 + ty + 16 * r;
    const float ls = lse[ty + 16 * r], de = delta[ty + 16 * r];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int j = j0 + tx + 16 * c;
      const bool seen = i < len && j <= i && (!WIN || i - j < a.window || j < a.sinks);
      p[r][c] = seen ? exp2f(fmaf(t[r][c], a.scale, -ls) * kLog2e) : 0.f;
      s[r][c] = seen && !(WIN && sees_itself(a.window, a.sinks)) ? p[r][c] * (s[r][c] - de) : 0.f;
    }
  }
}

// The log-sums and deltas of up to 64 rows.
__device__ __forceinline__ void load_stats(const AttnArgs& a, float* lse, float* delta, int head, int64_t row0,
                                           int rows) {
  if (threadIdx.x < kB) {
    const bool in = threadIdx.x < rows;
    lse[threadIdx.x] = in ? a.lse[static_cast<int64_t>(head) * a.tokens + row0 + threadIdx.x] : 0.f;
    delta[threadIdx.x] = in ? a.delta[static_cast<int64_t>(head) * a.tokens + row0 + threadIdx.x] : 0.f;
  }
}

template <typename T, int DP, bool WIN>
__device__ __forceinline__ void owned_keys(const AttnArgs& a, int64_t item, int kvh, float* sm, float* lse, float* delta) {
  float* K = sm;
  float* V = K + kB * ld<DP>();
  float* Q = V + kB * ld<DP>();
  float* dO = Q + kB * ld<DP>();
  float* Pt = dO + kB * ld<DP>();   // P^T, then dS^T: [key][query]
  float* St = Pt + kB * kPs;
  Rows w;
  if (!rows_of(a, a.by_key, a.n_keys, item, w)) return;
  const int64_t row0 = w.seq + w.first;
  if (!w.len) {
    const int rows = static_cast<int>(min(static_cast<int64_t>(kB), a.tokens - row0));
    zero_rows<T>(a.dk, row0, rows, kvh, a.dim);
    zero_rows<T>(a.dv, row0, rows, kvh, a.dim);
    return;
  }
  KeyPart part = {0, 0, -1, w.block.part == 0};
  if constexpr (WIN) part = key_part(w.block, a.window, a.sinks, a.chunk, a.slots);
  if (!part.fits) {
    if (threadIdx.x == 0) raise_host_flag(a.flags, kFlagLists);
    return;
  }
  const int rows = min(kB, w.len - w.first);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_tiles<T, DP>(K, a.k, V, a.v, row0, rows, kvh, a.dim);
  float4 dk[4][DP / 64], dv[4][DP / 64];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) dk[r][k] = dv[r][k] = make_float4(0.f, 0.f, 0.f, 0.f);
  int begin = w.first, end = w.len;
  if constexpr (WIN) {
    // to the last row that sees any of these keys
    if (w.first >= a.sinks) end = min(end, w.first + kB - 1 + a.window);
    begin = max(begin, 128 * part.first);
    end = min(end, 128 * part.end);
  }
  for (int g = 0; g < a.group; ++g) {
    const int head = kvh * a.group + g;
    for (int i0 = begin; i0 < end; i0 += kB) {
      const int qrows = min(kB, w.len - i0);
      __syncthreads();
      load_tiles<T, DP>(Q, a.q, dO, a.dout, w.seq + i0, qrows, head, a.dim);
      load_stats(a, lse, delta, head, w.seq + i0, qrows);
      __syncthreads();
      float p[4][4], s[4][4];
      grad_scores<DP, WIN>(a, Q, K, dO, V, lse, delta, i0, w.first, w.len, ty, tx, p, s);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          Pt[(tx + 16 * c) * kPs + ty + 16 * r] = p[r][c];
          St[(tx + 16 * c) * kPs + ty + 16 * r] = s[r][c];
        }
      __syncthreads();
      accumulate<DP>(Pt, dO, ty, tx, dv);
      accumulate<DP>(St, Q, ty, tx, dk);
    }
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, c[4] = {a.scale, a.scale, a.scale, a.scale};
  if (WIN && part.slot >= 0) {
    // 128 rows of the slot, these the first or second 64
    float* p = a.partial + ((static_cast<int64_t>(part.slot) * a.kv_heads + kvh) * 2 * 128 + (w.first & 127)) * a.dim;
    const AttnTensor pk = {p, a.dim, 0}, pv = {p + 128 * a.dim, a.dim, 0};
    store_tile<float, DP>(pk, 0, rows, 0, a.dim, ty, tx, dk, one);
    store_tile<float, DP>(pv, 0, rows, 0, a.dim, ty, tx, dv, one);
    return;
  }
  store_tile<T, DP>(a.dk, row0, rows, kvh, a.dim, ty, tx, dk, c);
  store_tile<T, DP>(a.dv, row0, rows, kvh, a.dim, ty, tx, dv, one);
}

template <typename T, int DP, bool WIN>
__device__ __forceinline__ void owned_queries(const AttnArgs& a, int64_t item, int head, float* sm, float* lse, float* delta) {
  float* Q = sm;
  float* dO = Q + kB * ld<DP>();
  float* K = dO + kB * ld<DP>();
  float* V = K + kB * ld<DP>();
  float* S = V + kB * ld<DP>();
  const int kvh = head / a.group;
  Rows w;
  if (!rows_of(a, a.by_query, a.n_blocks, item, w)) return;
  const int64_t row0 = w.seq + w.first;
  if (!w.len) {
    zero_rows<T>(a.dq, row0, static_cast<int>(min(static_cast<int64_t>(kB), a.tokens - row0)), head, a.dim);
    return;
  }
  const int rows = min(kB, w.len - w.first);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_tiles<T, DP>(Q, a.q, dO, a.dout, row0, rows, head, a.dim);
  load_stats(a, lse, delta, head, row0, rows);
  float4 dq[4][DP / 64];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) dq[r][k] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto tile = [&](int j0, auto groups) {
    constexpr int NC = decltype(groups)::value;
    const int krows = min(16 * NC, w.len - j0);
    __syncthreads();
    load_tiles<T, DP>(K, a.k, V, a.v, w.seq + j0, krows, kvh, a.dim);
    __syncthreads();
    float p[4][4], s[4][4];
    grad_scores<DP, WIN, NC>(a, Q, K, dO, V, lse, delta, w.first, j0, w.len, ty, tx, p, s);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < NC; ++c) S[(ty + 16 * r) * kPs + tx + 16 * c] = s[r][c];
    __syncthreads();
    accumulate<DP, NC>(S, K, ty, tx, dq);
  };
  if constexpr (WIN) {
    const int lo = max(0, w.first - a.window + 1) / kB * kB, sink = min(lo, (a.sinks + kB - 1) / kB * kB);
    for (int j0 = sink ? 0 : lo; j0 <= w.first; j0 = j0 + kB == sink ? lo : j0 + kB) {
      if (j0 < sink && a.sinks - j0 <= 16) tile(j0, Groups<1>());
      else tile(j0, Groups<4>());
    }
  } else {
    for (int j0 = 0; j0 <= w.first; j0 += kB) tile(j0, Groups<4>());
  }
  const float c[4] = {a.scale, a.scale, a.scale, a.scale};
  store_tile<T, DP>(a.dq, row0, rows, head, a.dim, ty, tx, dq, c);
}

// Both kinds of work in one launch, side by side for each 64 rows, so that the
// SMs that run out of the one take the other.  At head dimensions up to 64 two
// CTAs share an SM.
template <typename T, int DP, bool WIN>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) k_attn_bwd(const __grid_constant__ AttnArgs a) {
  extern __shared__ float sm[];
  __shared__ float lse[kB], delta[kB];
  const int all = a.kv_heads + a.heads, which = static_cast<int>(blockIdx.x % all);
  const int64_t item = blockIdx.x / all;
  if (which < a.kv_heads) owned_keys<T, DP, WIN>(a, item, which, sm, lse, delta);
  else owned_queries<T, DP, WIN>(a, item, which - a.kv_heads, sm, lse, delta);
}

// LANES (8 or 16) lanes per row and head, 8 columns each; EACH rows and heads a
// thread, whose loads are in flight together, where there are enough.  Index: type
// of the number of rows and heads, 32 bits where they do (the division took most of
// the time).  Bound by HBM: 8192 rows, 16 heads of 128 in bf16, 67 MB in 11 us.
template <typename T, int LANES, int EACH, typename Index>
__global__ void __launch_bounds__(256) k_attn_delta(const __grid_constant__ AttnArgs a) {
  constexpr int kStep = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  float s[EACH];
  Index row[EACH];
  int head[EACH];
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const Index i = (static_cast<Index>(blockIdx.x) * EACH + u) * kStep + threadIdx.x / LANES;   // token-major
    row[u] = i / static_cast<Index>(a.heads);
    head[u] = static_cast<int>(i - row[u] * a.heads);
    s[u] = 0.f;
    if (row[u] < a.total && lane * 8 < a.dim) {
      float x[8], y[8];
      load8(static_cast<const T*>(a.o.p) + row[u] * a.o.ts + head[u] * a.o.hs + lane * 8, x);
      load8(static_cast<const T*>(a.dout.p) + row[u] * a.dout.ts + head[u] * a.dout.hs + lane * 8, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[u] = fmaf(x[e], y[e], s[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) s[u] += __shfl_xor_sync(0xffffffffu, s[u], o);
    if (lane == 0 && row[u] < a.total) a.delta[static_cast<int64_t>(head[u]) * a.tokens + row[u]] = s[u];
  }
}

// `each`: CTAs for every 64 rows.
template <auto kernel>
cudaError_t run(const AttnArgs& a, int each, size_t smem, cudaStream_t s) {
  const cudaError_t e = allow_smem<kernel>(smem);
  if (e) return e;
  const int64_t ctas = (2 * static_cast<int64_t>(each == a.heads ? a.n_blocks : max(a.n_blocks, a.n_keys)) + cdiv(a.tokens - a.total, kB)) * each;
  if (!ctas) return cudaSuccess;
  if (ctas >= (int64_t(1) << 31)) return cudaErrorInvalidConfiguration;
  kernel<<<static_cast<unsigned>(ctas), kThreads, smem, s>>>(a);
  return cudaGetLastError();
}

template <int DP> constexpr size_t fwd_smem() { return sizeof(float) * (2 * kB * ld<DP>() + kB * kPs); }
template <int DP> constexpr size_t bwd_smem() { return sizeof(float) * (4 * kB * ld<DP>() + 2 * kB * kPs); }

}  // namespace

template <int DP, bool WIN>
static cudaError_t forward(const AttnArgs& a, cudaStream_t s) {
  return run<k_attn_fwd<float, DP, WIN>>(a, a.heads, fwd_smem<DP>(), s);
}
cudaError_t launch_attn_forward_simt(const AttnArgs& a, cudaStream_t s) {
  if (window_kind(a) == kWhole) return a.dim <= 64 ? forward<64, false>(a, s) : forward<128, false>(a, s);
  return a.dim <= 64 ? forward<64, true>(a, s) : forward<128, true>(a, s);
}

template <int DP, bool WIN>
static cudaError_t backward(const AttnArgs& a, cudaStream_t s) {
  return run<k_attn_bwd<float, DP, WIN>>(a, a.kv_heads + a.heads, bwd_smem<DP>(), s);
}
cudaError_t launch_attn_backward_simt(const AttnArgs& a, cudaStream_t s) {
  if (window_kind(a) == kWhole) return a.dim <= 64 ? backward<64, false>(a, s) : backward<128, false>(a, s);
  return a.dim <= 64 ? backward<64, true>(a, s) : backward<128, true>(a, s);
}

// One CTA for 16 rows of dk or dv of a split key block and head: 16 lanes a row,
// eight columns each.  Bound by the latency of its few loads.
template <typename T>
static __global__ void __launch_bounds__(256) k_attn_join(const __grid_constant__ AttnArgs a) {
  const int head = blockIdx.y, row = 16 * (blockIdx.x & 7) + threadIdx.x / 16, c = 8 * (threadIdx.x & 15);
  const AttnBlock b = a.by_split[blockIdx.x >> 3];
  int n = 0;
  if (block_fits(b, a.total) && 128 * b.blk + 128 <= b.len && a.chunk > 0)
    n = key_parts(last_query(b.blk, b.len, a.window, a.sinks) - b.blk + 1, a.chunk);
  if (n < 2 || b.part < 0 || n > a.slots - b.part) {
    if (threadIdx.x == 0) raise_host_flag(a.flags, kFlagLists);
    return;
  }
  if (c >= a.dim) return;
  const int which = blockIdx.z;
  float sum[8] = {};
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    float v[8];
    load8(a.partial + (((static_cast<int64_t>(b.part + i) * a.kv_heads + head) * 2 + which) * 128 + row) * a.dim + c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
  }
  const AttnTensor& t = which ? a.dv : a.dk;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] *= which ? 1.f : a.scale;
  store8(static_cast<T*>(t.p) + (static_cast<int64_t>(b.start) + 128 * b.blk + row) * t.ts + head * t.hs + c, sum);
}

cudaError_t launch_attn_join(const AttnArgs& a, int dtype, cudaStream_t s) {
  if (!a.n_split) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>(8 * a.n_split), static_cast<unsigned>(a.kv_heads), 2);
  if (dtype == 0) k_attn_join<float><<<grid, 256, 0, s>>>(a);
  else k_attn_join<bf16><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, int LANES>
static cudaError_t delta(const AttnArgs& a, cudaStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.total) * a.heads, each = 256 / LANES;
  if (!rows) return cudaSuccess;
  const bool many = rows > 8 * each * device_sm_count();
  const int64_t ctas = cdiv(rows, many ? 4 * each : each);
  if (ctas >= (int64_t(1) << 31)) return cudaErrorInvalidConfiguration;
  const unsigned grid = static_cast<unsigned>(ctas);
  if (!many) k_attn_delta<T, LANES, 1, int><<<grid, 256, 0, s>>>(a);
  else if (rows < (int64_t(1) << 30)) k_attn_delta<T, LANES, 4, int><<<grid, 256, 0, s>>>(a);
  else k_attn_delta<T, LANES, 4, int64_t><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T>
static cudaError_t delta(const AttnArgs& a, cudaStream_t s) {
  return a.dim <= 64 ? delta<T, 8>(a, s) : delta<T, 16>(a, s);
}

cudaError_t launch_attn_delta(const AttnArgs& a, int dtype, cudaStream_t s) {
  return dtype == 0 ? delta<float>(a, s) : delta<bf16>(a, s);
}

}  // namespace normpre
