// Packed causal attention in fp32 arithmetic: one CTA of 256 threads per 64
// rows of one sequence and head.
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
// 8 x 1024 tokens: 0.39 ms (33 TFLOP/s) and 1.27 ms (25).
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

// s[r][c] = <A row ty + 16 r, B row tx + 16 c>
template <int DP>
__device__ __forceinline__ void scores(const float* A, const float* B, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) s[r][c] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * ld<DP>() + d);
      b[i] = *reinterpret_cast<const float4*>(B + (tx + 16 * i) * ld<DP>() + d);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = fmaf(a[r].x, b[c].x, s[r][c]);
        s[r][c] = fmaf(a[r].y, b[c].y, s[r][c]);
        s[r][c] = fmaf(a[r].z, b[c].z, s[r][c]);
        s[r][c] = fmaf(a[r].w, b[c].w, s[r][c]);
      }
  }
}

// acc[r] (row ty + 16 r, columns 4 tx + 64 k ..) += sum_j P[ty + 16 r][j] V[j][...]
template <int DP>
__device__ __forceinline__ void accumulate(const float* P, const float* V, int ty, int tx, float4 (&acc)[4][DP / 64]) {
#pragma unroll 2
  for (int j = 0; j < kB; j += 4) {
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
};
__device__ __forceinline__ bool rows_of(const AttnArgs& a, const AttnBlock* list, int64_t i, Rows& w) {
  if (i < 2 * static_cast<int64_t>(a.n_blocks)) {
    const AttnBlock b = list[i >> 1];
    if (!block_fits(b, a.total)) {
      if (threadIdx.x == 0) raise_host_flag(a.flags, kFlagLists);
      return false;
    }
    w.seq = b.start;
    w.first = 128 * b.blk + 64 * static_cast<int>(i & 1);
    w.len = b.len;
    return w.first < w.len;
  }
  w.seq = a.total + 64 * (i - 2 * static_cast<int64_t>(a.n_blocks));
  w.first = w.len = 0;
  return w.seq < a.tokens;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) k_attn_fwd(const __grid_constant__ AttnArgs a) {
  extern __shared__ float sm[];
  float* Q = sm;
  float* KV = Q + kB * ld<DP>();
  float* P = KV + kB * ld<DP>();
  const int head = static_cast<int>(blockIdx.x % a.heads), kvh = head / a.group;
  Rows w;
  if (!rows_of(a, a.by_query, blockIdx.x / a.heads, w)) return;
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
  for (int jb = diag; jb >= 0; --jb) {
    const int krows = min(kB, w.len - jb * kB);
    __syncthreads();
    load_tile<T, DP>(KV, a.k, w.seq + jb * kB, krows, kvh, a.dim);
    __syncthreads();
    float s[4][4];
    scores<DP>(Q, KV, ty, tx, s);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = jb == diag && tx + 16 * c > ty + 16 * r ? -INFINITY : s[r][c] * a.scale;
        mx = fmaxf(mx, s[r][c]);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      mx = fmaxf(mx, m[r]);
      const float keep = exp2f((m[r] - mx) * kLog2e);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float p = jb == diag && tx + 16 * c > ty + 16 * r ? 0.f : exp2f((s[r][c] - mx) * kLog2e);
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
    accumulate<DP>(P, KV, ty, tx, acc);
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
template <int DP>
__device__ __forceinline__ void grad_scores(const AttnArgs& a, const float* Q, const float* K, const float* dO,
                                            const float* V, const float* lse, const float* delta, int i0, int j0,
                                            int len, int ty, int tx, float (&p)[4][4], float (&s)[4][4]) {
  float t[4][4];
  scores<DP>(Q, K, ty, tx, t);
  scores<DP>(dO, V, ty, tx, s);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = i0 + ty + 16 * r;
    const float ls = lse[ty + 16 * r], de = delta[ty + 16 * r];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool seen = i < len && j0 + tx + 16 * c <= i;
      p[r][c] = seen ? exp2f(fmaf(t[r][c], a.scale, -ls) * kLog2e) : 0.f;
      s[r][c] = seen ? p[r][c] * (s[r][c] - de) : 0.f;
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

template <typename T, int DP>
__device__ __forceinline__ void owned_keys(const AttnArgs& a, int64_t item, int kvh, float* sm, float* lse, float* delta) {
  float* K = sm;
  float* V = K + kB * ld<DP>();
  float* Q = V + kB * ld<DP>();
  float* dO = Q + kB * ld<DP>();
  float* Pt = dO + kB * ld<DP>();   // P^T, then dS^T: [key][query]
  float* St = Pt + kB * kPs;
  Rows w;
  if (!rows_of(a, a.by_key, item, w)) return;
  const int64_t row0 = w.seq + w.first;
  if (!w.len) {
    const int rows = static_cast<int>(min(static_cast<int64_t>(kB), a.tokens - row0));
    zero_rows<T>(a.dk, row0, rows, kvh, a.dim);
    zero_rows<T>(a.dv, row0, rows, kvh, a.dim);
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
  for (int g = 0; g < a.group; ++g) {
    const int head = kvh * a.group + g;
    for (int i0 = w.first; i0 < w.len; i0 += kB) {
      const int qrows = min(kB, w.len - i0);
      __syncthreads();
      load_tiles<T, DP>(Q, a.q, dO, a.dout, w.seq + i0, qrows, head, a.dim);
      load_stats(a, lse, delta, head, w.seq + i0, qrows);
      __syncthreads();
      float p[4][4], s[4][4];
      grad_scores<DP>(a, Q, K, dO, V, lse, delta, i0, w.first, w.len, ty, tx, p, s);
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
  store_tile<T, DP>(a.dk, row0, rows, kvh, a.dim, ty, tx, dk, c);
  store_tile<T, DP>(a.dv, row0, rows, kvh, a.dim, ty, tx, dv, one);
}

template <typename T, int DP>
__device__ __forceinline__ void owned_queries(const AttnArgs& a, int64_t item, int head, float* sm, float* lse, float* delta) {
  float* Q = sm;
  float* dO = Q + kB * ld<DP>();
  float* K = dO + kB * ld<DP>();
  float* V = K + kB * ld<DP>();
  float* S = V + kB * ld<DP>();
  const int kvh = head / a.group;
  Rows w;
  if (!rows_of(a, a.by_query, item, w)) return;
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
  for (int j0 = 0; j0 <= w.first; j0 += kB) {
    const int krows = min(kB, w.len - j0);
    __syncthreads();
    load_tiles<T, DP>(K, a.k, V, a.v, w.seq + j0, krows, kvh, a.dim);
    __syncthreads();
    float p[4][4], s[4][4];
    grad_scores<DP>(a, Q, K, dO, V, lse, delta, w.first, j0, w.len, ty, tx, p, s);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) S[(ty + 16 * r) * kPs + tx + 16 * c] = s[r][c];
    __syncthreads();
    accumulate<DP>(S, K, ty, tx, dq);
  }
  const float c[4] = {a.scale, a.scale, a.scale, a.scale};
  store_tile<T, DP>(a.dq, row0, rows, head, a.dim, ty, tx, dq, c);
}

// Both kinds of work in one launch, side by side for each 64 rows, so that the
// SMs that run out of the one take the other.  At head dimensions up to 64 two
// CTAs share an SM.
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) k_attn_bwd(const __grid_constant__ AttnArgs a) {
  extern __shared__ float sm[];
  __shared__ float lse[kB], delta[kB];
  const int all = a.kv_heads + a.heads, which = static_cast<int>(blockIdx.x % all);
  const int64_t item = blockIdx.x / all;
  if (which < a.kv_heads) owned_keys<T, DP>(a, item, which, sm, lse, delta);
  else owned_queries<T, DP>(a, item, which - a.kv_heads, sm, lse, delta);
}

// LANES (8 or 16) lanes per row and head, 8 columns each.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_attn_delta(const __grid_constant__ AttnArgs a) {
  const int lane = threadIdx.x % LANES;
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) / LANES;   // token-major
  const int64_t row = i / a.heads;
  const int head = static_cast<int>(i - row * a.heads);
  float s = 0.f;
  if (row < a.total && lane * 8 < a.dim) {
    float x[8], y[8];
    load8(static_cast<const T*>(a.o.p) + row * a.o.ts + head * a.o.hs + lane * 8, x);
    load8(static_cast<const T*>(a.dout.p) + row * a.dout.ts + head * a.dout.hs + lane * 8, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0 && row < a.total) a.delta[static_cast<int64_t>(head) * a.tokens + row] = s;
}

// `each`: CTAs for every 64 rows.
template <auto kernel>
cudaError_t run(const AttnArgs& a, int each, size_t smem, cudaStream_t s) {
  const cudaError_t e = allow_smem<kernel>(smem);
  if (e) return e;
  const int64_t ctas = (2 * static_cast<int64_t>(a.n_blocks) + cdiv(a.tokens - a.total, kB)) * each;
  if (!ctas) return cudaSuccess;
  if (ctas >= (int64_t(1) << 31)) return cudaErrorInvalidConfiguration;
  kernel<<<static_cast<unsigned>(ctas), kThreads, smem, s>>>(a);
  return cudaGetLastError();
}

template <int DP> constexpr size_t fwd_smem() { return sizeof(float) * (2 * kB * ld<DP>() + kB * kPs); }
template <int DP> constexpr size_t bwd_smem() { return sizeof(float) * (4 * kB * ld<DP>() + 2 * kB * kPs); }

}  // namespace

cudaError_t launch_attn_forward_simt(const AttnArgs& a, cudaStream_t s) {
  return a.dim <= 64 ? run<k_attn_fwd<float, 64>>(a, a.heads, fwd_smem<64>(), s)
                     : run<k_attn_fwd<float, 128>>(a, a.heads, fwd_smem<128>(), s);
}

cudaError_t launch_attn_backward_simt(const AttnArgs& a, cudaStream_t s) {
  const int each = a.kv_heads + a.heads;
  return a.dim <= 64 ? run<k_attn_bwd<float, 64>>(a, each, bwd_smem<64>(), s)
                     : run<k_attn_bwd<float, 128>>(a, each, bwd_smem<128>(), s);
}

template <typename T>
static cudaError_t delta(const AttnArgs& a, cudaStream_t s) {
  const int lanes = a.dim <= 64 ? 8 : 16;
  const int64_t ctas = cdiv(static_cast<int64_t>(a.total) * a.heads, 256 / lanes);
  if (!ctas) return cudaSuccess;
  if (lanes == 8) k_attn_delta<T, 8><<<static_cast<unsigned>(ctas), 256, 0, s>>>(a);
  else k_attn_delta<T, 16><<<static_cast<unsigned>(ctas), 256, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_attn_delta(const AttnArgs& a, int dtype, cudaStream_t s) {
  return dtype == 0 ? delta<float>(a, s) : delta<bf16>(a, s);
}

}  // namespace normpre
