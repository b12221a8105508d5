// Norms of queries and keys for each head with the rotation of their positions
// in the same pass, and their gradients: the normpre_qkrot_* entry points.
//
// For a row x (a token's d values of one head), with weights w and angles a_i:
//   r = 1 / sqrt(mean x^2 + eps),  xh = x r,  y = xh w,
//   z = y with the pairs of its first R values turned by their angles.
// Backward: g = dz turned back, u = g w,
//   dx = r (u - xh mean(u xh)),  dw = sum over rows of g xh.
// A row stays in registers between the sums and the result, so that every value
// is read once and written once: bound by HBM.
//
// A lane holds four pairs of a row (8 values), of two heads at once: with them
// the pairs' cos and sin, which it forms once per token and uses for all of its
// heads; 1 to 32 lanes share a row, and the rows' sums of both heads travel
// through the lanes together.  Half-split pairs (i, i + R/2) are two runs of up to
// four values, read V at a time (V: the largest of 4, 2, 1 that divides R/2, so
// that no access leaves its alignment); interleaved pairs two runs of four.
//
// Angles: a position is a whole number p, and a frequency is kept as a 64-bit
// fraction F of a turn.  p F mod 2^64 is the angle's fraction of a turn, exact
// for every p, however far: no table, no rounding that grows with p.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <string>

#include "../../include/normpre.h"
#include "common.cuh"
#include "heads.h"
#include "internal.h"

using namespace normpre;

struct normpre_qkrot {
  normpre_qkrot_config cfg;
  int half;              // pairs that turn
  uint64_t turns[64];    // a pair's frequency, 2^64 a turn
};

namespace normpre {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct RotArgs {
  HeadsView x[2], dz[2], out[2];   // queries, keys: inputs, gradients of the results, results
  const void* w[2];                // weights, null: ones
  float* part;                     // backward: weight gradients by CTA, [ctas][d]
  const void* pos;
  int pos64, w_bf16;
  int64_t tokens, used;
  int heads[2];
  int ctas;                        // CTAs of the queries; the others take the keys
  int dim, half, norm;
  int lanes;                       // lanes of a row, a power of two
  int rot_units;                   // lanes whose pairs turn (half-split)
  float eps, inv_dim;
  uint64_t turns[64];
};

__device__ __forceinline__ float weight(const RotArgs& a, int side, int i) {
  if (!a.w[side]) return 1.f;
  return a.w_bf16 ? to_f32(static_cast<const bf16*>(a.w[side])[i]) : static_cast<const float*>(a.w[side])[i];
}

// cos and sin of `turns` 2^-64 turns: to the nearest eighth of a turn first, so
// that the rest, at most 1/8, keeps all of its 24 bits.
__device__ __forceinline__ void circle(uint64_t turns, float& c, float& s) {
  const uint64_t u = turns + (uint64_t(1) << 61);
  const int quarter = static_cast<int>(u >> 62);
  const int64_t rest = static_cast<int64_t>(u & ((uint64_t(1) << 62) - 1)) - (int64_t(1) << 61);
  float cc, ss;
  sincospif(static_cast<float>(static_cast<int>(rest >> 30)) * 0x1p-33f, &ss, &cc);
  c = quarter & 1 ? ss : cc;
  s = quarter & 1 ? cc : ss;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter >= 2) s = -s;
}

// A lane's part of a row: runs of na and nb values from a and b.
struct Unit {
  int a, b, na, nb;
};
template <bool INTER>
__device__ __forceinline__ Unit unit_of(const RotArgs& g, int u) {
  Unit t;
  if (!INTER && u < g.rot_units) {
    t.a = 4 * u;
    t.b = g.half + 4 * u;
    t.na = t.nb = min(4, g.half - 4 * u);
  } else {
    t.a = INTER ? 8 * u : 2 * g.half + 8 * (u - g.rot_units);
    t.b = t.a + 4;
    t.na = max(0, min(4, g.dim - t.a));
    t.nb = max(0, min(4, g.dim - t.b));
  }
  return t;
}
// The e-th of the lane's values: where it lies in the row, -1: nowhere.
__device__ __forceinline__ int place(const Unit& t, int e) {
  return e < 4 ? (e < t.na ? t.a + e : -1) : (e - 4 < t.nb ? t.b + e - 4 : -1);
}

template <typename T, int V> struct alignas(V * sizeof(T)) Vec { T v[V]; };

// A lane's 8 values between memory and registers, V at a time; values past a run
// are zero, and not written.
template <typename T, int V> struct Raw {
  uint32_t w[8 * sizeof(T) / 4];
  // the V values at p into words i ..
  __device__ __forceinline__ void get(const T* p, int i) {
    constexpr int kBytes = V * sizeof(T);
    const int at = i * static_cast<int>(sizeof(T)) / 4;
    if constexpr (kBytes == 16) {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      w[at] = q.x; w[at + 1] = q.y; w[at + 2] = q.z; w[at + 3] = q.w;
    } else if constexpr (kBytes == 8) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      w[at] = q.x; w[at + 1] = q.y;
    } else if constexpr (kBytes == 4) {
      w[at] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[at] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p)) << (16 * (i & 1));
    }
  }
  __device__ __forceinline__ void load(const T* p, const Unit& t, bool live) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(8 * sizeof(T) / 4); ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < 4; i += V) {
      if (live && i < t.na) get(p + t.a + i, i);
      if (live && i < t.nb) get(p + t.b + i, 4 + i);
    }
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) {
    // the words stay words until here: converted where they are loaded, they
    // would be waited for there
#pragma unroll
    for (int i = 0; i < static_cast<int>(8 * sizeof(T) / 4); ++i) asm volatile("" : "+r"(w[i]));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = sizeof(T) == 4 ? __uint_as_float(w[i]) : i & 1 ? bf16hi(w[i / 2]) : bf16lo(w[i / 2]);
  }
  static __device__ __forceinline__ void store(T* p, const Unit& t, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i += V) {
      Vec<T, V> x, y;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x.v[e] = from_f32<T>(v[i + e]);
        y.v[e] = from_f32<T>(v[4 + i + e]);
      }
      if (i < t.na) *reinterpret_cast<Vec<T, V>*>(p + t.a + i) = x;
      if (i < t.nb) *reinterpret_cast<Vec<T, V>*>(p + t.b + i) = y;
    }
  }
};

// The e-th pair of a lane's values.
template <bool INTER> __device__ constexpr int first_of(int e) { return INTER ? 2 * e : e; }
template <bool INTER> __device__ constexpr int second_of(int e) { return INTER ? 2 * e + 1 : 4 + e; }

// Sums over the lanes of a row, of several values at once.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int lanes) {
  for (int o = 1; o < lanes; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

__device__ __forceinline__ float dot(const float (&x)[8], const float (&y)[8]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(x[e], y[e], sum);
  return sum;
}

// 1 / sqrt(sum / dim + eps)
__device__ __forceinline__ float inverse_root(float sum, const RotArgs& g, float eps) {
  const float m = fmaf(sum, g.inv_dim, eps);
  const float r = rsqrtf(m);
  // one Newton step: rsqrtf may be off by two units in the last place
  return m < INFINITY ? fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r) : r;
}
// Rows whose squares leave fp32's range are scaled by a power of two first.
constexpr float kLargeSum = 0x1p126f, kDown = 0x1p-96f;

// CTAs per SM, which the registers are bounded for.
template <typename T, bool BWD> constexpr int per_sm() { return BWD ? 2 : 3; }

// Each warp walks its share of the (token group, two heads) units: 32 / lanes
// tokens at once.  The next unit is on its way while one is worked on.  BWD:
// gradients.
template <typename T, int V, bool INTER, bool BWD>
__global__ void __launch_bounds__(kThreads, per_sm<T, BWD>()) k_qkrot(const __grid_constant__ RotArgs g) {
  const int side = blockIdx.x >= g.ctas;
  const int cta = side ? blockIdx.x - g.ctas : blockIdx.x, ctas = side ? gridDim.x - g.ctas : g.ctas;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int u = lane & (g.lanes - 1), rows = 32 / g.lanes, sub = lane / g.lanes;
  const Unit t = unit_of<INTER>(g, u);
  const int heads = g.heads[side], twos = (heads + 1) / 2;
  const int64_t units = (g.tokens + rows - 1) / rows * twos;
  const int64_t n_warps = static_cast<int64_t>(ctas) * kWarps, w = static_cast<int64_t>(cta) * kWarps + warp;
  int64_t unit = units * w / n_warps;
  const int64_t end = units * (w + 1) / n_warps;
  uint32_t turned = 0;
  float wt[8], dw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e < 4 && 4 * u + e < g.half && (INTER || u < g.rot_units)) turned |= 1u << e;
    const int at = place(t, e);
    wt[e] = at < 0 ? 0.f : weight(g, side, at);
    dw[e] = 0.f;
  }

  // the unit on its way: its place, values and position
  int64_t token = unit / twos * rows + sub, next_pos = 0;
  int head = 2 * static_cast<int>(unit % twos);
  Raw<T, V> nx[2], nz[2];
  const bool want_x = !BWD || g.norm;
  auto fetch = [&](bool position) {
    const bool live = token < g.used;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool in = live && head + i < heads;
      if (want_x) nx[i].load(static_cast<const T*>(g.x[side].p) + token * g.x[side].ts + (head + i) * g.x[side].hs, t, in);
      if constexpr (BWD)
        nz[i].load(static_cast<const T*>(g.dz[side].p) + token * g.dz[side].ts + (head + i) * g.dz[side].hs, t, in);
    }
    if (position) {
      next_pos = 0;
      if (turned && live) next_pos = g.pos64 ? static_cast<const int64_t*>(g.pos)[token] : static_cast<const int*>(g.pos)[token];
    }
  };
  float c[4], s[4];
  bool fresh = true;
  if (unit < end) fetch(true);
  while (unit < end) {
    float x[2][8], y[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (want_x) nx[i].unpack(x[i]);
      if constexpr (BWD) nz[i].unpack(y[i]);
    }
    if (fresh) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = 1.f;
        s[e] = 0.f;
        if (turned >> e & 1u) circle(static_cast<uint64_t>(next_pos) * g.turns[4 * u + e], c[e], s[e]);
      }
    }
    const int64_t here = token;
    const int at = head;
    ++unit;
    head += 2;
    fresh = head >= heads;
    if (fresh) {
      head = 0;
      token += rows;
    }
    if (unit < end) fetch(fresh);

    if constexpr (!BWD) {
      float r[2] = {1.f, 1.f};
      if (g.norm) {
        float sum[2] = {dot(x[0], x[0]), dot(x[1], x[1])};
        row_sums(sum, g.lanes);
        if (__any_sync(0xffffffffu, !(sum[0] < kLargeSum && sum[1] < kLargeSum))) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float scale = sum[i] < kLargeSum ? 1.f : kDown;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] *= scale;
            float again[1] = {dot(x[i], x[i])};
            row_sums(again, g.lanes);
            r[i] = inverse_root(again[0], g, g.eps * scale * scale);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) r[i] = inverse_root(sum[i], g, g.eps);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = first_of<INTER>(e), q = second_of<INTER>(e);
          const float a = x[i][p] * r[i] * wt[p], b = x[i][q] * r[i] * wt[q];
          y[i][p] = fmaf(a, c[e], -(b * s[e]));
          y[i][q] = fmaf(a, s[e], b * c[e]);
        }
    } else {
      // g in place of dz
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = first_of<INTER>(e), q = second_of<INTER>(e);
          const float a = y[i][p], b = y[i][q];
          y[i][p] = fmaf(a, c[e], b * s[e]);
          y[i][q] = fmaf(b, c[e], -(a * s[e]));
        }
      if (g.norm) {
        float sum[4], r[2], m[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sum[i] = dot(x[i], x[i]);
          sum[2 + i] = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[2 + i] = fmaf(y[i][e] * wt[e], x[i][e], sum[2 + i]);
        }
        row_sums(sum, g.lanes);
        const bool fits = sum[0] < kLargeSum && sum[1] < kLargeSum && fabsf(sum[2]) < INFINITY && fabsf(sum[3]) < INFINITY;
        if (__any_sync(0xffffffffu, !fits)) {
          // <u, x> may be out of range with x: from xh instead
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float scale = sum[i] < kLargeSum ? 1.f : kDown;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] *= scale;
            float again[1] = {dot(x[i], x[i])};
            row_sums(again, g.lanes);
            r[i] = inverse_root(again[0], g, g.eps * scale * scale);
            again[0] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[i][e] *= r[i];
              again[0] = fmaf(y[i][e] * wt[e], x[i][e], again[0]);
            }
            row_sums(again, g.lanes);
            m[i] = again[0] * g.inv_dim;
            r[i] *= scale;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            r[i] = inverse_root(sum[i], g, g.eps);
            m[i] = sum[2 + i] * g.inv_dim * r[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] *= r[i];
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            dw[e] = fmaf(y[i][e], x[i][e], dw[e]);
            y[i][e] = r[i] * fmaf(-x[i][e], m[i], y[i][e] * wt[e]);
          }
      }
    }
    if (here >= g.used) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i][e] = 0.f;
    }
    if (here < g.tokens) {
      T* po = static_cast<T*>(g.out[side].p) + here * g.out[side].ts + at * g.out[side].hs;
      Raw<T, V>::store(po, t, y[0]);
      if (at + 1 < heads) Raw<T, V>::store(po + g.out[side].hs, t, y[1]);
    }
  }
  if constexpr (BWD) {
    // the CTA's weight gradients: over the rows of a warp, then over the warps
    if (!g.part) return;
    __shared__ float sm[kWarps][8 * 32];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      for (int o = g.lanes; o < 32; o <<= 1) dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], o);
      if (sub == 0) sm[warp][8 * u + e] = dw[e];
    }
    __syncthreads();
    if (threadIdx.x < 8 * g.lanes) {
      const int to = place(unit_of<INTER>(g, threadIdx.x >> 3), threadIdx.x & 7);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) sum += sm[i][threadIdx.x];
      if (to >= 0) g.part[static_cast<int64_t>(blockIdx.x) * g.dim + to] = sum;
    }
  }
}

// Sums the CTAs' weight gradients in a fixed order: 32 columns of one weight.
__global__ void __launch_bounds__(1024) k_qkrot_fold(const float* part, int q_ctas, int ctas, int dim, void* dqw, void* dkw,
                                                     int w_bf16) {
  __shared__ float sm[32][33];
  const int side = blockIdx.y, col = 32 * blockIdx.x + threadIdx.x;
  const int first = side ? q_ctas : 0, last = side ? ctas : q_ctas;
  float sum = 0.f;
  if (col < dim)
    for (int i = first + threadIdx.y; i < last; i += 32) sum += part[static_cast<int64_t>(i) * dim + col];
  sm[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  sum = warp_sum(sm[threadIdx.x][threadIdx.y]);
  void* out = side ? dkw : dqw;
  const int to = 32 * blockIdx.x + threadIdx.y;
  if (threadIdx.x == 0 && to < dim && out) {
    if (w_bf16) static_cast<bf16*>(out)[to] = from_f32<bf16>(sum);
    else static_cast<float*>(out)[to] = sum;
  }
}

constexpr int kMaxCtas = 1024;   // of one call; the workspace holds their weight gradients

int fail(int code, const std::string& msg) {
  set_thread_error(msg);
  return code;
}
int done(cudaError_t e, const char* what) {
  return e ? fail(NORMPRE_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e)) : NORMPRE_OK;
}

// Shares the CTAs out by heads, every warp at least one unit; returns their number.
unsigned share(RotArgs* g, int per_sm) {
  const int64_t groups = cdiv(g->tokens, 32 / g->lanes);
  const int64_t most = std::min<int64_t>(kMaxCtas, static_cast<int64_t>(device_sm_count()) * per_sm);
  const int64_t twos[2] = {cdiv(g->heads[0], 2), cdiv(g->heads[1], 2)};
  const int64_t q = std::max<int64_t>(1, most * twos[0] / (twos[0] + twos[1])), k = std::max<int64_t>(1, most - q);
  g->ctas = static_cast<int>(std::min(q, cdiv(groups * twos[0], kWarps)));
  return static_cast<unsigned>(g->ctas + std::min(k, cdiv(groups * twos[1], kWarps)));
}

// Returns the number of CTAs.
template <typename T, bool BWD>
unsigned launch(RotArgs* g, int v, bool inter, cudaStream_t s) {
  const unsigned ctas = share(g, per_sm<T, BWD>());
  if (inter) k_qkrot<T, 4, true, BWD><<<ctas, kThreads, 0, s>>>(*g);
  else if (v == 4) k_qkrot<T, 4, false, BWD><<<ctas, kThreads, 0, s>>>(*g);
  else if (v == 2) k_qkrot<T, 2, false, BWD><<<ctas, kThreads, 0, s>>>(*g);
  else k_qkrot<T, 1, false, BWD><<<ctas, kThreads, 0, s>>>(*g);
  return ctas;
}

// What both directions take; fills in all but the gradients.
int base(const normpre_qkrot* p, int64_t tokens, int64_t used, const normpre_heads* q, const normpre_heads* k,
         const void* positions, int position_bytes, const void* qw, const void* kw, int w_dtype, RotArgs* g) {
  if (!p) return fail(NORMPRE_ERR_ARG, "null plan");
  const normpre_qkrot_config& c = p->cfg;
  if (tokens < 0 || tokens >= (int64_t(1) << 31)) return fail(NORMPRE_ERR_SHAPE, "tokens must be in [0, 2^31)");
  if (used < 0 || used > tokens) return fail(NORMPRE_ERR_SHAPE, "used must be in [0, tokens]");
  if (position_bytes != 4 && position_bytes != 8) return fail(NORMPRE_ERR_DTYPE, "positions must have 4 or 8 bytes");
  if (w_dtype != NORMPRE_F32 && w_dtype != NORMPRE_BF16)
    return fail(NORMPRE_ERR_DTYPE, "weights must be NORMPRE_F32 or NORMPRE_BF16");
  if (!c.norm && (qw || kw)) return fail(NORMPRE_ERR_ARG, "a plan without norms takes no weights");
  for (const void* w : {qw, kw})
    if (reinterpret_cast<uintptr_t>(w) % (w_dtype == NORMPRE_BF16 ? 2 : 4))
      return fail(NORMPRE_ERR_ALIGN, "a weight must be aligned to its elements");
  *g = RotArgs{};
  if (!tokens) return NORMPRE_OK;
  if (p->half) {
    if (!positions && used) return fail(NORMPRE_ERR_ARG, "positions: null");
    if (reinterpret_cast<uintptr_t>(positions) % position_bytes)
      return fail(NORMPRE_ERR_ALIGN, "positions must be aligned to their elements");
  }
  int rc;
  if ((rc = take_heads(q, tokens, c.n_heads, c.head_dim, c.dtype, "q", false, &g->x[0])) ||
      (rc = take_heads(k, tokens, c.n_kv_heads, c.head_dim, c.dtype, "k", false, &g->x[1])))
    return rc;
  g->w[0] = qw;
  g->w[1] = kw;
  g->pos = positions;
  g->pos64 = position_bytes == 8;
  g->w_bf16 = w_dtype == NORMPRE_BF16;
  g->tokens = tokens;
  g->used = used;
  g->heads[0] = c.n_heads;
  g->heads[1] = c.n_kv_heads;
  g->dim = c.head_dim;
  g->half = p->half;
  g->norm = c.norm;
  g->eps = c.eps;
  g->inv_dim = 1.f / static_cast<float>(c.head_dim);
  g->rot_units = static_cast<int>(cdiv(p->half, 4));
  const int units = c.interleaved ? c.head_dim / 8 : g->rot_units + static_cast<int>(cdiv(c.head_dim - 2 * p->half, 8));
  for (g->lanes = 1; g->lanes < units;) g->lanes *= 2;
  for (int i = 0; i < p->half; ++i) g->turns[i] = p->turns[i];
  return NORMPRE_OK;
}

// The most values that one access may take: of a run that starts at a multiple of half.
int width(int half) { return half % 4 == 0 ? 4 : half % 2 == 0 ? 2 : 1; }

}  // namespace
}  // namespace normpre

extern "C" {

int normpre_qkrot_init(const normpre_qkrot_config* cfg, const double* frequencies, normpre_qkrot** out) {
  if (!cfg || !out) return fail(NORMPRE_ERR_ARG, "null argument");
  *out = nullptr;
  if (cfg->dtype != NORMPRE_F32 && cfg->dtype != NORMPRE_BF16)
    return fail(NORMPRE_ERR_DTYPE, "dtype must be NORMPRE_F32 or NORMPRE_BF16");
  if (cfg->n_heads < 1 || cfg->n_kv_heads < 1 || cfg->n_heads > 65535 || cfg->n_kv_heads > 65535)
    return fail(NORMPRE_ERR_SHAPE, "n_heads and n_kv_heads must be in [1, 65535]");
  if (cfg->head_dim < 8 || cfg->head_dim > 128 || cfg->head_dim % 8)
    return fail(NORMPRE_ERR_SHAPE, "head_dim must be a multiple of 8 in [8, 128]");
  if (cfg->rotary_dim < 0 || cfg->rotary_dim > cfg->head_dim || cfg->rotary_dim % 2)
    return fail(NORMPRE_ERR_SHAPE, "rotary_dim must be even and in [0, head_dim]");
  if ((cfg->interleaved | 1) != 1 || (cfg->norm | 1) != 1) return fail(NORMPRE_ERR_ARG, "interleaved and norm must be 0 or 1");
  if (cfg->norm && !(cfg->eps >= 1e-30f && cfg->eps < INFINITY)) return fail(NORMPRE_ERR_ARG, "eps must be finite and >= 1e-30");
  if (cfg->rotary_dim && !frequencies) return fail(NORMPRE_ERR_ARG, "frequencies: null");
  std::unique_ptr<normpre_qkrot> p(new (std::nothrow) normpre_qkrot());
  if (!p) return fail(NORMPRE_ERR_CUDA, "out of host memory");
  p->cfg = *cfg;
  p->half = cfg->rotary_dim / 2;
  for (int i = 0; i < p->half; ++i) {
    if (!(std::fabs(frequencies[i]) <= 1e6)) return fail(NORMPRE_ERR_ARG, "a frequency must be finite and at most 1e6 in absolute value");
    double t = frequencies[i] * 0.15915494309189533577;   // 1 / (2 pi)
    t -= std::floor(t);
    p->turns[i] = t >= 1.0 ? 0 : static_cast<uint64_t>(std::ldexp(t, 64));
  }
  *out = p.release();
  return NORMPRE_OK;
}

int normpre_qkrot_bytes(const normpre_qkrot* p, int64_t* bytes) {
  if (!p || !bytes) return fail(NORMPRE_ERR_ARG, "null argument");
  *bytes = static_cast<int64_t>(kMaxCtas) * p->cfg.head_dim * static_cast<int64_t>(sizeof(float));
  return NORMPRE_OK;
}

int normpre_qkrot_forward(const normpre_qkrot* p, int64_t tokens, int64_t used, const normpre_heads* q,
                          const normpre_heads* k, const void* positions, int position_bytes, const void* q_weight,
                          const void* k_weight, int weight_dtype, const normpre_heads* q_out, const normpre_heads* k_out,
                          void* stream) {
  RotArgs g;
  int rc = base(p, tokens, used, q, k, positions, position_bytes, q_weight, k_weight, weight_dtype, &g);
  if (rc || !tokens) return rc;
  const normpre_qkrot_config& c = p->cfg;
  if ((rc = take_heads(q_out, tokens, c.n_heads, c.head_dim, c.dtype, "q_out", true, &g.out[0])) ||
      (rc = take_heads(k_out, tokens, c.n_kv_heads, c.head_dim, c.dtype, "k_out", true, &g.out[1])))
    return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (c.dtype == NORMPRE_BF16) launch<bf16, false>(&g, width(p->half), c.interleaved, s);
  else launch<float, false>(&g, width(p->half), c.interleaved, s);
  return done(cudaGetLastError(), "query and key norms");
}

int normpre_qkrot_backward(const normpre_qkrot* p, int64_t tokens, int64_t used, const normpre_heads* q,
                           const normpre_heads* k, const void* positions, int position_bytes, const void* q_weight,
                           const void* k_weight, int weight_dtype, const normpre_heads* dq_out,
                           const normpre_heads* dk_out, const normpre_heads* dq, const normpre_heads* dk,
                           void* dq_weight, void* dk_weight, void* workspace, void* stream) {
  RotArgs g;
  int rc = base(p, tokens, used, q, k, positions, position_bytes, q_weight, k_weight, weight_dtype, &g);
  if (rc) return rc;
  const normpre_qkrot_config& c = p->cfg;
  if (!c.norm && (dq_weight || dk_weight)) return fail(NORMPRE_ERR_ARG, "a plan without norms has no weight gradients");
  if ((dq_weight && !q_weight) || (dk_weight && !k_weight))
    return fail(NORMPRE_ERR_ARG, "a weight's gradient without the weight");
  const bool weights = dq_weight || dk_weight;
  if (weights) {
    if (!workspace) return fail(NORMPRE_ERR_ARG, "workspace: null");
    if (reinterpret_cast<uintptr_t>(workspace) & 15u) return fail(NORMPRE_ERR_ALIGN, "workspace must be 16-byte aligned");
    for (const void* w : {dq_weight, dk_weight})
      if (reinterpret_cast<uintptr_t>(w) % (weight_dtype == NORMPRE_BF16 ? 2 : 4))
        return fail(NORMPRE_ERR_ALIGN, "a weight's gradient must be aligned to its elements");
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  unsigned ctas = 0;
  if (tokens) {
    if ((rc = take_heads(dq_out, tokens, c.n_heads, c.head_dim, c.dtype, "dq_out", false, &g.dz[0])) ||
        (rc = take_heads(dk_out, tokens, c.n_kv_heads, c.head_dim, c.dtype, "dk_out", false, &g.dz[1])) ||
        (rc = take_heads(dq, tokens, c.n_heads, c.head_dim, c.dtype, "dq", true, &g.out[0])) ||
        (rc = take_heads(dk, tokens, c.n_kv_heads, c.head_dim, c.dtype, "dk", true, &g.out[1])))
      return rc;
    g.part = weights ? static_cast<float*>(workspace) : nullptr;
    ctas = c.dtype == NORMPRE_BF16 ? launch<bf16, true>(&g, width(p->half), c.interleaved, s)
                                   : launch<float, true>(&g, width(p->half), c.interleaved, s);
  }
  if (weights)
    k_qkrot_fold<<<dim3(static_cast<unsigned>(cdiv(c.head_dim, 32)), 2), dim3(32, 32), 0, s>>>(
        static_cast<const float*>(workspace), g.ctas, static_cast<int>(ctas), c.head_dim, dq_weight, dk_weight,
        weight_dtype == NORMPRE_BF16);
  return done(cudaGetLastError(), "query and key norms, backward");
}

void normpre_qkrot_free(normpre_qkrot* p) { delete p; }

}  // extern "C"
