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
// A lane holds eight pairs of its row (16 values) and with them the pairs' cos
// and sin, which it forms once per token and uses for all of its heads; 1 to 16
// lanes share a row.  Half-split pairs (i, i + R/2) are two runs of up to eight
// values, read V at a time (V: the largest of 8, 4, 2, 1 that divides R/2, so
// that no access leaves its alignment); interleaved pairs two runs of eight.
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
  if constexpr (INTER) {
    t.a = 16 * u;
    t.b = 16 * u + 8;
    t.na = max(0, min(8, g.dim - t.a));
    t.nb = max(0, min(8, g.dim - t.b));
  } else if (u < g.rot_units) {
    t.a = 8 * u;
    t.b = g.half + 8 * u;
    t.na = t.nb = min(8, g.half - 8 * u);
  } else {
    t.a = 2 * g.half + 16 * (u - g.rot_units);
    t.b = t.a + 8;
    t.na = max(0, min(8, g.dim - t.a));
    t.nb = max(0, min(8, g.dim - t.b));
  }
  return t;
}

template <typename T, int V> struct alignas(V * sizeof(T)) Vec { T v[V]; };

// Runs of values between memory and registers, V at a time; values past the
// run are zero.
template <typename T, int V>
__device__ __forceinline__ void load_run(const T* p, int n, float* v) {
  constexpr int L = V * sizeof(T) > 16 ? 16 / sizeof(T) : V;
#pragma unroll
  for (int i = 0; i < 8; i += L) {
    Vec<T, L> x;
    if (i < n) {
      x = *reinterpret_cast<const Vec<T, L>*>(p + i);
#pragma unroll
      for (int e = 0; e < L; ++e) v[i + e] = to_f32(x.v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < L; ++e) v[i + e] = 0.f;
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_run(T* p, int n, const float* v) {
  constexpr int L = V * sizeof(T) > 16 ? 16 / sizeof(T) : V;
#pragma unroll
  for (int i = 0; i < 8; i += L)
    if (i < n) {
      Vec<T, L> x;
#pragma unroll
      for (int e = 0; e < L; ++e) x.v[e] = from_f32<T>(v[i + e]);
      *reinterpret_cast<Vec<T, L>*>(p + i) = x;
    }
}

// The lane's 16 values turned by its angles (`back`: by minus them).
template <bool INTER>
__device__ __forceinline__ void turn(float (&y)[16], const float (&c)[8], const float (&s)[8], uint32_t turned, bool back) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float& p = INTER ? y[2 * e] : y[e];
    float& q = INTER ? y[2 * e + 1] : y[8 + e];
    const float sn = back ? -s[e] : s[e];
    const float u = p * c[e] - q * sn, v = p * sn + q * c[e];
    if (turned >> e & 1u) {
      p = u;
      q = v;
    }
  }
}

__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ float squares(const float (&x)[16]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
  return sum;
}

// x becomes xh; returns the factor r that did it (0 where x has no finite norm).
__device__ __forceinline__ float normalize(float (&x)[16], const RotArgs& g) {
  float sum = row_sum(squares(x), g.lanes), scale = 1.f;
  // Where squares leave fp32's range the row is scaled by a power of two first.
  const bool large = !(sum < 0x1p126f);
  if (__any_sync(0xffffffffu, large)) {
    scale = large ? 0x1p-96f : 1.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= scale;
    sum = row_sum(squares(x), g.lanes);
  }
  const float m = fmaf(sum, g.inv_dim, g.eps * scale * scale);
  float r = rsqrtf(m);
  // one Newton step: rsqrtf may be off by two units in the last place
  if (m < INFINITY) r = fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r);
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] *= r;
  return r * scale;
}

// Each warp walks its share of the (token group, head) units: 32 / lanes tokens
// of a head at once.  BWD: gradients.
template <typename T, int V, bool INTER, bool BWD>
__global__ void __launch_bounds__(kThreads) k_qkrot(const __grid_constant__ RotArgs g) {
  const int side = blockIdx.x >= g.ctas;
  const int cta = side ? blockIdx.x - g.ctas : blockIdx.x, ctas = side ? gridDim.x - g.ctas : g.ctas;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int u = lane & (g.lanes - 1), rows = 32 / g.lanes, sub = lane / g.lanes;
  const Unit t = unit_of<INTER>(g, u);
  const int heads = g.heads[side];
  const int64_t units = (g.tokens + rows - 1) / rows * heads;
  const int64_t n_warps = static_cast<int64_t>(ctas) * kWarps, w = static_cast<int64_t>(cta) * kWarps + warp;
  int64_t unit = units * w / n_warps, group = unit / heads;
  const int64_t end = units * (w + 1) / n_warps;
  int head = static_cast<int>(unit - group * heads);
  uint32_t turned = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (8 * u + e < g.half && (INTER || u < g.rot_units)) turned |= 1u << e;
  float wt[16], dw[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const bool in = e < 8 ? e < t.na : e - 8 < t.nb;
    wt[e] = in ? weight(g, side, e < 8 ? t.a + e : t.b + e - 8) : 0.f;
    dw[e] = 0.f;
  }
  float c[8], s[8];
  bool fresh = true;
  for (; unit < end; ++unit) {
    const int64_t token = group * rows + sub;
    const bool live = token < g.used;
    if (fresh) {
      int64_t p = 0;
      if (turned && live) p = g.pos64 ? static_cast<const int64_t*>(g.pos)[token] : static_cast<const int*>(g.pos)[token];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = 1.f;
        s[e] = 0.f;
        if (turned >> e & 1u) circle(static_cast<uint64_t>(p) * g.turns[8 * u + e], c[e], s[e]);
      }
      fresh = false;
    }
    const int na = live ? t.na : 0, nb = live ? t.nb : 0;
    float x[16], y[16];
    float r = 1.f;
    if (!BWD || g.norm) {
      const T* px = static_cast<const T*>(g.x[side].p) + token * g.x[side].ts + head * g.x[side].hs;
      load_run<T, V>(px + t.a, na, x);
      load_run<T, V>(px + t.b, nb, x + 8);
      if (g.norm) r = normalize(x, g);
    }
    if constexpr (BWD) {
      const T* pz = static_cast<const T*>(g.dz[side].p) + token * g.dz[side].ts + head * g.dz[side].hs;
      load_run<T, V>(pz + t.a, na, y);
      load_run<T, V>(pz + t.b, nb, y + 8);
      turn<INTER>(y, c, s, turned, true);
      if (g.norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          dw[e] = fmaf(y[e], x[e], dw[e]);
          y[e] *= wt[e];
          sum = fmaf(y[e], x[e], sum);
        }
        const float m = row_sum(sum, g.lanes) * g.inv_dim;
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = r * fmaf(-x[e], m, y[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = x[e] * wt[e];
      turn<INTER>(y, c, s, turned, false);
    }
    if (!live) {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = 0.f;
    }
    if (token < g.tokens) {
      T* po = static_cast<T*>(g.out[side].p) + token * g.out[side].ts + head * g.out[side].hs;
      store_run<T, V>(po + t.a, t.na, y);
      store_run<T, V>(po + t.b, t.nb, y + 8);
    }
    if (++head == heads) {
      head = 0;
      ++group;
      fresh = true;
    }
  }
  if constexpr (BWD) {
    // the CTA's weight gradients: over the rows of a warp, then over the warps
    if (!g.part) return;
    __shared__ float sm[kWarps][16 * 16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      for (int o = g.lanes; o < 32; o <<= 1) dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], o);
      if (sub == 0) sm[warp][16 * u + e] = dw[e];
    }
    __syncthreads();
    if (threadIdx.x < 16 * g.lanes) {
      const Unit m = unit_of<INTER>(g, threadIdx.x >> 4);
      const int e = threadIdx.x & 15;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) sum += sm[i][threadIdx.x];
      if (e < 8 ? e < m.na : e - 8 < m.nb)
        g.part[static_cast<int64_t>(blockIdx.x) * g.dim + (e < 8 ? m.a + e : m.b + e - 8)] = sum;
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

template <typename T, bool BWD>
void launch(const RotArgs& g, int v, bool inter, unsigned ctas, cudaStream_t s) {
  if (inter) k_qkrot<T, 8, true, BWD><<<ctas, kThreads, 0, s>>>(g);
  else if (v == 8) k_qkrot<T, 8, false, BWD><<<ctas, kThreads, 0, s>>>(g);
  else if (v == 4) k_qkrot<T, 4, false, BWD><<<ctas, kThreads, 0, s>>>(g);
  else if (v == 2) k_qkrot<T, 2, false, BWD><<<ctas, kThreads, 0, s>>>(g);
  else k_qkrot<T, 1, false, BWD><<<ctas, kThreads, 0, s>>>(g);
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
  g->rot_units = static_cast<int>(cdiv(p->half, 8));
  const int units = c.interleaved ? static_cast<int>(cdiv(c.head_dim, 16))
                                  : g->rot_units + static_cast<int>(cdiv(c.head_dim - 2 * p->half, 16));
  for (g->lanes = 1; g->lanes < units;) g->lanes *= 2;
  for (int i = 0; i < p->half; ++i) g->turns[i] = p->turns[i];
  return NORMPRE_OK;
}

// Shares the CTAs out by heads, every warp at least one unit; returns their number.
unsigned share(RotArgs* g, int per_sm) {
  const int64_t groups = cdiv(g->tokens, 32 / g->lanes);
  const int64_t most = std::min<int64_t>(kMaxCtas, static_cast<int64_t>(device_sm_count()) * per_sm);
  const int64_t all = g->heads[0] + g->heads[1];
  const int64_t q = std::max<int64_t>(1, most * g->heads[0] / all), k = std::max<int64_t>(1, most - q);
  g->ctas = static_cast<int>(std::min(q, cdiv(groups * g->heads[0], kWarps)));
  return static_cast<unsigned>(g->ctas + std::min(k, cdiv(groups * g->heads[1], kWarps)));
}

// The most values that one access may take: of a run that starts at a multiple of half.
int width(int half) { return half % 8 == 0 ? 8 : half % 4 == 0 ? 4 : half % 2 == 0 ? 2 : 1; }

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
  const unsigned ctas = share(&g, 4);
  if (c.dtype == NORMPRE_BF16) launch<bf16, false>(g, width(p->half), c.interleaved, ctas, s);
  else launch<float, false>(g, width(p->half), c.interleaved, ctas, s);
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
    ctas = share(&g, 2);
    if (c.dtype == NORMPRE_BF16) launch<bf16, true>(g, width(p->half), c.interleaved, ctas, s);
    else launch<float, true>(g, width(p->half), c.interleaved, ctas, s);
  }
  if (weights)
    k_qkrot_fold<<<dim3(static_cast<unsigned>(cdiv(c.head_dim, 32)), 2), dim3(32, 32), 0, s>>>(
        static_cast<const float*>(workspace), g.ctas, static_cast<int>(ctas), c.head_dim, dq_weight, dk_weight,
        weight_dtype == NORMPRE_BF16);
  return done(cudaGetLastError(), "query and key norms, backward");
}

void normpre_qkrot_free(normpre_qkrot* p) { delete p; }

}  // extern "C"
