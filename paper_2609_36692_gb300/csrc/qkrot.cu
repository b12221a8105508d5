// Norms of queries and keys for each head with the rotation of their positions
// in the same pass, and their gradients: the normpre_qkrot_* entry points.
//
// For a row x (a token's d values of one head), with weights w and angles a_i:
//   r = 1 / sqrt(mean x^2 + eps),  xh = x r,  y = xh w,
//   z = y with the pairs of its first R values turned by their angles.
// Backward: g = dz turned back, u = g w,
//   dx = r (u - xh mean(u xh)),  dw = sum over rows of g xh.
// A row stays in registers between the sums and the result, so that every value
// is read once and written once.
//
// What bounds it: HBM would (16384 tokens of 16 / 8 heads of 128 in bf16: 30 us
// forward, 45 backward at 6.75 TB/s), but a unit of work, four rows, takes 250 and
// 400 instructions, of which the scheduler's 4 to 6 warps issue one in two cycles:
// 42 us and 66 (45 and 70 with the launch, 4.3 TB/s).  More warps have fewer
// registers: with four CTAs an SM instead of three, or heads one by one, 51 to 70.
//
// A lane holds four pairs of a row (8 values), in bf16 of two heads at once, and with
// them the pairs' cos and sin, which it forms once per token and uses for all of its
// heads; 1 to 32 lanes share a row, and all sums of a unit travel through the
// lanes together.  Half-split pairs (i, i + R/2) are two runs of up to
// four values, read V at a time (V: the largest of 4, 2, 1 that divides R/2, so
// that no access leaves its alignment); interleaved pairs two runs of four.
//
// Angles: a position is a whole number p, and a frequency is kept as a 64-bit
// fraction F of a turn, the nearest one.  p F mod 2^64 is the product's fraction of a
// turn without a rounding, and there is no table; what grows with p is F's own
// rounding alone, at most 2^-65 of a turn for each position.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <string>

#include "../../include/normpre.h"
#include "common.cuh"
#include "heads.h"
#include "internal.h"
#include "tc.cuh"

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

// A sum hi + lo of two fp32 numbers: the exact difference that an addition to hi
// rounds off goes to lo (the two-sum of Knuth and Moller), so that it carries about
// 46 bits.  16384 tokens, 16 / 8 heads of 128 in bf16 take 70.5 us backward (69 with
// one fp32 number), 333 tokens of 32 / 32 heads of 64 12.3 us; with fp64 sums from
// the threads on they took 74.6 and 18.5.
struct Two {
  float hi, lo;
  __device__ __forceinline__ void add(float v) {
    const float s = hi + v, b = s - hi;
    lo += (hi - (s - b)) + (v - b);
    hi = s;
  }
  __device__ __forceinline__ void add(const Two& v) {
    add(v.hi);
    lo += v.lo;
  }
  // what an infinite sum rounds off is NaN
  __device__ __forceinline__ float value() const { return fabsf(hi) < INFINITY ? hi + lo : hi; }
};
__device__ __forceinline__ Two shuffled(const Two& v, int o) {
  return Two{__shfl_xor_sync(0xffffffffu, v.hi, o), __shfl_xor_sync(0xffffffffu, v.lo, o)};
}

struct RotArgs {
  HeadsView x[2], dz[2], out[2];   // queries, keys: inputs, gradients of the results, results
  const void* w[2];                // weights, null: ones
  Two* part;                       // backward: weight gradients by CTA, [ctas][d]
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

// cos and sin of `turns` 2^-64 turns: to the nearest quarter of a turn first, so
// that the rest x, at most 1/4 of a half turn, keeps all of its 24 bits.  Then
// sin(pi x) = x P(x^2) and cos(pi x) = 1 + x^2 Q(x^2), P and Q of third degree
// through the Chebyshev points of [0, 1/16]: within 2.2 and 1.4 units of 2^-24 of
// their values over all x.
__device__ __forceinline__ void circle(uint64_t turns, float& c, float& s) {
  const uint64_t u = turns + (uint64_t(1) << 61);
  const int quarter = static_cast<int>(u >> 62);
  const int64_t rest = static_cast<int64_t>(u & ((uint64_t(1) << 62) - 1)) - (int64_t(1) << 61);
  const float x = static_cast<float>(static_cast<int>(rest >> 30)) * 0x1p-33f, z = x * x;
  float ss = fmaf(z, -0.5890750885009766f, 2.549767017364502f);
  ss = fmaf(z, ss, -5.167707920074463f);
  ss = x * fmaf(z, ss, 3.1415927410125732f);
  float cc = fmaf(z, 0.2321254163980484f, -1.3351378440856934f);
  cc = fmaf(z, cc, 4.05871057510376f);
  cc = fmaf(z, fmaf(z, cc, -4.934802055358887f), 1.f);
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
// The e-th of the lane's values, its pairs' first ones and then their second
// ones: where it lies in the row, -1: nowhere.
template <bool INTER>
__device__ __forceinline__ int place(const Unit& t, int e) {
  const int m = !INTER ? e : e < 4 ? 2 * e : 2 * (e - 4) + 1;
  return m < 4 ? (m < t.na ? t.a + m : -1) : (m - 4 < t.nb ? t.b + m - 4 : -1);
}

template <typename T, int V> struct alignas(V * sizeof(T)) Vec { T v[V]; };

// A lane's 8 values as they lie in memory, read and written V at a time.
template <typename T, int V> struct Raw {
  static constexpr int kWords = 8 * sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  // the V values at p become the i-th ..
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
      const uint32_t v = *reinterpret_cast<const uint16_t*>(p);
      w[at] = i & 1 ? (w[at] & 0xFFFFu) | v << 16 : v;
    }
  }
  // a: the lane's first run.  What lies past a run stays as it is.
  __device__ __forceinline__ void load(const T* a, const Unit& t) {
#pragma unroll
    for (int i = 0; i < 4; i += V) {
      if (i < t.na) get(a + i, i);
      if (i < t.nb) get(a + (t.b - t.a) + i, 4 + i);
    }
  }
  // Pairs of values: 0, 1 the pairs' first ones, 2, 3 their second ones.
  template <bool INTER> __device__ __forceinline__ void unpack(uint64_t (&v)[4]) {
    // the words stay words until here: converted where they are loaded, they
    // would be waited for there
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+r"(w[i]));
    auto at = [&](int m) {
      return sizeof(T) == 4 ? __uint_as_float(w[m]) : m & 1 ? bf16hi(w[m / 2]) : bf16lo(w[m / 2]);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[i] = INTER ? tc::pack2(at(4 * i), at(4 * i + 2)) : tc::pack2(at(2 * i), at(2 * i + 1));
      v[2 + i] = INTER ? tc::pack2(at(4 * i + 1), at(4 * i + 3)) : tc::pack2(at(4 + 2 * i), at(4 + 2 * i + 1));
    }
  }
  template <bool INTER> static __device__ __forceinline__ void store(T* a, const Unit& t, const uint64_t (&v)[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = INTER ? (i < 2 ? 4 * i : 4 * i - 7) : 2 * i;
      tc::unpack2(v[i], f[e], f[e + (INTER ? 2 : 1)]);
    }
#pragma unroll
    for (int i = 0; i < 4; i += V) {
      Vec<T, V> x, y;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x.v[e] = from_f32<T>(f[i + e]);
        y.v[e] = from_f32<T>(f[4 + i + e]);
      }
      if (i < t.na) *reinterpret_cast<Vec<T, V>*>(a + i) = x;
      if (i < t.nb) *reinterpret_cast<Vec<T, V>*>(a + (t.b - t.a) + i) = y;
    }
  }
};

// Sums over the lanes of a row, of several values at once.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int lanes) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < lanes) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
}

__device__ __forceinline__ float dot(const uint64_t (&x)[4], const uint64_t (&y)[4]) {
  uint64_t sum = tc::mul2(x[0], y[0]);
#pragma unroll
  for (int e = 1; e < 4; ++e) sum = tc::fma2(x[e], y[e], sum);
  float lo, hi;
  tc::unpack2(sum, lo, hi);
  return lo + hi;
}
// The same of x with itself, scaled first.
__device__ __forceinline__ float squares(const uint64_t (&x)[4], float f) {
  uint64_t v[4];
  const uint64_t f2 = tc::pack2(f, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = tc::mul2(x[e], f2);
  return dot(v, v);
}
__device__ __forceinline__ void scale(uint64_t (&x)[4], float f) {
  const uint64_t f2 = tc::pack2(f, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = tc::mul2(x[e], f2);
}

// The sums of two heads over the lanes of a row (two or more): the row's upper
// half of lanes ends with the second head's, the lower half with the first's, in
// one shuffle a step instead of two.  (Forward only: backward, where two sums travel,
// it gained nothing, 69.4 us against 68.6 with the sums of then.)
__device__ __forceinline__ float split_sum(float first, float second, int lanes, bool upper) {
  float mine = (upper ? second : first) + __shfl_xor_sync(0xffffffffu, upper ? first : second, lanes >> 1);
#pragma unroll
  for (int o = 8; o; o >>= 1)
    if (o < lanes >> 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  return mine;
}
// A value of each half's head, for all lanes.
__device__ __forceinline__ void join_halves(float mine, int lanes, bool upper, float (&both)[2]) {
  const float other = __shfl_xor_sync(0xffffffffu, mine, lanes >> 1);
  both[0] = upper ? other : mine;
  both[1] = upper ? mine : other;
}

// 1 / sqrt(sum / dim + eps); that sum is a normal number or infinite.
__device__ __forceinline__ float inverse_root(float sum, const RotArgs& g, float eps) {
  const float m = fmaf(sum, g.inv_dim, eps);
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(m));
  // one Newton step: the approximation may be off by two units in the last place
  return m < INFINITY ? fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r) : r;
}
// Rows whose squares leave fp32's range are scaled by a power of two first.
constexpr float kLargeSum = 0x1p126f, kDown = 0x1p-96f;

// CTAs per SM, which the registers are bounded for.
template <typename T, bool BWD> constexpr int per_sm() { return BWD ? 2 : 3; }

// Heads of a unit: fp32 has no registers for two on their way.
template <typename T> constexpr int kUnitHeads = sizeof(T) == 2 ? 2 : 1;

// Backward: a thread's sums over rows of its 8 weight gradients.  Eight units at a
// time are summed in fp32 registers; all beyond, of threads, warps and CTAs too, as
// Two.  So a sum is off by what 16 rows' additions and the terms round, however many
// tokens there are.
struct alignas(16) Sums {
  float4 hi[2][kThreads], lo[2][kThreads];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 2; ++i) hi[i][threadIdx.x] = lo[i][threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // pairs of values; they start again from zero
  __device__ __forceinline__ void take(uint64_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 h = hi[i][threadIdx.x], l = lo[i][threadIdx.x];
      Two t[4] = {{h.x, l.x}, {h.y, l.y}, {h.z, l.z}, {h.w, l.w}};
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        float a, b;
        tc::unpack2(v[2 * i + e / 2], a, b);
        t[e].add(a);
        t[e + 1].add(b);
        v[2 * i + e / 2] = 0;
      }
      hi[i][threadIdx.x] = make_float4(t[0].hi, t[1].hi, t[2].hi, t[3].hi);
      lo[i][threadIdx.x] = make_float4(t[0].lo, t[1].lo, t[2].lo, t[3].lo);
    }
  }
  __device__ __forceinline__ Two get(int e) const {
    return Two{reinterpret_cast<const float*>(&hi[e >> 2][threadIdx.x])[e & 3],
               reinterpret_cast<const float*>(&lo[e >> 2][threadIdx.x])[e & 3]};
  }
};
constexpr int kSumUnits = 8;   // a power of two

template <bool BWD> struct alignas(16) Shared {
  float w[8 * 32];   // the weights by lane
};
template <> struct alignas(16) Shared<true> {
  float w[8 * 32];
  Sums sums;
  Two by_warp[kWarps][8 * 32];
};

// Each warp walks its share of the (token group, heads) units: 32 / lanes tokens
// at once.  The next unit is on its way while one is worked on.  BWD:
// gradients.  side: 0 queries, 1 keys, known to the compiler so that what the
// launch's arguments hold for it needs no registers.
template <typename T, int V, bool INTER, bool BWD, int side>
__device__ __forceinline__ void walk(const RotArgs& g, Shared<BWD>& sh) {
  constexpr int H = kUnitHeads<T>;
  using tc::fma2;
  using tc::mul2;
  const int cta = side ? blockIdx.x - g.ctas : blockIdx.x, ctas = side ? gridDim.x - g.ctas : g.ctas;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int u = lane & (g.lanes - 1), rows = 32 / g.lanes, sub = lane / g.lanes;
  const Unit t = unit_of<INTER>(g, u);
  const int heads = g.heads[side], parts = (heads + H - 1) / H;
  const int64_t units = (g.tokens + rows - 1) / rows * parts;
  const int64_t n_warps = static_cast<int64_t>(ctas) * kWarps, w = static_cast<int64_t>(cta) * kWarps + warp;
  const int64_t begin = units * w / n_warps;
  int left = static_cast<int>(units * (w + 1) / n_warps - begin);
  const bool upper = u >= g.lanes >> 1;
  uint32_t turned = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * u + e < g.half && (INTER || u < g.rot_units)) turned |= 1u << e;
  float* const sw = sh.w;
  if (threadIdx.x < 8 * g.lanes) {
    const int at = place<INTER>(unit_of<INTER>(g, threadIdx.x >> 3), threadIdx.x & 7);
    sw[threadIdx.x] = at < 0 ? 0.f : weight(g, side, at);
  }
  __syncthreads();
  auto weights = [&](int e) { return reinterpret_cast<const uint64_t*>(sw)[4 * u + e]; };
  uint64_t dw[4] = {0, 0, 0, 0};
  if constexpr (BWD) {
    if (g.part) sh.sums.clear();
  }

  // the unit on its way: its place, values and position
  const bool want_x = !BWD || g.norm;
  int token = static_cast<int>(begin / parts) * rows + sub;   // at most 2^30 + 31
  int head = H * static_cast<int>(begin % parts);
  int64_t pos = 0;
  const T *px = nullptr, *pz = nullptr;      // its first head's row, from this lane's first run on
  T* po = nullptr;
  bool live = false, exists = false, all = false;   // its token counts, is a row of the call; all of the warp's count
  Raw<T, V> nx[H], nz[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    nx[i].clear();
    nz[i].clear();
  }
  auto enter = [&]() {
    auto row = [&](const HeadsView& v) { return static_cast<T*>(v.p) + token * v.ts + (head * v.hs + t.a); };
    if (want_x) px = row(g.x[side]);
    if (BWD) pz = row(g.dz[side]);
    po = row(g.out[side]);
    live = token < g.used;
    exists = token < g.tokens;
    all = token - sub + rows <= g.used;
    pos = 0;
    if (turned && live) pos = g.pos64 ? static_cast<const int64_t*>(g.pos)[token] : static_cast<const int*>(g.pos)[token];
  };
  auto fetch = [&]() {
    if (!all || head + H > heads) {
#pragma unroll
      for (int i = 0; i < H; ++i) {
        nx[i].clear();
        nz[i].clear();
      }
    }
#pragma unroll
    for (int i = 0; i < H; ++i)
      if (live && (i == 0 || head + i < heads)) {
        if (want_x) nx[i].load(px + i * g.x[side].hs, t);
        if (BWD) nz[i].load(pz + i * g.dz[side].hs, t);
      }
  };
  // cos, sin of the pairs' angles; forward with the weights: first = x1 k0 + x2 k1, second = x1 k2 + x2 k3
  uint64_t k0[2], k1[2], k2[2], k3[2];
  bool fresh = true;
  if (left) {
    enter();
    fetch();
  }
  while (left) {
    uint64_t x[H][4], y[H][4];
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if (want_x) nx[i].template unpack<INTER>(x[i]);
      if (BWD) nz[i].template unpack<INTER>(y[i]);
    }
    if (fresh) {
      float c[4], s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = 1.f;
        s[e] = 0.f;
        if (turned >> e & 1u) circle(static_cast<uint64_t>(pos) * g.turns[4 * u + e], c[e], s[e]);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint64_t c2 = tc::pack2(c[2 * e], c[2 * e + 1]), s2 = tc::pack2(s[2 * e], s[2 * e + 1]);
        const uint64_t n2 = tc::pack2(-s[2 * e], -s[2 * e + 1]);
        const uint64_t w0 = BWD ? 0 : weights(e), w1 = BWD ? 0 : weights(2 + e);
        k0[e] = BWD ? c2 : mul2(c2, w0);
        k1[e] = BWD ? s2 : mul2(n2, w1);
        k2[e] = BWD ? n2 : mul2(s2, w0);
        k3[e] = BWD ? c2 : mul2(c2, w1);
      }
    }
    T* const to = po;
    const int here = heads - head;             // heads from the unit's first one on
    const bool count = live, write = exists, whole = all;
    head += H;
    fresh = head >= heads;
    if (--left) {
      if (fresh) {
        head = 0;
        token += rows;
        enter();
      } else {
        if (want_x) px += H * g.x[side].hs;
        if (BWD) pz += H * g.dz[side].hs;
        po += H * g.out[side].hs;
      }
      fetch();
    }

    // the pairs turned, or turned back
    auto turn = [&](uint64_t (&v)[4]) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint64_t a = v[e], b = v[2 + e];
        v[e] = fma2(a, k0[e], mul2(b, k1[e]));
        v[2 + e] = fma2(a, k2[e], mul2(b, k3[e]));
      }
    };
    if (!g.norm) {
      // rotation only: what does not turn passes as it is, infinities too
#pragma unroll
      for (int i = 0; i < H; ++i) {
        uint64_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = y[i][e] = BWD ? y[i][e] : x[i][e];
        turn(y[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float was[2], is[2];
          tc::unpack2(v[e], was[0], was[1]);
          tc::unpack2(y[i][e], is[0], is[1]);
          const uint32_t both = turned >> (2 * (e & 1));
          y[i][e] = tc::pack2(both & 1u ? is[0] : was[0], both & 2u ? is[1] : was[1]);
        }
      }
    } else if constexpr (!BWD) {
      // 1 / root mean square of the rows; `down`: by how much they are scaled for it
      float sum[H], down[H], r[H];
      const bool split = H == 2 && g.lanes > 1;
      auto roots = [&](bool scaled) {
#pragma unroll
        for (int i = 0; i < H; ++i) sum[i] = scaled ? squares(x[i], down[i]) : dot(x[i], x[i]);
        if (split) {
          if constexpr (H == 2) {
            const float mine = split_sum(sum[0], sum[1], g.lanes, upper), d = upper ? down[1] : down[0];
            join_halves(inverse_root(mine, g, g.eps * d * d), g.lanes, upper, r);
            return mine < kLargeSum;
          }
        }
        row_sums(sum, g.lanes);
        bool fits = true;
#pragma unroll
        for (int i = 0; i < H; ++i) {
          r[i] = inverse_root(sum[i], g, g.eps * down[i] * down[i]);
          fits = fits && sum[i] < kLargeSum;
        }
        return fits;
      };
#pragma unroll
      for (int i = 0; i < H; ++i) down[i] = 1.f;
      if (__any_sync(0xffffffffu, !roots(false))) {
        // once more, the large rows scaled (small values of theirs only after their
        // root has raised them); the others come out as they were
        if (split) row_sums(sum, g.lanes);
#pragma unroll
        for (int i = 0; i < H; ++i) down[i] = sum[i] < 0.5f * kLargeSum ? 1.f : kDown;
        roots(true);
#pragma unroll
        for (int i = 0; i < H; ++i) {
          scale(x[i], r[i]);
          r[i] = down[i];
        }
      }
#pragma unroll
      for (int i = 0; i < H; ++i) {
        scale(x[i], r[i]);
        turn(x[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[i][e] = x[i][e];
      }
    } else {
      float sum[2 * H], r[H], m[H];
      bool fits = true;
      // the weights are fetched each time: held, they take registers that the next
      // unit's values need
      uint64_t wt[4];
      const uint32_t wa = tc::su32(sw + 8 * u);
      asm volatile("ld.shared.v2.b64 {%0, %1}, [%4];\n\tld.shared.v2.b64 {%2, %3}, [%4 + 16];"
                   : "=l"(wt[0]), "=l"(wt[1]), "=l"(wt[2]), "=l"(wt[3]) : "r"(wa));
      auto slope = [&](int i) {                 // <u, x>
        uint64_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(y[i][e], wt[e]);
        return dot(v, x[i]);
      };
#pragma unroll
      for (int i = 0; i < H; ++i) {
        turn(y[i]);
        sum[i] = dot(x[i], x[i]);
        sum[H + i] = slope(i);
      }
      row_sums(sum, g.lanes);
#pragma unroll
      for (int i = 0; i < H; ++i) fits = fits && sum[i] < kLargeSum && fabsf(sum[H + i]) < INFINITY;
      if (__any_sync(0xffffffffu, !fits)) {
        // <u, x> may be out of range with x: from xh instead; rows that are in range
        // come out as they would have
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const float down = sum[i] < kLargeSum ? 1.f : kDown;
          const bool in = sum[i] < kLargeSum && fabsf(sum[H + i]) < INFINITY;
          float again[1] = {squares(x[i], down)};
          row_sums(again, g.lanes);
          r[i] = inverse_root(again[0], g, g.eps * down * down);
          scale(x[i], r[i]);
          scale(x[i], down);
          again[0] = slope(i);
          row_sums(again, g.lanes);
          m[i] = in ? sum[H + i] * g.inv_dim * r[i] : again[0] * g.inv_dim;
          r[i] *= down;
        }
      } else {
#pragma unroll
        for (int i = 0; i < H; ++i) {
          r[i] = inverse_root(sum[i], g, g.eps);
          m[i] = sum[H + i] * g.inv_dim * r[i];
          scale(x[i], r[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const uint64_t m2 = tc::pack2(-m[i], -m[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dw[e] = fma2(y[i][e], x[i][e], dw[e]);
          y[i][e] = fma2(x[i][e], m2, mul2(y[i][e], wt[e]));
        }
        scale(y[i], r[i]);
      }
    }
    if (!whole && !count) {
#pragma unroll
      for (int i = 0; i < H; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[i][e] = 0;
    }
    if (write) {
#pragma unroll
      for (int i = 0; i < H; ++i)
        if (i == 0 || i < here) Raw<T, V>::template store<INTER>(to + i * g.out[side].hs, t, y[i]);
    }
    if constexpr (BWD) {
      if (g.part && left % kSumUnits == 0) sh.sums.take(dw);
    }
  }
  if constexpr (BWD) {
    // the CTA's weight gradients: over the rows of a warp, then over the warps
    if (!g.part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      Two v = sh.sums.get(e);
      for (int o = g.lanes; o < 32; o <<= 1) v.add(shuffled(v, o));
      if (sub == 0) sh.by_warp[warp][8 * u + e] = v;
    }
    __syncthreads();
    if (threadIdx.x < 8 * g.lanes) {
      const int to = place<INTER>(unit_of<INTER>(g, threadIdx.x >> 3), threadIdx.x & 7);
      Two sum = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWarps; ++i) sum.add(sh.by_warp[i][threadIdx.x]);
      if (to >= 0) g.part[static_cast<int64_t>(blockIdx.x) * g.dim + to] = sum;
    }
  }
}

template <typename T, int V, bool INTER, bool BWD>
__global__ void __launch_bounds__(kThreads, per_sm<T, BWD>()) k_qkrot(const __grid_constant__ RotArgs g) {
  __shared__ Shared<BWD> sh;
  if (blockIdx.x < g.ctas) walk<T, V, INTER, BWD, 0>(g, sh);
  else walk<T, V, INTER, BWD, 1>(g, sh);
}

// Sums the CTAs' weight gradients in a fixed order: 32 columns of one weight.
__global__ void __launch_bounds__(1024) k_qkrot_fold(const Two* part, int q_ctas, int ctas, int dim, void* dqw, void* dkw,
                                                     int w_bf16) {
  __shared__ Two sm[32][33];
  const int side = blockIdx.y, col = 32 * blockIdx.x + threadIdx.x;
  const int first = side ? q_ctas : 0, last = side ? ctas : q_ctas;
  Two sum = {0.f, 0.f};
  if (col < dim)
    for (int i = first + threadIdx.y; i < last; i += 32) sum.add(part[static_cast<int64_t>(i) * dim + col]);
  sm[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  sum = sm[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o; o >>= 1) sum.add(shuffled(sum, o));
  void* out = side ? dkw : dqw;
  const int to = 32 * blockIdx.x + threadIdx.y;
  if (threadIdx.x == 0 && to < dim && out) {
    if (w_bf16) static_cast<bf16*>(out)[to] = from_f32<bf16>(sum.value());
    else static_cast<float*>(out)[to] = sum.value();
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
unsigned share(RotArgs* g, int per_sm, int unit) {
  const int64_t groups = cdiv(g->tokens, 32 / g->lanes);
  const int64_t most = std::min<int64_t>(kMaxCtas, static_cast<int64_t>(device_sm_count()) * per_sm);
  const int64_t parts[2] = {cdiv(g->heads[0], unit), cdiv(g->heads[1], unit)};
  const int64_t q = std::max<int64_t>(1, most * parts[0] / (parts[0] + parts[1])), k = std::max<int64_t>(1, most - q);
  g->ctas = static_cast<int>(std::min(q, cdiv(groups * parts[0], kWarps)));
  return static_cast<unsigned>(g->ctas + std::min(k, cdiv(groups * parts[1], kWarps)));
}

// Returns the number of CTAs.
template <typename T, bool BWD>
unsigned launch(RotArgs* g, int v, bool inter, cudaStream_t s) {
  const unsigned ctas = share(g, per_sm<T, BWD>(), kUnitHeads<T>);
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
  if (tokens < 0 || tokens > (int64_t(1) << 30)) return fail(NORMPRE_ERR_SHAPE, "tokens must be in [0, 2^30]");
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

// A frequency in radians as a fraction of a turn, in units of 2^-64: |f| / (2 pi) in
// two parts, high + low, with 1 / (2 pi) in two parts as well (106 bits), so that the
// whole turns of a large frequency cost nothing.
uint64_t turns_of(double f) {
  constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
  const double a = std::fabs(f), high = a * kHigh, low = std::fma(a, kHigh, -high) + a * kLow;
  const double part = std::ldexp(high - std::floor(high), 64), whole = std::floor(part);   // exact
  const uint64_t t = static_cast<uint64_t>(whole) + static_cast<uint64_t>(std::llround(part - whole + std::ldexp(low, 64)));
  return f < 0 ? 0 - t : t;
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
    p->turns[i] = turns_of(frequencies[i]);
  }
  *out = p.release();
  return NORMPRE_OK;
}

int normpre_qkrot_bytes(const normpre_qkrot* p, int64_t* bytes) {
  if (!p || !bytes) return fail(NORMPRE_ERR_ARG, "null argument");
  *bytes = static_cast<int64_t>(kMaxCtas) * p->cfg.head_dim * static_cast<int64_t>(sizeof(Two));
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
    g.part = weights ? static_cast<Two*>(workspace) : nullptr;
    ctas = c.dtype == NORMPRE_BF16 ? launch<bf16, true>(&g, width(p->half), c.interleaved, s)
                                   : launch<float, true>(&g, width(p->half), c.interleaved, s);
  }
  if (weights)
    k_qkrot_fold<<<dim3(static_cast<unsigned>(cdiv(c.head_dim, 32)), 2), dim3(32, 32), 0, s>>>(
        static_cast<const Two*>(workspace), g.ctas, static_cast<int>(ctas), c.head_dim, dq_weight, dk_weight,
        weight_dtype == NORMPRE_BF16);
  return done(cudaGetLastError(), "query and key norms, backward");
}

void normpre_qkrot_free(normpre_qkrot* p) { delete p; }

}  // extern "C"
