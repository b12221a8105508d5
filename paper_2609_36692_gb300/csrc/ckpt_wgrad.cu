// Weight gradient of a linear layer from its input's 8-bit checkpoint:
// dW = dY^T xhat, summed over the tokens.
//
// k_wgrad_tc: bf16 dY on tcgen05.  xhat is exact in bf16 and so is dY, so that
// one kind::f16 product with fp32 accumulation computes the sums.  A tile of
// 128 features x 256 outputs (the transposed piece of dW: a TMEM lane is a
// feature, so that a warp stores 32 consecutive elements of a row of dW) is
// summed 64 tokens at a time: TMA brings the codes and the dY boxes into a
// ring, sixteen warps turn codes into swizzled bf16 tiles (a byte becomes an
// fp32 by permutation into 2^23 + byte, a packed addition takes off the offset,
// a packed product scales, a permutation packs two), one thread issues the MMAs,
// and four warps drain a finished accumulator (two in TMEM) while the next tile runs.
// Both operands are read along their rows (MN-major), as they lie in memory:
// nothing is transposed.  The 128 side is the converted one: half the bytes to
// convert of the 256 side.
//   A pair of CTAs takes two neighbouring feature tiles of the same outputs as
// one product of 256 features: each converts its own 128 features and loads the
// dY of 128 outputs, and a thread of the even CTA issues the MMAs that read both.
//   What bounds it: shared memory, whose 128 bytes a cycle pass 80 KB a step (24
// KB in, 24 KB through the conversion, 32 KB of MMA operands: 625 cycles against
// the MMAs' 512).  From L2 an SM takes in 24 KB, 375 cycles of its port's 64 bytes
// a cycle (40 KB, 660 cycles, when each CTA works for itself; a multicast saves
// L2 reads but not the port).  256 x 192 tiles of one
// CTA take in fewer bytes too, but their conversion (4 cycles an element and SM
// sub-partition, byte permutations at half rate) then takes 1000 cycles of the
// MMAs' 768.  16384 x 6144 x 2048: 0.251 ms (1640 TFLOP/s), 0.28 ms in a long
// loop, where the clock falls with the power limit.
//   With too few tiles for the SMs, clusters of 2 to 8 CTAs split a tile's
// tokens instead and join through distributed shared memory: each CTA lays its
// accumulator out in its (then idle) ring and sums one slice of the outputs
// over the ranks in rank order.  8192 x 768 x 768: 0.022 ms, of which the join
// takes 0.005 (112 KB a CTA from its neighbours, pulled or pushed alike).
//
// k_wgrad_simt: fp32 arithmetic, one CTA of 256 threads per 64 x 64 piece of
// dW, 16 tokens at a time through shared memory, a 4 x 4 piece per thread; any
// dtype, stride and size.  Loads and products take turns, and a CTA walks all
// tokens: 8192 x 768 x 768 with fp32 dY 0.73 ms (13 TFLOP/s, 144 CTAs), 16384 x
// 6144 x 2048 16.7 ms (25).
#include <algorithm>

#include "ckpt.h"
#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

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

constexpr int kTileK = 128, kTileN = 256, kStep = 64;   // features, outputs (at most), tokens of a step
// dY and the codes have rings of their own: codes are given back as soon as
// they are converted, so that conversion runs ahead and only dY's load latency
// stands between the rings and the tensor cores.
constexpr int kRing = 4;
constexpr int kBox = 64 * 128;                           // bytes of 64 rows of 64 bf16
constexpr int kCodeBytes = kStep * kTileK, kXBytes = 2 * kBox;
constexpr int kDyRingBytes = 16 * kBox;                  // 4 places of 4 boxes, or 8 of a pair's 2
constexpr int kConvert = 4, kGroups = 4;                 // converting warps of a step; groups that take turns
constexpr int kTma = 4 + kGroups * kConvert, kMma = kTma + 1, kCodes = kTma + 2;   // warps: drain, convert, these
constexpr int kTcThreads = 32 * (kCodes + 1);
constexpr size_t kTcSmem = kDyRingBytes + kRing * (kXBytes + kCodeBytes) + 512;

struct WgradTcArgs {
  WgradArgs a;
  CUtensorMap dy, codes;
  int tiles_k, tiles_n, units;   // units: tiles, or pairs of feature tiles
  int tile_n;                    // outputs of a tile
};

struct WgradBars {
  // of dY, the codes, the converted tiles (of this CTA, and both operands of the
  // pair's other), the accumulators
  uint64_t full[8], empty[8], cfull[kRing], cempty[kRing], xfull[kRing], xempty[kRing], ofull[kRing];
  uint64_t tfull[2], tempty[2], drain;
  uint32_t tmem;
  int abort;
  uint32_t issued[8], cissued[kRing];   // last parity + 1 of full and cfull
};

// A float of another CTA's shared memory in the cluster.
__device__ __forceinline__ float4 remote_float4(uint32_t addr, uint32_t rank) {
  uint32_t r;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(r) : "memory");
  return v;
}

// Four codes -> two bf16 pairs, code * step.  The offset comes off before the
// product, exactly: a multiple of a large step by 2^23 is beyond fp32.
__device__ __forceinline__ void convert4(uint32_t w, uint64_t step2, uint32_t& p0, uint32_t& p1) {
  w ^= 0x80808080u;   // code + 128
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 + i));   // 2^23 + code + 128
  const uint64_t off2 = tc::pack2(-8388736.f, -8388736.f);                                       // -(2^23 + 128)
  float lo, hi;
  // the values are bf16 numbers: their upper halves are all of them
  tc::unpack2(tc::mul2(tc::add2(tc::pack2(f[0], f[1]), off2), step2), lo, hi);
  p0 = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
  tc::unpack2(tc::mul2(tc::add2(tc::pack2(f[2], f[3]), off2), step2), lo, hi);
  p1 = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}

// SPLIT: the cluster's CTAs share a tile and split its tokens; otherwise a pair
// of CTAs takes two feature tiles, each with half of dY's columns, and one thread
// of the even CTA issues the MMAs of both.
template <typename TW, bool SPLIT>
__global__ void __launch_bounds__(kTcThreads, 1) k_wgrad_tc(const __grid_constant__ WgradTcArgs f) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr int kDyRing = SPLIT ? 4 : 8, kDyBytes = kDyRingBytes / kDyRing;
  uint8_t* ring = smem;                                   // [kDyRing] dY boxes
  uint8_t* xbuf = ring + kDyRingBytes;                    // [kRing] the codes as bf16
  uint8_t* codes = xbuf + kRing * kXBytes;                // [kRing]
  WgradBars* b = reinterpret_cast<WgradBars*>(codes + kRing * kCodeBytes);
  static_assert(sizeof(WgradBars) <= 512, "barriers");
  const WgradArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  uint32_t csize;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(csize));
  const int unit0 = blockIdx.x / csize, nunits = gridDim.x / csize;
  const int total = static_cast<int>((a.tokens + kStep - 1) / kStep);
  const int s0 = SPLIT ? static_cast<int>(static_cast<int64_t>(total) * rank / csize) : 0;
  const int s1 = SPLIT ? static_cast<int>(static_cast<int64_t>(total) * (rank + 1) / csize) : total;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kDyRing; ++i) {
      tc::mbar_init(&b->full[i], 1);
      tc::mbar_init(&b->empty[i], 1);
      b->issued[i] = 0;
    }
    for (int i = 0; i < kRing; ++i) {
      tc::mbar_init(&b->ofull[i], 1);
      tc::mbar_init(&b->cfull[i], 1);
      tc::mbar_init(&b->cempty[i], kConvert);
      tc::mbar_init(&b->xfull[i], kConvert);
      tc::mbar_init(&b->xempty[i], 1);
      b->cissued[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&b->tfull[i], 1);
      tc::mbar_init(&b->tempty[i], SPLIT ? 4 : 8);
    }
    tc::mbar_init(&b->drain, 1);
    b->abort = 0;
    tc::fence_barrier_init();
    tc::prefetch_map(&f.dy);
    tc::prefetch_map(&f.codes);
  }
  __syncthreads();
  tc::cluster_sync();   // the peer's barriers exist before an arrival reaches them
  if (warp == kMma) {
    if (SPLIT) {
      tc::tmem_alloc(&b->tmem, 512);
      tc::tmem_relinquish();
    } else {
      tc::tmem_alloc_pair(&b->tmem, 512);
      tc::tmem_relinquish_pair();
    }
    tc::fence_before();
  }
  __syncthreads();
  if (!SPLIT) tc::cluster_sync();   // both have their accumulators
  tc::fence_after();
  const uint32_t tmem = b->tmem;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, &b->abort));
    return ok;
  };
  auto wait1 = [&](uint64_t* bar, uint32_t parity) { return ok = ok && tc::mbar_wait(bar, parity, &b->abort); };
  // feature tile and first output of a unit
  auto tile_k = [&](int u) { return SPLIT ? u % f.tiles_k : 2 * (u % ((f.tiles_k + 1) / 2)) + static_cast<int>(rank); };
  auto first_n = [&](int u) { return (SPLIT ? u / f.tiles_k : u / ((f.tiles_k + 1) / 2)) * f.tile_n; };
  struct Place {         // in a ring of N, and the parity of its uses
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int n) {
      if (++at == n) { at = 0; phase ^= 1u; }
    }
  };
  Place y, x;            // of dY's ring and the others

  if (warp == kTma) {
    // ---------------- dY by TMA (one thread) ----------------
    if (tc::elect_one()) {
      for (int u = unit0; u < f.units && ok; u += nunits) {
        const int n0 = first_n(u) + (SPLIT ? 0 : static_cast<int>(rank) * f.tile_n / 2);
        for (int s = s0; s < s1; ++s, y.next(kDyRing)) {
          if (!wait1(&b->empty[y.at], y.phase ^ 1u)) break;
          uint8_t* dst = ring + y.at * kDyBytes;
          tc::mbar_expect_tx(&b->full[y.at], kDyBytes);
          b->issued[y.at] = y.phase + 1;
          for (int i = 0; i < kDyBytes / kBox; ++i)
            tc::tma_load_3d(dst + i * kBox, &f.dy, &b->full[y.at], n0 + 64 * i, s * kStep, 0);
        }
      }
    }
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok);
  } else if (warp == kCodes) {
    // ---------------- codes by TMA (one thread) ----------------
    if (tc::elect_one()) {
      for (int u = unit0; u < f.units && ok; u += nunits) {
        const int k0 = tile_k(u) * kTileK;
        for (int s = s0; s < s1; ++s, x.next(kRing)) {
          if (!wait1(&b->cempty[x.at], x.phase ^ 1u)) break;
          tc::mbar_expect_tx(&b->cfull[x.at], kCodeBytes);
          b->cissued[x.at] = x.phase + 1;
          tc::tma_load_3d(codes + x.at * kCodeBytes, &f.codes, &b->cfull[x.at], k0, s * kStep, 0);
        }
      }
    }
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok);
  } else if (warp == kMma) {
    // ---------------- MMA (one thread) ----------------
    if (!SPLIT && rank != 0) {
      // The pair's other CTA: its operands are in place.  The converting warps
      // handed their writes to the asynchronous proxy and to this thread; its
      // arrival releases them to the thread that issues the MMAs.
      if (tc::elect_one()) {
        for (int u = unit0; u < f.units && ok; u += nunits)
          for (int s = s0; s < s1; ++s, y.next(kDyRing), x.next(kRing)) {
            if (!wait1(&b->full[y.at], y.phase) || !wait1(&b->xfull[x.at], x.phase)) break;
            tc::mbar_arrive_remote(&b->ofull[x.at], 0);
          }
        // the issuing thread's last arrival: none is under way after it
        int never = 0;
        tc::mbar_wait(&b->drain, 0, &never);
      }
    } else if (tc::elect_one()) {
      const uint32_t idesc = tc::idesc_bf16(SPLIT ? kTileK : 2 * kTileK, f.tile_n, 1, 1);
      auto commit = [&](uint64_t* bar) {   // in both CTAs of a pair
        if (SPLIT) tc::mma_commit(bar);
        else tc::mma_commit_pair(bar, 3);
      };
      // arrivals of both CTAs
      auto wait_pair = [&](uint64_t* bar, uint32_t parity) { return ok = ok && tc::mbar_wait<!SPLIT>(bar, parity, &b->abort); };
      int acc = 0, never = 0;
      uint32_t tphase = 0;
      for (int u = unit0; u < f.units && ok; u += nunits) {
        if (!wait_pair(&b->tempty[acc], tphase ^ 1u)) break;
        for (int s = s0; s < s1; ++s, y.next(kDyRing), x.next(kRing)) {
          if (!wait1(&b->full[y.at], y.phase) || !wait1(&b->xfull[x.at], x.phase)) break;
          if (!SPLIT && !wait_pair(&b->ofull[x.at], x.phase)) break;
          tc::fence_after();
          const uint64_t bd = tc::sdesc(tc::su32(ring + y.at * kDyBytes), kBox, 1024);
          const uint64_t ad = tc::sdesc(tc::su32(xbuf + x.at * kXBytes), kBox, 1024);
#pragma unroll
          for (int kk = 0; kk < kStep / 16; ++kk) {
            const uint32_t d = tmem + 256 * acc, add = s != s0 || kk != 0;
            if (SPLIT) tc::mma_bf16(d, ad + kk * (2048 >> 4), bd + kk * (2048 >> 4), idesc, add);
            else tc::mma_bf16_pair(d, ad + kk * (2048 >> 4), bd + kk * (2048 >> 4), idesc, add);
          }
          commit(&b->empty[y.at]);
          commit(&b->xempty[x.at]);
        }
        if (!ok) break;
        commit(&b->tfull[acc]);
        acc ^= 1;
        if (acc == 0) tphase ^= 1u;
      }
      // every MMA issued has completed once `drain` fires
      commit(&b->drain);
      tc::mbar_wait(&b->drain, 0, &never);
    }
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok);
  } else if (warp >= 4) {
    // ---------------- codes -> bf16 ----------------
    // The groups take the steps in turn: a group's waits, which outweigh its
    // work, then have other steps' time.  A group always works in the same
    // place of the rings, where it waits for its own last step, never two uses
    // ahead (a barrier's parity would lie there).  8 rows x 4 blocks per warp at
    // a time: lanes of 8 rows, whose 16-byte pieces the swizzle spreads over all
    // banks.
    static_assert(kGroups == kRing, "a group's place in the rings");
    constexpr int kPer = kStep / (8 * kConvert);   // rows of a lane
    const int group = (warp - 4) / kConvert;
    const int row = 8 * ((warp - 4) % kConvert) + (lane & 7), blk = lane >> 3, sw = row & 7;
    const uint8_t* src = codes + group * kCodeBytes + row * kTileK;
    uint8_t* dst = xbuf + group * kXBytes + (blk >> 1) * kBox + row * 128;
    // The rows' step words come from global memory, a group's turn ahead.
    uint32_t word[kPer], ahead[kPer];
    const uint32_t* words = nullptr;       // of the unit's panel, if it has one
    int s = s0 + group, u = unit0;         // the group's next step
    uint32_t parity = 0;
    auto enter = [&]() {
      const int tk = tile_k(u);
      words = u < f.units && tk < f.tiles_k ? a.x.steps + static_cast<int64_t>(tk) * a.tokens : nullptr;
    };
    auto settle = [&]() {                  // in this unit, or that far into one after it
      while (s >= s1 && u < f.units) {
        s -= s1 - s0;
        u += nunits;
        enter();
      }
    };
    auto fetch = [&]() {
#pragma unroll
      for (int r = 0; r < kPer; ++r) {
        const int64_t t = static_cast<int64_t>(s) * kStep + row + 8 * kConvert * r;
        ahead[r] = words && t < a.tokens ? __ldg(words + t) : 0u;
      }
    };
    if (s0 >= s1) u = f.units;
    if (u < f.units) {
      enter();
      settle();
      fetch();
    }
    for (; u < f.units; parity ^= 1u) {
#pragma unroll
      for (int r = 0; r < kPer; ++r) word[r] = ahead[r];
      s += kGroups;
      settle();
      fetch();
      if (!wait(&b->cfull[group], parity)) break;
      uint4 c[kPer][2];
#pragma unroll
      for (int r = 0; r < kPer; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          c[r][i] = *reinterpret_cast<const uint4*>(src + 8 * kConvert * kTileK * r + (((2 * blk + i) ^ sw) << 4));
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&b->cempty[group]);
      if (!wait(&b->xempty[group], parity ^ 1u)) break;
#pragma unroll
      for (int r = 0; r < kPer; ++r) {
        const float step = ckpt_step(word[r], blk);
        const uint64_t step2 = tc::pack2(step, step);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t w[4] = {c[r][i].x, c[r][i].y, c[r][i].z, c[r][i].w};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 v;
            convert4(w[2 * h], step2, v.x, v.y);
            convert4(w[2 * h + 1], step2, v.z, v.w);
            *reinterpret_cast<uint4*>(dst + 8 * kConvert * 128 * r + (((4 * (blk & 1) + 2 * i + h) ^ sw) << 4)) = v;
          }
        }
      }
      tc::fence_smem_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&b->xfull[group]);
    }
  } else if (!SPLIT) {
    // ---------------- drain: warp's 32 features x a tile's outputs ----------------
    int acc = 0;
    uint32_t tphase = 0;
    for (int u = unit0; u < f.units && ok; u += nunits) {
      if (!wait(&b->tfull[acc], tphase)) break;
      tc::fence_after();
      const int k = tile_k(u) * kTileK + 32 * warp + lane, n0 = first_n(u), n1 = min(f.tile_n, a.n - n0);
      TW* dw = static_cast<TW*>(a.dw) + static_cast<int64_t>(n0) * a.dw_ld + k;
#pragma unroll 1
      for (int c = 0; c < n1; c += 32) {
        uint32_t r[32];
        tc::tmem_ld32(tmem + 256 * acc + c + (static_cast<uint32_t>(32 * warp) << 16), r);
        tc::tmem_ld_wait();
        if (k < a.k) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (c + e < n1) {
              TW* p = dw + (c + e) * a.dw_ld;
              const float v = __uint_as_float(r[e]);
              *p = from_f32<TW>(a.accumulate ? to_f32(*p) + v : v);
            }
        }
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive_remote(&b->tempty[acc], 0);   // where the MMAs are issued
      acc ^= 1;
      if (acc == 0) tphase ^= 1u;
    }
  }
  if (SPLIT) {
    // one unit per cluster; each CTA's partial tile goes to its ring as
    // [outputs][features], free once the accumulator is complete
    float* part = reinterpret_cast<float*>(ring);
    if (warp >= 4 && warp < 4 + kGroups * kConvert) {   // idle by now: 4 warps a lane quarter, 64 outputs each
      const int q = warp & 3, c0 = 64 * ((warp - 4) >> 2);
      if (s1 > s0 && wait(&b->tfull[0], 0)) {
        tc::fence_after();
#pragma unroll 1
        for (int c = c0; c < c0 + 64; c += 32) {
          uint32_t r[32];
          tc::tmem_ld32(tmem + c + (static_cast<uint32_t>(32 * q) << 16), r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) part[(c + e) * kTileK + 32 * q + lane] = __uint_as_float(r[e]);
        }
      }
    }
    __syncthreads();
    tc::cluster_sync();
    const int k0 = tile_k(unit0) * kTileK, n0 = first_n(unit0), rows = (kTileN + csize - 1) / csize;
    for (int i = threadIdx.x; i < rows * (kTileK / 4); i += kTcThreads) {
      const int n = rank * rows + i / (kTileK / 4), k = 4 * (i % (kTileK / 4));
      if (n >= kTileN || n0 + n >= a.n || k0 + k >= a.k) continue;
      // all ranks' pieces are fetched before any is added
      float4 piece[8];
#pragma unroll
      for (uint32_t q = 0; q < 8; ++q) {
        piece[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (q < csize && static_cast<int64_t>(total) * q / csize != static_cast<int64_t>(total) * (q + 1) / csize)
          piece[q] = remote_float4(tc::su32(part + n * kTileK + k), q);
      }
      float v[4] = {};
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        v[0] += piece[q].x; v[1] += piece[q].y; v[2] += piece[q].z; v[3] += piece[q].w;
      }
      TW* p = static_cast<TW*>(a.dw) + static_cast<int64_t>(n0 + n) * a.dw_ld + k0 + k;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k0 + k + e < a.k) p[e] = from_f32<TW>(a.accumulate ? to_f32(p[e]) + v[e] : v[e]);
    }
  }
  if (!ok && lane == 0) {
    *static_cast<volatile int*>(&b->abort) = 1;
    raise_host_flag(a.flags, kFlagTimeout);
  }
  __syncthreads();
  if (threadIdx.x == 0 && *static_cast<volatile int*>(&b->abort)) {
    // let every TMA copy still in flight land before the CTA exits
    volatile int never = 0;
    for (int i = 0; i < kDyRing; ++i)
      if (b->issued[i]) tc::mbar_wait(&b->full[i], b->issued[i] - 1, &never);
    for (int i = 0; i < kRing; ++i)
      if (b->cissued[i]) tc::mbar_wait(&b->cfull[i], b->cissued[i] - 1, &never);
  }
  __syncthreads();
  // no CTA exits while the other may still arrive on its barriers, work on its
  // operands or read its partial tile
  tc::cluster_sync();
  if (warp == kMma) {
    tc::fence_after();
    if (SPLIT) tc::tmem_dealloc(tmem, 512);
    else tc::tmem_dealloc_pair(tmem, 512);
  }
}

struct ClusterLaunch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  ClusterLaunch(int cluster, int clusters, cudaStream_t s) {
    cfg.gridDim = dim3(cluster * clusters);
    cfg.blockDim = dim3(kTcThreads);
    cfg.dynamicSmemBytes = kTcSmem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
};

// Clusters of a size that the current device holds at once (a cluster stays
// within a GPC, so that some SMs are left over).  The kernel is allowed its
// shared memory there first; a launch of it follows such a question.
template <typename TW, bool SPLIT>
cudaError_t clusters_at_once(int cluster, int* fit) {
  static PerDevice known[9];
  return known[cluster].get(fit, [cluster](int* n) {
    ClusterLaunch l(cluster, std::max(1, device_sm_count() / cluster), nullptr);
    cudaError_t e = allow_smem<k_wgrad_tc<TW, SPLIT>>(kTcSmem);
    if (!e) e = cudaOccupancyMaxActiveClusters(n, k_wgrad_tc<TW, SPLIT>, &l.cfg);
    if (!e) *n = std::max(1, *n);
    return e;
  });
}

template <typename TW>
cudaError_t launch_tc(WgradTcArgs f, cudaStream_t s) {
  f.tiles_k = static_cast<int>(cdiv(f.a.k, kTileK));
  f.tile_n = kTileN;
  f.tiles_n = static_cast<int>(cdiv(f.a.n, kTileN));
  const int64_t tiles = static_cast<int64_t>(f.tiles_k) * f.tiles_n, steps = cdiv(f.a.tokens, kStep);
  // The largest split of the tokens whose clusters all run at once, each CTA
  // with at least two steps: twice the CTAs halve the time until the join
  // (about four steps) weighs in.
  int split = tiles == 1 ? 1 : 0, fit = 0;
  for (int c = 2; c <= 8 && steps >= 2 * c && tiles * c <= device_sm_count(); ++c) {
    const cudaError_t e = clusters_at_once<TW, true>(c, &fit);
    if (e) return e;
    if (tiles <= fit) split = c;
  }
  if (split) {
    f.units = static_cast<int>(tiles);
    const cudaError_t e = clusters_at_once<TW, true>(split, &fit);
    if (e) return e;
    ClusterLaunch l(split, f.units, s);
    return cudaLaunchKernelEx(&l.cfg, k_wgrad_tc<TW, true>, f);
  }
  const cudaError_t e = clusters_at_once<TW, false>(2, &fit);
  if (e) return e;
  // The tile width whose rounds over the clusters take least.  A step's time goes
  // as 512 + tn / 2, so that a narrower tile gains little (16384 x 4096 x 2432,
  // three rounds each: 252 us at 256, 248 at 224, 238 at 192) and a further round
  // costs all of it (16384 x 6912 x 2048: 266 us at 256, 327 at 224).
  int64_t least = -1;
  for (int tn = kTileN; tn >= 192; tn -= 32) {
    const int64_t units = (f.tiles_k + 1) / 2 * cdiv(f.a.n, tn), cost = cdiv(units, fit) * (512 + tn / 2);
    if (least >= 0 && cost >= least) continue;
    least = cost;
    f.tile_n = tn;
    f.units = static_cast<int>(units);
  }
  ClusterLaunch l(2, std::min(f.units, fit), s);
  return cudaLaunchKernelEx(&l.cfg, k_wgrad_tc<TW, false>, f);
}

}  // namespace

cudaError_t launch_ckpt_wgrad_tc(const WgradArgs& a, int dw_dtype, cudaStream_t s, std::string* err) {
  WgradTcArgs f;
  f.a = a;
  const uint64_t t = static_cast<uint64_t>(a.tokens);
  const uint64_t dy_dims[3] = {static_cast<uint64_t>(a.n), t, 1};
  const uint64_t dy_strides[2] = {static_cast<uint64_t>(a.dy_ld) * 2, static_cast<uint64_t>(a.dy_ld) * 2};
  const uint32_t dy_box[3] = {64, kStep, 1};
  const uint64_t c_dims[3] = {static_cast<uint64_t>(a.x_ld), t, 1};
  const uint64_t c_strides[2] = {static_cast<uint64_t>(a.x_ld), static_cast<uint64_t>(a.x_ld)};
  const uint32_t c_box[3] = {kTileK, kStep, 1};
  if (!driver_encode_tiled(&f.dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.dy), dy_dims, dy_strides,
                           dy_box, err) ||
      !driver_encode_tiled(&f.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<int8_t*>(a.x.codes), c_dims,
                           c_strides, c_box, err))
    return cudaErrorInvalidValue;
  return dw_dtype == 0 ? launch_tc<float>(f, s) : launch_tc<bf16>(f, s);
}

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
