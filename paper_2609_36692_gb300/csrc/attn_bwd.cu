// Packed causal attention, backward, bf16 on tcgen05 tensor cores.
//
//   P = exp2(c S - log2(e) lse),  dS = P (dP - delta),  S = Q K^T, dP = dO V^T,
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
//
// Two kernels: k_attn_dkdv owns 128 keys and walks the queries that see them
// (over the heads of the group and the later blocks), k_attn_dq owns 128
// queries and walks their keys.  Every gradient is then summed by one CTA in
// one accumulator in a fixed order, without atomics or fp32 partials in global
// memory; the price is that S and dP are formed twice, 7 products of a tile
// instead of 5.
//
// Both: one CTA per SM walks the work list; the owned tiles stay in shared
// memory, the others pass through a ring filled by a TMA warp; one thread
// issues the MMAs; eight softmax warps each take 32 rows x 64 columns of a
// score tile, one thread per row.  P and dS go back to TMEM as bf16 over the
// scores they came from (each warp group inside its own half of the columns)
// and are the A operands of the products that follow.
//
// k_attn_dkdv forms the transposed tiles S^T, dP^T (rows: keys), so that P^T
// and dS^T lie in TMEM as the A operands of dV and dK.  TMEM at head_dim 128:
// S^T 128, dP^T 128, dV 128, dK 128 columns.  The order dV(i), S(i+1), dK(i),
// dP(i+1) keeps the tensor cores on two products while the softmax warps form
// dS(i) and then P(i+1).
// k_attn_dq: S in two buffers, dP, dQ; dS lies over S, so that dP(j+1) starts
// as soon as dP(j) has been read.
//
// Roundings to bf16: P and dS once each (MMA operands), the gradients once.
#include <algorithm>

#include "attn_tc.cuh"

namespace normpre {
namespace {

constexpr int kThreads = 384;   // softmax 8 warps, TMA, MMA, statistics, padding rows

template <int DP> struct Bwd {
  static constexpr int kChunks = DP / 64;
  static constexpr int kTileBytes = kChunks * kChunk;
  static constexpr int kSlots = DP == 128 ? 5 : 10;
  static constexpr int kOther = 2048 + 512;            // statistics, barriers
  static constexpr size_t kSmem = (2 + kSlots) * kTileBytes + kOther;
};

struct BwdArgs {
  AttnArgs a;
  CUtensorMap q, k, v, dout;
};

// Barriers of both kernels.
template <int kSlots> struct Bars {
  uint64_t full[kSlots], empty[kSlots];    // ring
  uint64_t own_full[2], own_empty;         // the owned tiles: one barrier each, freed together
  uint64_t s_full[2], dp_full, p_ready, ds_ready, dp_free;
  uint64_t acc_full, acc_empty;
  uint64_t stat_full[2], stat_empty[2];
  uint64_t drain;
  uint32_t tmem;
  int abort;
  uint32_t issued[kSlots], own_issued[2];  // last parity + 1 of full and own_full
};

template <int kSlots>
__device__ __forceinline__ void init_bars(Bars<kSlots>* b) {
  for (int i = 0; i < kSlots; ++i) {
    tc::mbar_init(&b->full[i], 1);
    tc::mbar_init(&b->empty[i], 1);
    b->issued[i] = 0;
  }
  for (int i = 0; i < 2; ++i) {
    tc::mbar_init(&b->own_full[i], 1);
    tc::mbar_init(&b->s_full[i], 1);
    tc::mbar_init(&b->stat_full[i], 1);
    tc::mbar_init(&b->stat_empty[i], 8);
    b->own_issued[i] = 0;
  }
  tc::mbar_init(&b->own_empty, 1);
  tc::mbar_init(&b->dp_full, 1);
  tc::mbar_init(&b->p_ready, 8);
  tc::mbar_init(&b->ds_ready, 8);
  tc::mbar_init(&b->dp_free, 8);
  tc::mbar_init(&b->acc_full, 1);
  tc::mbar_init(&b->acc_empty, 8);
  tc::mbar_init(&b->drain, 1);
  b->abort = 0;
  tc::fence_barrier_init();
}

// What every role carries: the barriers and whether its waits still hold.
template <int kSlots> struct Role {
  Bars<kSlots>* b;
  int lane;
  bool ok;
  int slot;
  uint32_t phase;
  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, &b->abort));
    tc::fence_after();
    return ok;
  }
  __device__ __forceinline__ void next() {
    if (++slot == kSlots) { slot = 0; phase ^= 1u; }
  }
  // one arrival per warp, after all its lanes' TMEM accesses
  __device__ __forceinline__ void arrive(uint64_t* bar) {
    tc::fence_before();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar);
  }
  // TMA warp: fills the next ring slot
  __device__ __forceinline__ void load(uint8_t* ring, int tile_bytes, const CUtensorMap* map, int64_t row, int head,
                                       int chunks) {
    if (!wait(&b->empty[slot], phase ^ 1u)) return;
    if (lane == 0) {
      tc::mbar_expect_tx(&b->full[slot], tile_bytes);
      b->issued[slot] = phase + 1;
      load_rows(ring + slot * tile_bytes, map, &b->full[slot], row, head, chunks);
    }
    __syncwarp();
    next();
  }
  // MMA warp: the next ring slot, once it is full
  __device__ __forceinline__ int take() {
    const int s = slot;
    wait(&b->full[s], phase);
    next();
    return s;
  }
};

// The end of both kernels: copies in flight land, TMEM is freed.
template <int kSlots>
__device__ __forceinline__ void finish(Bars<kSlots>* b, int warp) {
  __syncthreads();
  if (threadIdx.x == 0 && *static_cast<volatile int*>(&b->abort)) {
    volatile int never = 0;
    for (int i = 0; i < kSlots; ++i)
      if (b->issued[i]) tc::mbar_wait(&b->full[i], b->issued[i] - 1, &never);
    for (int i = 0; i < 2; ++i)
      if (b->own_issued[i]) tc::mbar_wait(&b->own_full[i], b->own_issued[i] - 1, &never);
  }
  __syncthreads();
  if (warp == 9) {
    tc::fence_after();
    tc::tmem_dealloc(b->tmem, 512);
  }
}

// A warp's 32 rows x (DP / 2) columns of an accumulator, scaled, to global memory.
template <int DP>
__device__ __forceinline__ void store_acc(const AttnTensor& t, uint32_t acc, int64_t row, bool in, int head, int half,
                                          float w, int dim) {
  bf16* p = static_cast<bf16*>(t.p) + row * t.ts + head * t.hs;
#pragma unroll 1
  for (int d = half * (DP / 2); d < (half + 1) * (DP / 2); d += 32) {
    uint32_t o[32];
    tc::tmem_ld32(acc + d, o);
    tc::tmem_ld_wait();
    if (in) store_row32(p, o, w, d, dim);
  }
}

struct Item {
  int64_t start;
  int len, blk, head;
};
__device__ __forceinline__ bool get_item(const AttnArgs& a, const AttnBlock* list, int heads, int64_t r, Item& it) {
  const int64_t i = walk_item(r);
  if (i >= static_cast<int64_t>(a.n_blocks) * heads) return false;
  const AttnBlock b = list[i / heads];
  it.start = b.start;
  it.len = b.len;
  it.blk = b.blk;
  it.head = static_cast<int>(i % heads);
  return true;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dkdv_tc(const __grid_constant__ BwdArgs f) {
  using B = Bwd<DP>;
  constexpr int kSlots = B::kSlots, kTileBytes = B::kTileBytes, kChunks = B::kChunks;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sK = smem;
  uint8_t* sV = sK + kTileBytes;
  uint8_t* ring = sV + kTileBytes;
  float* stat = reinterpret_cast<float*>(ring + kSlots * kTileBytes);   // [2][-log2(e) lse, delta][128]
  Bars<kSlots>* b = reinterpret_cast<Bars<kSlots>*>(stat + 512);
  static_assert(sizeof(Bars<kSlots>) <= 512, "barriers");
  const AttnArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    init_bars(b);
    for (const CUtensorMap* m : {&f.q, &f.k, &f.v, &f.dout}) tc::prefetch_map(m);
  }
  if (warp == 9) {
    tc::tmem_alloc(&b->tmem, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  const uint32_t cS = b->tmem, cP = cS + 128, cV = cS + 256, cK = cV + DP;
  Role<kSlots> role = {b, lane, true, 0, 0};
  Item it;

  if (warp == 8) {
    // ---------------- TMA ----------------
    uint32_t own = 0;
    for (int64_t r = 0; role.ok && get_item(a, a.by_key, a.kv_heads, r, it); ++r) {
      if (!role.wait(&b->own_empty, own ^ 1u)) break;
      const int64_t row = it.start + static_cast<int64_t>(kTile) * it.blk;
      if (lane == 0) {
        for (int i = 0; i < 2; ++i) {
          tc::mbar_expect_tx(&b->own_full[i], kTileBytes);
          b->own_issued[i] = own + 1;
          load_rows(i ? sV : sK, i ? &f.v : &f.k, &b->own_full[i], row, it.head, kChunks);
        }
      }
      __syncwarp();
      own ^= 1u;
      for (int g = 0; g < a.group && role.ok; ++g)
        for (int i = it.blk; i * kTile < it.len && role.ok; ++i) {
          const int64_t qrow = it.start + static_cast<int64_t>(kTile) * i;
          role.load(ring, kTileBytes, &f.q, qrow, it.head * a.group + g, kChunks);
          if (role.ok) role.load(ring, kTileBytes, &f.dout, qrow, it.head * a.group + g, kChunks);
        }
    }
  } else if (warp == 9) {
    // ---------------- MMA ----------------
    uint32_t own = 0, p_phase = 0, ds_phase = 0, acc_phase = 0;
    const uint32_t k = tc::su32(sK), v = tc::su32(sV);
    auto tile = [&](int s) { return tc::su32(ring + s * kTileBytes); };
    for (int64_t r = 0; role.ok && get_item(a, a.by_key, a.kv_heads, r, it); ++r) {
      const int nq = (it.len - 1) / kTile - it.blk + 1, n = nq * a.group;
      const int last = it.len - kTile * (it.blk + nq - 1);     // rows of the last query block
      // the tile's rows past the sequence's end become zeros
      auto take = [&](int i) {
        const int s = role.take();
        if (role.ok && last < kTile && i % nq == nq - 1) zero_tail(ring + s * kTileBytes, last, kChunks, lane);
        return s;
      };
      if (!role.wait(&b->own_full[0], own)) break;
      int q = take(0);
      if (!role.ok) break;
      if (tc::elect_one()) {
        product_ss<DP>(cS, k, tile(q));
        tc::mma_commit(&b->s_full[0]);
      }
      __syncwarp();
      if (!role.wait(&b->own_full[1], own)) break;
      own ^= 1u;
      int o = take(0);
      if (!role.ok) break;
      if (tc::elect_one()) {
        product_ss<DP>(cP, v, tile(o));
        tc::mma_commit(&b->dp_full);
        if (n == 1) tc::mma_commit(&b->own_empty);
      }
      __syncwarp();
      if (!role.wait(&b->acc_empty, acc_phase ^ 1u)) break;
      acc_phase ^= 1u;
      for (int i = 0; i < n; ++i) {
        int q2 = 0, o2 = 0;
        if (!role.wait(&b->p_ready, p_phase)) break;
        p_phase ^= 1u;
        if (tc::elect_one()) {
          product_ts<DP>(cV, cS, tile(o), i == 0, 32);
          tc::mma_commit(&b->empty[o]);
        }
        __syncwarp();
        if (i + 1 < n) {
          q2 = take(i + 1);
          if (!role.ok) break;
          if (tc::elect_one()) {
            product_ss<DP>(cS, k, tile(q2));
            tc::mma_commit(&b->s_full[0]);
          }
          __syncwarp();
        }
        if (!role.wait(&b->ds_ready, ds_phase)) break;
        ds_phase ^= 1u;
        if (tc::elect_one()) {
          product_ts<DP>(cK, cP, tile(q), i == 0, 32);
          tc::mma_commit(&b->empty[q]);
        }
        __syncwarp();
        if (i + 1 < n) {
          o2 = take(i + 1);
          if (!role.ok) break;
          if (tc::elect_one()) {
            product_ss<DP>(cP, v, tile(o2));
            tc::mma_commit(&b->dp_full);
            if (i + 2 == n) tc::mma_commit(&b->own_empty);
          }
          __syncwarp();
        }
        q = q2;
        o = o2;
      }
      if (role.ok && tc::elect_one()) tc::mma_commit(&b->acc_full);
      __syncwarp();
    }
    // every MMA issued has completed once `drain` fires
    if (tc::elect_one()) {
      tc::mma_commit(&b->drain);
      volatile int never = 0;
      tc::mbar_wait(&b->drain, 0, &never);
    }
    __syncwarp();
  } else if (warp == 10) {
    // ---------------- log-sums and deltas of the query blocks ----------------
    uint32_t phase = 0;
    int st = 0;
    for (int64_t r = 0; role.ok && get_item(a, a.by_key, a.kv_heads, r, it); ++r)
      for (int g = 0; g < a.group && role.ok; ++g) {
        const int64_t base = static_cast<int64_t>(it.head * a.group + g) * a.tokens + it.start;
        for (int i = it.blk * kTile; i < it.len; i += kTile) {
          float ls[4], de[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = i + 32 * e + lane;
            ls[e] = j < it.len ? a.lse[base + j] * -kLog2e : -INFINITY;   // past the end: P = 0
            de[e] = j < it.len ? a.delta[base + j] : 0.f;
          }
          if (!role.wait(&b->stat_empty[st], phase ^ 1u)) break;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            stat[st * 256 + 32 * e + lane] = ls[e];
            stat[st * 256 + 128 + 32 * e + lane] = de[e];
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&b->stat_full[st]);
          st ^= 1;
          if (st == 0) phase ^= 1u;
        }
      }
  } else if (warp == 11) {
    // ---------------- rows past the sequences ----------------
    zero_padding(a, a.dk, a.kv_heads, blockIdx.x, gridDim.x, lane);
    zero_padding(a, a.dv, a.kv_heads, blockIdx.x, gridDim.x, lane);
  } else {
    // ---------------- softmax ----------------
    const int half = warp >> 2, row = 32 * (warp & 3) + lane;    // columns 64 half .., row of the tile
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t mS = cS + lanes + 64 * half, mP = cP + lanes + 64 * half;
    const uint64_t c2 = tc::pack2(a.scale_log2, a.scale_log2);
    uint32_t phase = 0, stat_phase = 0, acc_phase = 0;
    int st = 0;
    for (int64_t r = 0; role.ok && get_item(a, a.by_key, a.kv_heads, r, it); ++r) {
      const int nq = (it.len - 1) / kTile - it.blk + 1, n = nq * a.group;
      for (int i = 0; i < n; ++i) {
        const float* ls = stat + st * 256 + 64 * half;
        if (!role.wait(&b->stat_full[st], stat_phase) || !role.wait(&b->s_full[0], phase)) break;
        const bool diag = i % nq == 0;
        float p[64];
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[32];
          tc::tmem_ld32(mS + 32 * h, x);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const ulonglong2 l2 = *reinterpret_cast<const ulonglong2*>(ls + 32 * h + e);
            float y[4];
            tc::unpack2(tc::fma2(tc::pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, l2.x), y[0], y[1]);
            tc::unpack2(tc::fma2(tc::pack2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])), c2, l2.y), y[2], y[3]);
#pragma unroll
            for (int u = 0; u < 4; ++u) p[32 * h + e + u] = tc::exp2_fast(y[u]);
          }
        }
        if (diag) {   // key `row` is seen by queries row ..
#pragma unroll
          for (int e = 0; e < 64; ++e)
            if (64 * half + e < row) p[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) w[e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
        tc::tmem_st32(mS, w);
        tc::tmem_st_drain();
        role.arrive(&b->p_ready);
        if (!role.wait(&b->dp_full, phase)) break;
        phase ^= 1u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[32];
          tc::tmem_ld32(mP + 32 * h, x);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 de = *reinterpret_cast<const float4*>(ls + 128 + 32 * h + e);
            const float d4[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
            for (int u = 0; u < 4; u += 2) {
              float y0 = p[32 * h + e + u] * (__uint_as_float(x[e + u]) - d4[u]);
              float y1 = p[32 * h + e + u + 1] * (__uint_as_float(x[e + u + 1]) - d4[u + 1]);
              w[16 * h + (e + u) / 2] = pack_bf16x2(y0, y1);
            }
          }
        }
        if (diag) {   // 0 * NaN in an unseen place
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            if (64 * half + 2 * e < row) w[e] &= 0xFFFF0000u;
            if (64 * half + 2 * e + 1 < row) w[e] &= 0x0000FFFFu;
          }
        }
        tc::tmem_st32(mP, w);
        tc::tmem_st_drain();
        role.arrive(&b->ds_ready);
        if (lane == 0) tc::mbar_arrive(&b->stat_empty[st]);
        st ^= 1;
        if (st == 0) stat_phase ^= 1u;
      }
      if (!role.wait(&b->acc_full, acc_phase)) break;
      acc_phase ^= 1u;
      const int64_t at = it.start + static_cast<int64_t>(kTile) * it.blk + row;
      const bool in = kTile * it.blk + row < it.len;
      store_acc<DP>(a.dv, cV + lanes, at, in, it.head, half, 1.f, a.dim);
      store_acc<DP>(a.dk, cK + lanes, at, in, it.head, half, a.scale, a.dim);
      role.arrive(&b->acc_empty);
    }
  }
  if (!role.ok && lane == 0) {
    *static_cast<volatile int*>(&b->abort) = 1;
    raise_flag(a.flags, kFlagTimeout);
  }
  finish(b, warp);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dq_tc(const __grid_constant__ BwdArgs f) {
  using B = Bwd<DP>;
  constexpr int kSlots = B::kSlots, kTileBytes = B::kTileBytes, kChunks = B::kChunks;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sQ = smem;
  uint8_t* sO = sQ + kTileBytes;
  uint8_t* ring = sO + kTileBytes;
  Bars<kSlots>* b = reinterpret_cast<Bars<kSlots>*>(ring + kSlots * kTileBytes);
  const AttnArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    init_bars(b);
    for (const CUtensorMap* m : {&f.q, &f.k, &f.v, &f.dout}) tc::prefetch_map(m);
  }
  if (warp == 9) {
    tc::tmem_alloc(&b->tmem, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  const uint32_t cS = b->tmem, cP = cS + 256, cQ = cS + 384;    // S: two buffers
  Role<kSlots> role = {b, lane, true, 0, 0};
  Item it;

  if (warp == 8) {
    // ---------------- TMA ----------------
    uint32_t own = 0;
    for (int64_t r = 0; role.ok && get_item(a, a.by_query, a.heads, r, it); ++r) {
      if (!role.wait(&b->own_empty, own ^ 1u)) break;
      const int64_t row = it.start + static_cast<int64_t>(kTile) * it.blk;
      if (lane == 0) {
        for (int i = 0; i < 2; ++i) {
          tc::mbar_expect_tx(&b->own_full[i], kTileBytes);
          b->own_issued[i] = own + 1;
          load_rows(i ? sO : sQ, i ? &f.dout : &f.q, &b->own_full[i], row, it.head, kChunks);
        }
      }
      __syncwarp();
      own ^= 1u;
      for (int j = 0; j <= it.blk && role.ok; ++j) {
        const int64_t krow = it.start + static_cast<int64_t>(kTile) * j;
        role.load(ring, kTileBytes, &f.k, krow, it.head / a.group, kChunks);
        if (role.ok) role.load(ring, kTileBytes, &f.v, krow, it.head / a.group, kChunks);
      }
    }
  } else if (warp == 9) {
    // ---------------- MMA ----------------
    uint32_t own = 0, free_phase = 0, ds_phase = 0, acc_phase = 0;
    int buf = 0;                                              // S buffer of block j
    const uint32_t q = tc::su32(sQ), o = tc::su32(sO);
    auto tile = [&](int s) { return tc::su32(ring + s * kTileBytes); };
    for (int64_t r = 0; role.ok && get_item(a, a.by_query, a.heads, r, it); ++r) {
      const int n = it.blk + 1;
      const int last = it.len - kTile * it.blk;               // keys of the diagonal block
      // the keys past the sequence's end become zeros
      auto take_k = [&](int j) {
        const int s = role.take();
        if (role.ok && last < kTile && j == it.blk) zero_tail(ring + s * kTileBytes, last, kChunks, lane);
        return s;
      };
      if (!role.wait(&b->own_full[0], own)) break;
      int k = take_k(0);
      if (!role.ok) break;
      if (tc::elect_one()) {
        product_ss<DP>(cS + 128 * buf, q, tile(k));
        tc::mma_commit(&b->s_full[buf]);
      }
      __syncwarp();
      if (!role.wait(&b->own_full[1], own)) break;
      own ^= 1u;
      int v = role.take();
      // dP's columns are free once the previous item's last block has been read
      if (!role.wait(&b->dp_free, free_phase ^ 1u)) break;
      free_phase ^= 1u;
      if (tc::elect_one()) {
        product_ss<DP>(cP, o, tile(v));
        tc::mma_commit(&b->dp_full);
        tc::mma_commit(&b->empty[v]);
        if (n == 1) tc::mma_commit(&b->own_empty);
      }
      __syncwarp();
      if (!role.wait(&b->acc_empty, acc_phase ^ 1u)) break;
      acc_phase ^= 1u;
      for (int j = 0; j < n; ++j) {
        int k2 = 0;
        if (j + 1 < n) {
          k2 = take_k(j + 1);
          if (!role.ok) break;
          if (tc::elect_one()) {
            product_ss<DP>(cS + 128 * (buf ^ 1), q, tile(k2));
            tc::mma_commit(&b->s_full[buf ^ 1]);
          }
          __syncwarp();
          v = role.take();
          if (!role.wait(&b->dp_free, free_phase ^ 1u)) break;
          free_phase ^= 1u;
          if (tc::elect_one()) {
            product_ss<DP>(cP, o, tile(v));
            tc::mma_commit(&b->dp_full);
            tc::mma_commit(&b->empty[v]);
            if (j + 2 == n) tc::mma_commit(&b->own_empty);
          }
          __syncwarp();
        }
        if (!role.wait(&b->ds_ready, ds_phase)) break;
        ds_phase ^= 1u;
        if (tc::elect_one()) {
          product_ts<DP>(cQ, cS + 128 * buf, tile(k), j == 0, 32);
          tc::mma_commit(&b->empty[k]);
        }
        __syncwarp();
        k = k2;
        buf ^= 1;
      }
      if (role.ok && tc::elect_one()) tc::mma_commit(&b->acc_full);
      __syncwarp();
    }
    if (tc::elect_one()) {
      tc::mma_commit(&b->drain);
      volatile int never = 0;
      tc::mbar_wait(&b->drain, 0, &never);
    }
    __syncwarp();
  } else if (warp >= 10) {
    // ---------------- rows past the sequences ----------------
    zero_padding(a, a.dq, a.heads, 2 * static_cast<int64_t>(blockIdx.x) + warp - 10, 2 * static_cast<int64_t>(gridDim.x),
                 lane);
  } else {
    // ---------------- softmax ----------------
    const int half = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint64_t c2 = tc::pack2(a.scale_log2, a.scale_log2);
    uint32_t s_phase[2] = {0, 0}, dp_phase = 0, acc_phase = 0;
    int buf = 0;
    for (int64_t r = 0; role.ok && get_item(a, a.by_query, a.heads, r, it); ++r) {
      const int64_t at = it.start + static_cast<int64_t>(kTile) * it.blk + row;
      const bool in = kTile * it.blk + row < it.len;
      const int64_t si = static_cast<int64_t>(it.head) * a.tokens + at;
      const float ls = in ? a.lse[si] * -kLog2e : -INFINITY, de = in ? a.delta[si] : 0.f;
      const uint64_t ls2 = tc::pack2(ls, ls);
      for (int j = 0; j <= it.blk; ++j) {
        const uint32_t mS = cS + 128 * buf + lanes + 64 * half, mP = cP + lanes + 64 * half;
        if (!role.wait(&b->s_full[buf], buf ? s_phase[1] : s_phase[0])) break;
        if (buf) s_phase[1] ^= 1u; else s_phase[0] ^= 1u;
        float p[64];
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[32];
          tc::tmem_ld32(mS + 32 * h, x);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float y0, y1;
            tc::unpack2(tc::fma2(tc::pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, ls2), y0, y1);
            p[32 * h + e] = tc::exp2_fast(y0);
            p[32 * h + e + 1] = tc::exp2_fast(y1);
          }
        }
        if (!role.wait(&b->dp_full, dp_phase)) break;
        dp_phase ^= 1u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[32];
          tc::tmem_ld32(mP + 32 * h, x);
          tc::tmem_ld_wait();
          if (h == 1) role.arrive(&b->dp_free);
#pragma unroll
          for (int e = 0; e < 32; e += 2)
            w[16 * h + e / 2] = pack_bf16x2(p[32 * h + e] * (__uint_as_float(x[e]) - de),
                                            p[32 * h + e + 1] * (__uint_as_float(x[e + 1]) - de));
        }
        if (j == it.blk) {   // query `row` sees keys .. row
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            if (64 * half + 2 * e > row) w[e] &= 0xFFFF0000u;
            if (64 * half + 2 * e + 1 > row) w[e] &= 0x0000FFFFu;
          }
        }
        tc::tmem_st32(mS, w);
        tc::tmem_st_drain();
        role.arrive(&b->ds_ready);
        buf ^= 1;
      }
      if (!role.wait(&b->acc_full, acc_phase)) break;
      acc_phase ^= 1u;
      store_acc<DP>(a.dq, cQ + lanes, at, in, it.head, half, a.scale, a.dim);
      role.arrive(&b->acc_empty);
    }
  }
  if (!role.ok && lane == 0) {
    *static_cast<volatile int*>(&b->abort) = 1;
    raise_flag(a.flags, kFlagTimeout);
  }
  finish(b, warp);
}

template <typename K>
cudaError_t launch(K* kernel, const BwdArgs& f, int heads, size_t smem, cudaStream_t s) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e) return e;
  const int64_t items = std::max<int64_t>(1, static_cast<int64_t>(f.a.n_blocks) * heads);
  kernel<<<static_cast<int>(std::min<int64_t>(items, device_sm_count())), kThreads, smem, s>>>(f);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attn_backward_tc(const AttnArgs& a, cudaStream_t s, std::string* err) {
  BwdArgs f;
  f.a = a;
  if (!rows_map(&f.q, a.q, a.tokens, a.heads, a.dim, err) || !rows_map(&f.k, a.k, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.v, a.v, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.dout, a.dout, a.tokens, a.heads, a.dim, err))
    return cudaErrorInvalidValue;
  cudaError_t e;
  if (a.dim <= 64) {
    e = launch(k_attn_dkdv_tc<64>, f, a.kv_heads, Bwd<64>::kSmem, s);
    return e ? e : launch(k_attn_dq_tc<64>, f, a.heads, Bwd<64>::kSmem, s);
  }
  e = launch(k_attn_dkdv_tc<128>, f, a.kv_heads, Bwd<128>::kSmem, s);
  return e ? e : launch(k_attn_dq_tc<128>, f, a.heads, Bwd<128>::kSmem, s);
}

}  // namespace normpre
