// Packed causal attention, backward, bf16 on tcgen05 tensor cores.
//
//   P = exp2(log2(e) (scale S - lse)),  dS = P (dP - delta),  S = Q K^T, dP = dO V^T,
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
//
// Two walks: one (k_attn_dkdv) owns 128 keys and walks the queries that see them
// (over the heads of the group and the later blocks), one (k_attn_dq) owns 128
// queries and walks their keys.  Every gradient is then summed by one CTA in
// one accumulator in a fixed order, without atomics or fp32 partials in global
// memory; the price is that S and dP are formed twice, 7 products of a tile
// instead of 5.
//
// Both: one CTA per SM walks the work list; the owned tiles stay in shared
// memory, the others pass through a ring filled by a TMA warp; sixteen softmax
// warps each take 32 rows x 32 columns of a score tile, one row a thread.  P
// and dS go back to TMEM as bf16 over the scores they came from (each warp
// group inside its own quarter of the columns) and are the A operands of the
// products that follow.  Two warps issue the MMAs, each one of the two chains
// below: a thread's MMAs run almost as it issues them, so that while it waits
// the tensor cores need another's.
//
// k_attn_dkdv forms the transposed tiles S^T, dP^T (rows: keys), so that P^T
// and dS^T lie in TMEM as the A operands of dV and dK.  Chains: P(i) -> dV(i),
// S(i+1) and dS(i) -> dK(i), dP(i+1).  TMEM at head_dim 128: S^T 128, dP^T 128,
// dV 128, dK 128 columns, all there is.
// With a window, the walks are those of the rows that see each other, in one
// launch (k_attn_bwd_tc); of the last sink block that a query block meets, the walk
// of dQ takes 32 keys only where no more are visible (see WindowKind).  A key block
// of sinks meets all later queries: its item is split (see KeyPart) and the parts'
// fp32 sums are joined by k_attn_join.
// k_attn_dq: S in two buffers, dP, dQ; dS lies over S, so that dP(j+1) starts
// as soon as dP(j) has been read.  Chains: dS(j) -> dQ(j), S(j+2) and dP(j).
// Head dimensions up to 64 leave room for a second set of owned tiles and a
// second set of accumulators, so that an item's start and end overlap its
// neighbours.
//
// scale S - lse is one FMA, rounded once and where it matters small: scaled by
// log2(e) beforehand, scale S and lse would each carry a rounding of their own
// size into the exponent.
//
// Roundings to bf16: P and dS once each (MMA operands), the gradients once.
//
// What bounds it: the products.  16384 tokens, 16 / 8 heads of 128: 2.5 ms alone,
// 2.58 ms in a loop, where the seven products run at 1490 TFLOP/s and the clock
// falls with the power limit.  Short sequences add the items' ends (the
// gradients' way from TMEM to memory, 2000 cycles against 2050 an iteration of
// dK, dV at head_dim 64): 8 x 1024 tokens, 12 heads of 64, 0.091 ms.  With few key
// / value heads the key blocks of a long sequence do not fill the GPU: one of 4096
// tokens, 8 / 1 heads of 128, is 32 items of dK, dV, 0.45 ms (190 TFLOP/s of the
// five products that are needed).  32768 tokens, 16 / 8 heads of 128, window 4096, 4
// sinks: 2.6 ms (990 TFLOP/s of the five products of the visible pairs, 1470 of the
// seven with the tiles' hidden ones, under the power limit).  8 x 1024 tokens, 12
// heads of 64, window 256: 0.066 to 0.070 ms, three steps an item, half of it the
// items' ends.
#include <algorithm>

#include "attn_tc.cuh"

namespace normpre {
namespace {

constexpr int kSoftmax = 16;    // warps
constexpr int kTma = 16, kMmaA = 17, kStats = 18, kMmaB = 19;   // warps: TMA, MMA, statistics and sequence ends, MMA
constexpr int kThreads = 640;

template <int DP> struct Bwd {
  static constexpr int kChunks = DP / 64;
  static constexpr int kTileBytes = kChunks * kChunk;
  static constexpr int kSlots = DP == 128 ? 5 : 8;
  static constexpr int kSets = DP == 128 ? 1 : 2;      // owned tiles, accumulators
  static constexpr int kOther = 2048 + 512 + 512;      // statistics, barriers, items
  static constexpr size_t kSmem = (2 * kSets + kSlots) * kTileBytes + kOther;
};

struct BwdArgs {
  AttnArgs a;
  CUtensorMap q, k, v, dout;
};

// Barriers of both kernels.
template <int kSlots> struct Bars {
  // raw: a tile that ends its sequence lands here first; once its tail is
  // zeroed it counts as full
  uint64_t full[kSlots], empty[kSlots], raw[kSlots];
  uint64_t own_full[2][2], own_empty[2];   // per set: the two owned tiles, freed together
  // ds_ready, dQ: one per buffer of S.  The softmax warps can be done with both
  // buffers before the MMA thread looks: on one barrier that would be two phases
  // ahead, which its parity cannot tell from none.
  uint64_t s_full[2], dp_full, p_ready, ds_ready[2], dp_free;
  uint64_t acc_full[2], acc_empty[2];
  uint64_t stat_empty[2];
  uint64_t drain[2];
  uint32_t tmem;
  int abort;
  uint32_t issued[kSlots], raw_issued[kSlots], own_issued[2];  // loads so far
};

// `users`: MMA chains that read a ring tile, and that add to an accumulator set
// (two in dK, dV, one in dQ).
template <int kSlots>
__device__ __forceinline__ void init_bars(Bars<kSlots>* b, int users) {
  for (int i = 0; i < kSlots; ++i) {
    tc::mbar_init(&b->full[i], 1);
    tc::mbar_init(&b->empty[i], users);
    tc::mbar_init(&b->raw[i], 1);
    b->issued[i] = b->raw_issued[i] = 0;
  }
  for (int i = 0; i < 2; ++i) {
    tc::mbar_init(&b->own_full[i][0], 1);
    tc::mbar_init(&b->own_full[i][1], 1);
    tc::mbar_init(&b->own_empty[i], 2);
    tc::mbar_init(&b->s_full[i], users);             // dK, dV: the scores and their statistics
    tc::mbar_init(&b->stat_empty[i], kSoftmax);
    tc::mbar_init(&b->acc_full[i], users);
    tc::mbar_init(&b->acc_empty[i], kSoftmax);
    tc::mbar_init(&b->drain[i], 1);
    b->own_issued[i] = 0;
  }
  tc::mbar_init(&b->dp_full, 1);
  tc::mbar_init(&b->p_ready, kSoftmax);
  for (int i = 0; i < 2; ++i) tc::mbar_init(&b->ds_ready[i], kSoftmax);
  tc::mbar_init(&b->dp_free, kSoftmax);
  b->abort = 0;
  tc::fence_barrier_init();
}

// Alternates over `sets` buffers; `parity` is of the current one's uses.
template <int sets> struct Turn {
  int i = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void next() {
    if (++i == sets) { i = 0; parity ^= 1u; }
  }
};

// What a warp carries: the barriers, whether its waits still hold, and its
// place in the ring.
template <int kSlots> struct Warp {
  Bars<kSlots>* b;
  int lane;
  bool ok;
  int slot;
  uint32_t phase;
  // all lanes of the warp
  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, &b->abort));
    tc::fence_after();
    return ok;
  }
  // one thread
  __device__ __forceinline__ bool wait1(uint64_t* bar, uint32_t parity) {
    ok = ok && tc::mbar_wait(bar, parity, &b->abort);
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
  // TMA thread: fills the next ring slot
  __device__ __forceinline__ void load(uint8_t* ring, int tile_bytes, const CUtensorMap* map, int64_t row, int head,
                                       int chunks, bool tail) {
    if (!wait1(&b->empty[slot], phase ^ 1u)) return;
    uint64_t* bar = tail ? &b->raw[slot] : &b->full[slot];
    tc::mbar_expect_tx(bar, tile_bytes);
    if (tail) ++b->raw_issued[slot];
    else b->issued[slot] = phase + 1;
    load_rows(ring + slot * tile_bytes, map, bar, row, head, chunks);
    next();
  }
  // TMA thread: the two owned tiles of a set
  __device__ __forceinline__ bool load_own(uint8_t* tiles, int tile_bytes, int set, uint32_t parity,
                                           const CUtensorMap* m0, const CUtensorMap* m1, int64_t row, int head,
                                           int chunks) {
    if (!wait1(&b->own_empty[set], parity ^ 1u)) return false;
    for (int i = 0; i < 2; ++i) {
      tc::mbar_expect_tx(&b->own_full[set][i], tile_bytes);
      load_rows(tiles + (2 * set + i) * tile_bytes, i ? m1 : m0, &b->own_full[set][i], row, head, chunks);
    }
    ++b->own_issued[set];
    return true;
  }
  // MMA thread: the ring slot `ahead` places on, once it is full
  __device__ __forceinline__ int take() {
    const int s = slot;
    wait1(&b->full[s], phase);
    next();
    return s;
  }
  // warp: zeroes the end of a ring tile that just arrived, and passes it on
  __device__ __forceinline__ bool end_tile(uint8_t* ring, int tile_bytes, int s, uint32_t& seen, int rows, int chunks) {
    if (!wait(&b->raw[s], (seen >> s) & 1u)) return false;
    seen ^= 1u << s;
    zero_tail(ring + s * tile_bytes, rows, chunks, lane);
    if (lane == 0) tc::mbar_arrive(&b->full[s]);
    return true;
  }
  // MMA thread: every MMA issued has completed when this returns
  __device__ __forceinline__ void drain(int i) {
    int never = 0;
    tc::mma_commit(&b->drain[i]);
    tc::mbar_wait(&b->drain[i], 0, &never);
  }
};

// The end of both walks: copies in flight land.  False if a wait gave up.
template <int kSlots>
__device__ __forceinline__ bool finish(const Warp<kSlots>& w, int* flags) {
  Bars<kSlots>* b = w.b;
  if (!w.ok && w.lane == 0) {
    *static_cast<volatile int*>(&b->abort) = 1;
    raise_host_flag(flags, kFlagTimeout);
  }
  __syncthreads();
  const bool gave_up = *static_cast<volatile int*>(&b->abort);
  if (threadIdx.x == 0 && gave_up) {
    int never = 0;
    for (int i = 0; i < kSlots; ++i) {
      if (b->issued[i]) tc::mbar_wait(&b->full[i], b->issued[i] - 1, &never);
      if (b->raw_issued[i]) tc::mbar_wait(&b->raw[i], (b->raw_issued[i] - 1) & 1u, &never);
    }
    for (int i = 0; i < 4; ++i)
      if (b->own_issued[i >> 1]) tc::mbar_wait(&b->own_full[i >> 1][i & 1], (b->own_issued[i >> 1] - 1) & 1u, &never);
  }
  __syncthreads();
  return !gave_up;
}
__device__ __forceinline__ void free_tmem(uint32_t tmem) {
  if (threadIdx.x >> 5 == kMmaA) {
    tc::fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
}

// A warp's 32 rows x (DP / 4) columns of an accumulator, scaled, to the tile
// at row `row`, of which `rows` exist.
template <int DP>
__device__ __forceinline__ void store_acc(const AttnTensor& t, uint32_t acc, int64_t row, int rows, int head, int warp,
                                          float w, int dim, int lane) {
  constexpr int kCols = DP / 4;
  const int part = warp >> 2;
  uint32_t o[kCols];
  if constexpr (kCols == 32) tc::tmem_ld32(acc + kCols * part, o);
  else tc::tmem_ld16(acc + kCols * part, o);
  tc::tmem_ld_wait();
  store_rows<kCols>(static_cast<bf16*>(t.p) + row * t.ts + head * t.hs, t.ts, o, w, 32 * (warp & 3), rows, kCols * part,
                    dim, lane);
}

// An accumulator's 32 rows x (DP / 4) columns of a warp to a part's fp32 sums.
template <int DP>
__device__ __forceinline__ void store_part(float* to, uint32_t acc, int warp, int dim, int lane) {
  constexpr int kCols = DP / 4;
  const int c = kCols * (warp >> 2);
  uint32_t o[kCols];
  if constexpr (kCols == 32) tc::tmem_ld32(acc + c, o);
  else tc::tmem_ld16(acc + c, o);
  tc::tmem_ld_wait();
  float* p = to + static_cast<int64_t>(32 * (warp & 3) + lane) * dim + c;
#pragma unroll
  for (int i = 0; i < kCols; i += 4)
    if (c + i < dim) *reinterpret_cast<uint4*>(p + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
}

struct Item {
  int64_t start;
  int len, blk, head;
};

constexpr int kCached = 32;

// An item of dK, dV: a key block and head, and the query blocks first .. end.
struct alignas(16) KeyItem {
  int start, len, blk, head, first, end, slot, pad;   // blk -1: no item
};
constexpr int kKeyCached = 16;                        // 512 bytes
static_assert(kKeyCached * sizeof(KeyItem) <= 512, "items");
// Not inlined: in every role of the kernel, for the few items past the cached
// ones, it would push the roles' loops apart in the instruction cache (4 % of a
// pass over short items).  The same for the items of dQ.
template <bool WIN>
__device__ __noinline__ KeyItem key_item(const AttnArgs& a, int64_t r) {
  KeyItem k = {0, 0, -1, 0, 0, 0, -1, 0};
  const int64_t i = walk_item(a.walk_dkdv, r, static_cast<int64_t>(a.n_keys) * a.kv_heads, a.flags);
  if (i < 0) return k;
  const AttnBlock b = a.by_key[i / a.kv_heads];
  KeyPart p = {b.blk, (b.len - 1) / kTile + 1, -1, b.part == 0};
  if (WIN && block_fits(b, a.total)) p = key_part(b, a.window, a.sinks, a.chunk, a.slots);
  if (!block_fits(b, a.total) || !p.fits) {
    raise_host_flag(a.flags, kFlagLists);
    return k;
  }
  return KeyItem{b.start, b.len, b.blk, static_cast<int>(i % a.kv_heads), p.first, p.end, p.slot, 0};
}
__device__ __noinline__ ItemRef query_item(const AttnArgs& a, int64_t r) {
  return list_item(a, a.by_query, a.n_blocks, a.walk_dq, a.heads, r);
}

__device__ __forceinline__ bool get_item(const ItemRef& b, Item& it) {
  if (b.blk < 0) return false;
  it.start = b.start;
  it.len = b.len;
  it.blk = b.blk;
  it.head = b.head;
  return true;
}

// dK, dV.  WIN: the rows have a window.  Allocates all of TMEM.
template <int DP, bool WIN>
__device__ __forceinline__ bool walk_dkdv(const BwdArgs& f, uint8_t* smem, uint32_t& tmem) {
  using B = Bwd<DP>;
  constexpr int kSlots = B::kSlots, kTileBytes = B::kTileBytes, kChunks = B::kChunks, kSets = B::kSets;
  uint8_t* own = smem;                                // [kSets] K, V
  uint8_t* ring = own + 2 * kSets * kTileBytes;       // Q, dO, Q, dO ..
  float* stat = reinterpret_cast<float*>(ring + kSlots * kTileBytes);   // [2][-lse, delta][128]
  Bars<kSlots>* b = reinterpret_cast<Bars<kSlots>*>(stat + 512);
  static_assert(sizeof(Bars<kSlots>) <= 512, "barriers");
  KeyItem* items = reinterpret_cast<KeyItem*>(reinterpret_cast<uint8_t*>(b) + 512);   // [kKeyCached]
  const AttnArgs& a = f.a;
  auto get = [&](int64_t r, KeyItem& it) {
    it = r < kKeyCached ? items[r] : key_item<WIN>(a, r);
    return it.blk >= 0;
  };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    init_bars(b, 2);
    for (const CUtensorMap* m : {&f.q, &f.k, &f.v, &f.dout}) tc::prefetch_map(m);
  }
  if (warp == 2 && lane < kKeyCached) items[lane] = key_item<WIN>(a, lane);
  if (warp == kMmaA) {
    tc::tmem_alloc(&b->tmem, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  tmem = b->tmem;
  const uint32_t cS = tmem, cP = cS + 128, cAcc = cS + 256;     // per set: dV, dK
  Warp<kSlots> w = {b, lane, true, 0, 0};
  Turn<kSets> set;
  KeyItem it;

  if (warp == kTma) {
    // ---------------- TMA (one thread), then the rows past the sequences ----------------
    if (tc::elect_one()) {
      for (int64_t r = 0; w.ok && get(r, it); ++r, set.next()) {
        const int64_t row = it.start + static_cast<int64_t>(kTile) * it.blk;
        if (!w.load_own(own, kTileBytes, set.i, set.parity, &f.k, &f.v, row, it.head, kChunks)) break;
        if (a.test_stall == 2 && blockIdx.x == 0) break;          // no queries: the others' waits run out
        for (int g = 0; g < a.group && w.ok; ++g)
          for (int i = it.first; i < it.end && w.ok; ++i) {
            const int64_t qrow = it.start + static_cast<int64_t>(kTile) * i;
            const bool tail = kTile * (i + 1) > it.len;
            w.load(ring, kTileBytes, &f.q, qrow, it.head * a.group + g, kChunks, tail);
            if (w.ok) w.load(ring, kTileBytes, &f.dout, qrow, it.head * a.group + g, kChunks, tail);
          }
      }
    }
    w.ok = __all_sync(0xffffffffu, w.ok);
    zero_padding(a, a.dk, a.kv_heads, blockIdx.x, gridDim.x, lane);
    zero_padding(a, a.dv, a.kv_heads, blockIdx.x, gridDim.x, lane);
  } else if (warp == kMmaA) {
    // ---------------- MMA (one thread): dV(i), S(i + 1) ----------------
    if (tc::elect_one()) {
      uint32_t p_phase = 0;
      int st = 0;                                                 // parity of the block in the walk
      auto tile = [&](int s) { return tc::su32(ring + s * kTileBytes); };
      for (int64_t r = 0; w.ok && get(r, it); ++r, set.next()) {
        const int n = (it.end - it.first) * a.group;
        const uint32_t k = tc::su32(own + 2 * set.i * kTileBytes);
        if (!w.wait1(&b->own_full[set.i][0], set.parity)) break;
        int q = w.take();
        if (!w.ok) break;
        product_ss<DP>(cS, k, tile(q));
        tc::mma_commit(&b->s_full[st]);
        st ^= 1;
        tc::mma_commit(&b->empty[q]);
        if (n == 1) tc::mma_commit(&b->own_empty[set.i]);
        if (!w.wait1(&b->acc_empty[set.i], set.parity ^ 1u)) break;
        for (int i = 0; i < n; ++i) {
          const int o = w.take();
          if (!w.wait1(&b->p_ready, p_phase)) break;
          p_phase ^= 1u;
          product_ts<DP, 4>(cAcc + 2 * DP * set.i, cS, tile(o), i == 0);
          tc::mma_commit(&b->empty[o]);
          if (i + 1 == n) break;
          q = w.take();
          if (!w.ok) break;
          product_ss<DP>(cS, k, tile(q));
          tc::mma_commit(&b->s_full[st]);
          st ^= 1;
          tc::mma_commit(&b->empty[q]);
          if (i + 2 == n) tc::mma_commit(&b->own_empty[set.i]);
        }
        if (w.ok) tc::mma_commit(&b->acc_full[set.i]);
      }
      w.drain(0);
    }
    __syncwarp();
    w.ok = __all_sync(0xffffffffu, w.ok);
  } else if (warp == kMmaB) {
    // ---------------- MMA (one thread): dK(i), dP(i + 1) ----------------
    if (tc::elect_one()) {
      uint32_t ds_phase = 0;
      auto tile = [&](int s) { return tc::su32(ring + s * kTileBytes); };
      for (int64_t r = 0; w.ok && get(r, it); ++r, set.next()) {
        const int n = (it.end - it.first) * a.group;
        const uint32_t v = tc::su32(own + (2 * set.i + 1) * kTileBytes);
        if (!w.wait1(&b->own_full[set.i][1], set.parity)) break;
        int q = w.take(), o = w.take();
        if (!w.ok) break;
        product_ss<DP>(cP, v, tile(o));
        tc::mma_commit(&b->dp_full);
        tc::mma_commit(&b->empty[o]);
        if (n == 1) tc::mma_commit(&b->own_empty[set.i]);
        if (!w.wait1(&b->acc_empty[set.i], set.parity ^ 1u)) break;
        for (int i = 0; i < n; ++i) {
          if (!w.wait1(&b->ds_ready[0], ds_phase)) break;
          ds_phase ^= 1u;
          product_ts<DP, 4>(cAcc + 2 * DP * set.i + DP, cP, tile(q), i == 0);
          tc::mma_commit(&b->empty[q]);
          if (i + 1 == n) break;
          q = w.take();
          o = w.take();
          if (!w.ok) break;
          product_ss<DP>(cP, v, tile(o));
          tc::mma_commit(&b->dp_full);
          tc::mma_commit(&b->empty[o]);
          if (i + 2 == n) tc::mma_commit(&b->own_empty[set.i]);
        }
        if (w.ok) tc::mma_commit(&b->acc_full[set.i]);
      }
      w.drain(1);
    }
    __syncwarp();
    w.ok = __all_sync(0xffffffffu, w.ok);
  } else if (warp == kStats) {
    // ---------------- log-sums and deltas of the query blocks, sequence ends ----------------
    Turn<2> st;
    uint32_t seen = 0;
    int slot = 0;
    for (int64_t r = 0; w.ok && get(r, it); ++r) {
      const int end = min(it.len, kTile * it.end);
      for (int g = 0; g < a.group && w.ok; ++g) {
        const int64_t base = static_cast<int64_t>(it.head * a.group + g) * a.tokens + it.start;
        for (int i = it.first * kTile; i < end; i += kTile) {
          float ls[4], de[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = i + 32 * e + lane;
            ls[e] = j < it.len ? -a.lse[base + j] : -INFINITY;   // past the end: P = 0
            de[e] = j < it.len ? a.delta[base + j] : 0.f;
          }
          const int s0 = slot, s1 = s0 + 1 == kSlots ? 0 : s0 + 1;
          slot = s1 + 1 == kSlots ? 0 : s1 + 1;
          if (it.len - i < kTile && (!w.end_tile(ring, kTileBytes, s0, seen, it.len - i, kChunks) ||
                                     !w.end_tile(ring, kTileBytes, s1, seen, it.len - i, kChunks)))
            break;
          if (!w.wait(&b->stat_empty[st.i], st.parity ^ 1u)) break;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            stat[st.i * 256 + 32 * e + lane] = ls[e];
            stat[st.i * 256 + 128 + 32 * e + lane] = de[e];
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&b->s_full[st.i]);
          st.next();
        }
      }
    }
  } else {
    // ---------------- softmax ----------------
    const int part = warp >> 2, row = 32 * (warp & 3) + lane;    // columns 32 part .., row of the tile
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t mS = cS + lanes + 32 * part, mP = cP + lanes + 32 * part;
    const uint64_t c2 = tc::pack2(a.scale, a.scale), log2e2 = tc::pack2(kLog2e, kLog2e);
    uint32_t phase = 0;
    Turn<2> st;
    for (int64_t r = 0; w.ok && get(r, it); ++r, set.next()) {
      // what the loop needs of the item; the rest is fetched again after it
      const int nq = it.end - it.first, n = nq * a.group, gap = it.first - it.blk;
      const int sinks = WIN ? a.sinks - kTile * it.blk : 0;    // among these keys
      for (int i = 0; i < n; ++i) {
        const float* ls = stat + st.i * 256 + 32 * part;
        if (!w.wait(&b->s_full[st.i], st.parity)) break;
        const int up = gap + i % nq;   // blocks between the keys and the queries
        const bool diag = up == 0;
        // the window's end crosses the tile, and not only over sinks
        const bool edge = WIN && kTile * (up + 1) > a.window && sinks < kTile;
        // the tile's queries that do not see key `row`, a bit for each column
        uint32_t hide = 0;
        if (WIN && (diag || edge)) {
          hide = below_bits(row - kTile * up - 32 * part);
          if (row >= sinks) hide |= ~below_bits(row + a.window - kTile * up - 32 * part);
        }
        float p[32];
        uint32_t pk[16];
        uint32_t x[32];
        tc::tmem_ld32(mS, x);
        tc::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const ulonglong2 l2 = *reinterpret_cast<const ulonglong2*>(ls + e);
          float y[4];
          tc::unpack2(tc::mul2(tc::fma2(tc::pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, l2.x), log2e2), y[0], y[1]);
          tc::unpack2(tc::mul2(tc::fma2(tc::pack2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])), c2, l2.y), log2e2), y[2], y[3]);
#pragma unroll
          for (int u = 0; u < 4; ++u) p[e + u] = tc::exp2_fast(y[u]);
        }
        if constexpr (WIN) {
          if (diag || edge) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (hide >> e & 1u) p[e] = 0.f;
          }
        } else if (diag) {   // key `row` is seen by queries row ..
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * part + e < row) p[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) pk[e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
        tc::tmem_put16(mS, pk);
        tc::tmem_st_drain();
        w.arrive(&b->p_ready);
        if (!w.wait(&b->dp_full, phase)) break;
        phase ^= 1u;
        tc::tmem_ld32(mP, x);
        tc::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 de = *reinterpret_cast<const float4*>(ls + 128 + e);
          const float d4[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
          for (int u = 0; u < 4; u += 2)
            pk[(e + u) / 2] = pack_bf16x2(p[e + u] * (__uint_as_float(x[e + u]) - d4[u]),
                                          p[e + u + 1] * (__uint_as_float(x[e + u + 1]) - d4[u + 1]));
        }
        if constexpr (WIN) {
          if (diag || edge) {   // 0 * NaN in an unseen place
            if (sees_itself(a.window, a.sinks)) hide = ~0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if (hide >> (2 * e) & 1u) pk[e] &= 0xFFFF0000u;
              if (hide >> (2 * e + 1) & 1u) pk[e] &= 0x0000FFFFu;
            }
          }
        } else if (diag) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (32 * part + 2 * e < row) pk[e] &= 0xFFFF0000u;
            if (32 * part + 2 * e + 1 < row) pk[e] &= 0x0000FFFFu;
          }
        }
        tc::tmem_put16(mP, pk);
        tc::tmem_st_drain();
        w.arrive(&b->ds_ready[0]);
        if (lane == 0) tc::mbar_arrive(&b->stat_empty[st.i]);
        st.next();
      }
      if (!w.wait(&b->acc_full[set.i], set.parity) || !get(r, it)) break;
      const int64_t at = it.start + static_cast<int64_t>(kTile) * it.blk;
      const int rows = it.len - kTile * it.blk;
      const uint32_t acc = cAcc + 2 * DP * set.i + lanes;
      if (WIN && it.slot >= 0) {
        float* to = a.partial + (static_cast<int64_t>(it.slot) * a.kv_heads + it.head) * 2 * kTile * a.dim;
        store_part<DP>(to, acc + DP, warp, a.dim, lane);
        store_part<DP>(to + kTile * a.dim, acc, warp, a.dim, lane);
      } else {
        store_acc<DP>(a.dv, acc, at, rows, it.head, warp, 1.f, a.dim, lane);
        store_acc<DP>(a.dk, acc + DP, at, rows, it.head, warp, a.scale, a.dim, lane);
      }
      w.arrive(&b->acc_empty[set.i]);
    }
  }
  return finish(w, a.flags);
}

// dQ.  FIRST: allocates TMEM, else `tmem` is its address.  Its barriers lie where
// the other walk has its statistics: none of those that arrived there are touched.
template <int DP, int KIND, bool FIRST>
__device__ __forceinline__ void walk_dq(const BwdArgs& f, uint8_t* smem, uint32_t& tmem) {
  constexpr bool WIN = KIND != kWhole, kFew = KIND == kWindowNarrow;
  using B = Bwd<DP>;
  constexpr int kSlots = B::kSlots, kTileBytes = B::kTileBytes, kChunks = B::kChunks, kSets = B::kSets;
  uint8_t* own = smem;                                // [kSets] Q, dO
  uint8_t* ring = own + 2 * kSets * kTileBytes;       // K, V, K, V ..
  Bars<kSlots>* b = reinterpret_cast<Bars<kSlots>*>(ring + kSlots * kTileBytes);
  ItemRef* items = reinterpret_cast<ItemRef*>(reinterpret_cast<uint8_t*>(b) + 512);   // [kCached]
  const AttnArgs& a = f.a;
  auto keys = [&](const Item& it) { return WIN ? key_span(it.blk, a.window, a.sinks) : KeySpan{0, 0}; };
  auto item = [&](int64_t r) { return r < kCached ? items[r] : query_item(a, r); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    init_bars(b, 1);
    for (const CUtensorMap* m : {&f.q, &f.k, &f.v, &f.dout}) tc::prefetch_map(m);
  }
  if (warp == 2) items[lane] = query_item(a, lane);
  if (FIRST && warp == kMmaA) {
    tc::tmem_alloc(&b->tmem, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  if (FIRST) tmem = b->tmem;
  const uint32_t cS = tmem, cP = cS + 256, cAcc = cS + 384;    // S: two buffers; per set: dQ
  Warp<kSlots> w = {b, lane, true, 0, 0};
  Turn<kSets> set;
  Turn<2> buf;                                                    // of S
  Item it;

  if (warp == kTma) {
    // ---------------- TMA (one thread), then the rows past the sequences ----------------
    if (tc::elect_one()) {
      for (int64_t r = 0; w.ok && get_item(item(r), it); ++r, set.next()) {
        const int64_t row = it.start + static_cast<int64_t>(kTile) * it.blk;
        if (!w.load_own(own, kTileBytes, set.i, set.parity, &f.q, &f.dout, row, it.head, kChunks)) break;
        const KeySpan span = keys(it);
        for (int j = span.first(); j <= it.blk && w.ok; j = WIN ? span.up(j) : j + 1) {
          const int64_t krow = it.start + static_cast<int64_t>(kTile) * j;
          w.load(ring, kTileBytes, &f.k, krow, it.head / a.group, kChunks, kTile * (j + 1) > it.len);
          if (w.ok) w.load(ring, kTileBytes, &f.v, krow, it.head / a.group, kChunks, false);
        }
      }
    }
    w.ok = __all_sync(0xffffffffu, w.ok);
    zero_padding(a, a.dq, a.heads, blockIdx.x, gridDim.x, lane);
  } else if (warp == kMmaA) {
    // ---------------- MMA (one thread): dQ(j), S(j + 2) ----------------
    if (tc::elect_one()) {
      uint32_t ds_phase = 0;                                      // a bit per buffer
      auto tile = [&](int s) { return tc::su32(ring + s * kTileBytes); };
      for (int64_t r = 0; w.ok && get_item(item(r), it); ++r, set.next()) {
        const int n = keys(it).count(it.blk);
        const int narrow = kFew ? keys(it).narrow(a.sinks) : -1;     // a block's number in the walk too: the sinks' come first
        const uint32_t q = tc::su32(own + 2 * set.i * kTileBytes);
        int k[2] = {0, 0};                                        // ring slots of K(j), K(j + 1)
        auto scores = [&](int j, int& slot) {
          slot = w.take();
          w.next();                                               // V is the other chain's
          if (!w.ok) return;
          if (kFew && j == narrow) product_ss<DP, 0, DP / 16, 32>(cS + 128 * (buf.i ^ (j & 1)), q, tile(slot));
          else product_ss<DP>(cS + 128 * (buf.i ^ (j & 1)), q, tile(slot));
          tc::mma_commit(&b->s_full[buf.i ^ (j & 1)]);
          if (j + 1 == n) tc::mma_commit(&b->own_empty[set.i]);
        };
        if (!w.wait1(&b->own_full[set.i][0], set.parity)) break;
        scores(0, k[0]);
        if (n > 1 && w.ok) scores(1, k[1]);
        if (!w.wait1(&b->acc_empty[set.i], set.parity ^ 1u)) break;
        for (int j = 0; j < n; ++j) {
          const int at = buf.i ^ (j & 1);
          if (!w.wait1(&b->ds_ready[at], (ds_phase >> at) & 1u)) break;
          ds_phase ^= 1u << at;
          if (kFew && j == narrow) product_ts<DP, 4, 0, 2>(cAcc + DP * set.i, cS + 128 * at, tile(k[0]), j == 0);
          else product_ts<DP, 4>(cAcc + DP * set.i, cS + 128 * at, tile(k[0]), j == 0);
          tc::mma_commit(&b->empty[k[0]]);
          k[0] = k[1];
          if (j + 2 < n) {
            scores(j + 2, k[1]);
            if (!w.ok) break;
          }
        }
        buf.i ^= n & 1;
        if (w.ok) tc::mma_commit(&b->acc_full[set.i]);
      }
      w.drain(0);
    }
    __syncwarp();
    w.ok = __all_sync(0xffffffffu, w.ok);
  } else if (warp == kMmaB) {
    // ---------------- MMA (one thread): dP(j) ----------------
    if (tc::elect_one()) {
      uint32_t free_phase = 0;
      for (int64_t r = 0; w.ok && get_item(item(r), it); ++r, set.next()) {
        const uint32_t o = tc::su32(own + (2 * set.i + 1) * kTileBytes);
        if (!w.wait1(&b->own_full[set.i][1], set.parity)) break;
        const int all = keys(it).count(it.blk), narrow = kFew ? keys(it).narrow(a.sinks) : -1;
        for (int n = all; n > 0; --n) {
          w.next();
          const int v = w.take();
          // free once the last block's dP has been read
          if (!w.wait1(&b->dp_free, free_phase ^ 1u)) break;
          free_phase ^= 1u;
          if (kFew && all - n == narrow) product_ss<DP, 0, DP / 16, 32>(cP, o, tc::su32(ring + v * kTileBytes));
          else product_ss<DP>(cP, o, tc::su32(ring + v * kTileBytes));
          tc::mma_commit(&b->dp_full);
          tc::mma_commit(&b->empty[v]);
          if (n == 1) tc::mma_commit(&b->own_empty[set.i]);
        }
      }
      w.drain(1);
    }
    __syncwarp();
    w.ok = __all_sync(0xffffffffu, w.ok);
  } else if (warp == kStats) {
    // ---------------- sequence ends: K's rows past them become zeros ----------------
    uint32_t seen = 0;
    int next = 0;                                                 // ring slot of the item's first tile
    for (int64_t r = 0; w.ok && get_item(item(r), it); ++r) {
      const int rows = it.len - kTile * it.blk, n = keys(it).count(it.blk);
      if (rows < kTile) w.end_tile(ring, kTileBytes, (next + 2 * (n - 1)) % kSlots, seen, rows, kChunks);
      next = (next + 2 * n) % kSlots;
    }
  } else {
    // ---------------- softmax ----------------
    const int part = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint64_t c2 = tc::pack2(a.scale, a.scale), log2e2 = tc::pack2(kLog2e, kLog2e);
    uint32_t dp_phase = 0;
    for (int64_t r = 0; w.ok && get_item(item(r), it); ++r, set.next()) {
      const int64_t at = it.start + static_cast<int64_t>(kTile) * it.blk;
      const int rows = it.len - kTile * it.blk;
      const bool in = row < rows;
      const int64_t si = static_cast<int64_t>(it.head) * a.tokens + at + row;
      const float ls = in ? -a.lse[si] : -INFINITY, de = in ? a.delta[si] : 0.f;
      const uint64_t ls2 = tc::pack2(ls, ls);
      const KeySpan span = keys(it);
      const int narrow = kFew ? span.narrow(a.sinks) : -1;
      for (int j = span.first(); j <= it.blk; j = WIN ? span.up(j) : j + 1, buf.next()) {
        if (kFew && j == narrow && part) {                         // no columns of this part are seen
          if (!w.wait(&b->s_full[buf.i], buf.parity) || !w.wait(&b->dp_full, dp_phase)) break;
          dp_phase ^= 1u;
          w.arrive(&b->dp_free);
          w.arrive(&b->ds_ready[buf.i]);
          continue;
        }
        const uint32_t mS = cS + 128 * buf.i + lanes + 32 * part, mP = cP + lanes + 32 * part;
        if (!w.wait(&b->s_full[buf.i], buf.parity)) break;
        float p[32];
        uint32_t pk[16];
        uint32_t x[32];
        tc::tmem_ld32(mS, x);
        tc::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float y0, y1;
          tc::unpack2(tc::mul2(tc::fma2(tc::pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, ls2), log2e2), y0, y1);
          p[e] = tc::exp2_fast(y0);
          p[e + 1] = tc::exp2_fast(y1);
        }
        if (!w.wait(&b->dp_full, dp_phase)) break;
        dp_phase ^= 1u;
        tc::tmem_ld32(mP, x);
        tc::tmem_ld_wait();
        w.arrive(&b->dp_free);
#pragma unroll
        for (int e = 0; e < 32; e += 2)
          pk[e / 2] = pack_bf16x2(p[e] * (__uint_as_float(x[e]) - de), p[e + 1] * (__uint_as_float(x[e + 1]) - de));
        if constexpr (WIN) {
          if (kTile * (it.blk - j + 1) > a.window || j == it.blk) {
            const int up = kTile * (it.blk - j) - 32 * part;
            uint32_t hide = hidden_bits(up + row, up + row - a.window + 1, a.sinks - kTile * j - 32 * part);
            if (sees_itself(a.window, a.sinks)) hide = ~0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if (hide >> (2 * e) & 1u) pk[e] &= 0xFFFF0000u;
              if (hide >> (2 * e + 1) & 1u) pk[e] &= 0x0000FFFFu;
            }
          }
        } else if (j == it.blk) {   // query `row` sees keys .. row
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (32 * part + 2 * e > row) pk[e] &= 0xFFFF0000u;
            if (32 * part + 2 * e + 1 > row) pk[e] &= 0x0000FFFFu;
          }
        }
        tc::tmem_put16(mS, pk);
        tc::tmem_st_drain();
        w.arrive(&b->ds_ready[buf.i]);
      }
      if (!w.wait(&b->acc_full[set.i], set.parity)) break;
      store_acc<DP>(a.dq, cAcc + DP * set.i + lanes, at, rows, it.head, warp, a.scale, a.dim, lane);
      w.arrive(&b->acc_empty[set.i]);
    }
  }
  finish(w, a.flags);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dkdv_tc(const __grid_constant__ BwdArgs f) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint32_t tmem;
  walk_dkdv<DP, false>(f, smem, tmem);
  free_tmem(tmem);
}
template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dq_tc(const __grid_constant__ BwdArgs f) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint32_t tmem;
  walk_dq<DP, kWhole, true>(f, smem, tmem);
  free_tmem(tmem);
}

// With a window both walks run in one launch, one after the other in each CTA and
// dealt out together: items are short, so that a second launch's start and the
// walks' uneven ends show.  (Without one the two launches of before remain.)
template <int DP, int KIND>
__global__ void __launch_bounds__(kThreads, 1) k_attn_bwd_tc(const __grid_constant__ BwdArgs f) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint32_t tmem;
  if (walk_dkdv<DP, true>(f, smem, tmem)) {
    // tiles whose tails were zeroed through the generic proxy are loaded over
    tc::fence_smem_async();
    __syncthreads();
    walk_dq<DP, KIND, false>(f, smem, tmem);
  }
  free_tmem(tmem);
}

template <auto kernel>
cudaError_t launch(const BwdArgs& f, int64_t items, size_t smem, cudaStream_t s) {
  const cudaError_t e = allow_smem<kernel>(smem);
  if (e) return e;
  kernel<<<walk_grid(items), kThreads, smem, s>>>(f);
  return cudaGetLastError();
}

template <int DP>
cudaError_t both(const BwdArgs& f, cudaStream_t s) {
  const int64_t by_key = static_cast<int64_t>(f.a.n_keys) * f.a.kv_heads, by_query = static_cast<int64_t>(f.a.n_blocks) * f.a.heads;
  switch (window_kind(f.a)) {
    case kWindow: return launch<k_attn_bwd_tc<DP, kWindow>>(f, std::max(by_key, by_query), Bwd<DP>::kSmem, s);
    case kWindowNarrow: return launch<k_attn_bwd_tc<DP, kWindowNarrow>>(f, std::max(by_key, by_query), Bwd<DP>::kSmem, s);
    default: break;
  }
  const cudaError_t e = launch<k_attn_dkdv_tc<DP>>(f, by_key, Bwd<DP>::kSmem, s);
  return e ? e : launch<k_attn_dq_tc<DP>>(f, by_query, Bwd<DP>::kSmem, s);
}

}  // namespace

cudaError_t launch_attn_backward_tc(const AttnArgs& a, cudaStream_t s, std::string* err) {
  BwdArgs f;
  f.a = a;
  if (!rows_map(&f.q, a.q, a.tokens, a.heads, a.dim, err) || !rows_map(&f.k, a.k, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.v, a.v, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.dout, a.dout, a.tokens, a.heads, a.dim, err))
    return cudaErrorInvalidValue;
  return a.dim <= 64 ? both<64>(f, s) : both<128>(f, s);
}

}  // namespace normpre
