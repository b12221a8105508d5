// Packed causal attention, forward, bf16 on tcgen05 tensor cores.
//
// For a tile of 128 query rows, over the sequence's key blocks of 128 from the
// diagonal one down to the first:
//   S = Q K^T;  m' = max(m, max_j S);  P = exp2(c (S - m'));
//   l = l exp2(c (m - m')) + sum_j P;  O = O exp2(c (m - m')) + P V
// and O / l at the end, with c = scale log2(e).  The diagonal block comes
// first: every row sees itself there, so m is finite from then on, and no
// other block needs a mask (a sequence's end lies in its last diagonal block).
//
// One CTA per SM walks the work list.  An item is two query tiles that read
// the same keys: two heads of a group, or with an odd group two neighbouring
// tiles of one head.  Each has its own 128 columns of scores and its output
// accumulator in TMEM (2 * 128 + 2 * 128 = all 512 columns at head_dim 128),
// and its own four softmax warps, one thread per row, so that row statistics
// need no shuffles; while one tile's warps take exponentials, the tensor cores
// work on the other tile.  P goes back to TMEM as bf16 over the scores it came
// from and is the A operand of P V.  Q stays in shared memory for the item; K
// and V tiles pass through one ring that a TMA warp fills.
//
// The running maximum is only raised when it would grow by more than 2^8
// (O and l then are rescaled by the softmax warps themselves): P stays below
// 2^8 relative to the row's maximum, which bf16 and the fp32 sums hold as
// precisely, and the rescale, which has to wait for P V, is rare.
//
// S - m' is formed before the scale: near the maximum it is exact however large
// the scores, while c S - c m' would carry the rounding of c m' (0.002 in the
// exponent at scores of 3e4).  That addition and P's conversion, which shares the
// exponentials' pipe, cost 3 % against one FMA and a cut.
//
// Roundings to bf16: P once (the MMA operand; l sums the unrounded values) and
// the output once.
//
// What bounds it: a step (two tiles x 128 keys) costs the tensor cores 2 x 2 x
// 512 cycles and a scheduler's two softmax warps 2 x 128 exponentials of 4
// cycles beside their scaling, sums and conversions, about as much; the two stay within
// a fifth of each other.  Under load the clock falls with the power limit.
// 16384 tokens, 16 / 8 heads of 128: 0.62 ms alone (1760 TFLOP/s), 0.70 ms in a
// loop; 8192 tokens in seven sequences 0.074 ms with everything in L2 (1320
// TFLOP/s: the CTAs' last items), 0.090 to 0.098 ms otherwise.
#include "attn_tc.cuh"

namespace normpre {
namespace {

constexpr int kThreads = 384;   // softmax 2 x 4 warps, TMA, MMA of tile 0, sequence ends, MMA of tile 1
constexpr float kGrow = 8.f;    // log2 of the growth that raises the maximum

template <int DP> struct Fwd {
  static constexpr int kChunks = DP / 64;
  static constexpr int kTileBytes = kChunks * kChunk;
  static constexpr int kSlots = DP == 128 ? 5 : 10;    // K / V ring
  static constexpr int kAcc = DP == 128 ? 1 : 2;       // output accumulators of a tile
  static constexpr size_t kSmem = (2 + kSlots) * kTileBytes + 2048;
};

struct FwdArgs {
  AttnArgs a;
  CUtensorMap q, k, v;
  const AttnBlock* list;
  int n_list;      // blocks, or pairs of blocks
  int pair_heads;  // the two tiles are two heads of a group
};

template <int kSlots> struct Bars {
  // raw: a tile that ends its sequence lands here first; once its tail is
  // zeroed it counts as full
  uint64_t full[kSlots], empty[kSlots], raw[kSlots];
  uint64_t q_full[2], q_empty[2], s_full[2], p_ready[2][2], pv_done[2], o_empty[2][2], turn[2], drain[2];
  uint32_t tmem;
  int abort;
  uint32_t issued[kSlots], raw_issued[kSlots], q_issued[2];   // last parity + 1
};

struct Item {
  int64_t start;   // the sequence's first row
  int len;
  int top;         // the topmost block of keys
  int blk0, blk1;  // the tiles' block in the sequence, -1: no tile
  int head0, head1;
  int kvh;
};

constexpr int kCached = 64;

__device__ __forceinline__ ItemRef find_item(const FwdArgs& f, int64_t r) {
  return list_item(f.a, f.list, f.n_list, f.a.walk_fwd, f.pair_heads ? f.a.heads / 2 : f.a.heads, r);
}

__device__ __forceinline__ bool get_item(const FwdArgs& f, const ItemRef* cached, int64_t r, Item& it) {
  const ItemRef b = r < kCached ? cached[r] : find_item(f, r);
  if (b.blk < 0) return false;
  it.start = b.start;
  it.len = b.len;
  it.blk0 = b.blk;
  if (f.pair_heads) {
    it.blk1 = b.blk;
    it.head0 = 2 * b.head;
    it.head1 = 2 * b.head + 1;
  } else {
    it.blk1 = (b.blk + 1) * kTile < b.len ? b.blk + 1 : -1;
    it.head0 = it.head1 = b.head;
  }
  it.top = max(it.blk0, it.blk1);
  it.kvh = it.head0 / f.a.group;
  return true;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_fwd_tc(const __grid_constant__ FwdArgs f) {
  using F = Fwd<DP>;
  constexpr int kSlots = F::kSlots, kTileBytes = F::kTileBytes, kChunks = F::kChunks, kAcc = F::kAcc;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sQ = smem;                          // [2]
  uint8_t* ring = smem + 2 * kTileBytes;       // [kSlots]
  Bars<kSlots>* b = reinterpret_cast<Bars<kSlots>*>(ring + kSlots * kTileBytes);
  static_assert(sizeof(Bars<kSlots>) <= 1024, "barriers");
  ItemRef* items = reinterpret_cast<ItemRef*>(reinterpret_cast<uint8_t*>(b) + 1024);   // [kCached]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      tc::mbar_init(&b->full[i], 1);
      tc::mbar_init(&b->empty[i], 2);          // both tiles' MMAs
      tc::mbar_init(&b->raw[i], 1);
      b->issued[i] = b->raw_issued[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&b->q_full[i], 1);
      tc::mbar_init(&b->q_empty[i], 1);
      tc::mbar_init(&b->s_full[i], 1);
      tc::mbar_init(&b->p_ready[i][0], 4);
      tc::mbar_init(&b->p_ready[i][1], 4);
      tc::mbar_init(&b->pv_done[i], 1);
      tc::mbar_init(&b->o_empty[i][0], 4);
      tc::mbar_init(&b->o_empty[i][1], 4);
      tc::mbar_init(&b->turn[i], 1);
      tc::mbar_init(&b->drain[i], 1);
      b->q_issued[i] = 0;
    }
    b->abort = 0;
    tc::fence_barrier_init();
    tc::prefetch_map(&f.q);
    tc::prefetch_map(&f.k);
    tc::prefetch_map(&f.v);
  }
  if (threadIdx.x >= 64 && threadIdx.x < 64 + kCached) items[threadIdx.x - 64] = find_item(f, threadIdx.x - 64);
  if (warp == 9) {
    tc::tmem_alloc(&b->tmem, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = b->tmem;
  auto s_col = [&](int s) { return tmem + static_cast<uint32_t>(128 * s); };
  auto o_col = [&](int s, int acc) { return tmem + static_cast<uint32_t>(256 + DP * (kAcc * s + acc)); };
  bool ok = true;
  Item it;

  // of the launch's 384 * 168 registers: 256 * 200 + 128 * 96
  if (warp >= 8) {
    tc::regs_fewer<96>();
    if (warp == 8) {
      // ---------------- TMA (one thread), then the rows past the sequences ----------------
      if (tc::elect_one()) {
        int slot = 0;
        uint32_t phase = 0, q_phase[2] = {0, 0};
        const bool stall = f.a.test_stall && blockIdx.x == 0;   // nothing is loaded: the others' waits run out
        auto load = [&](const CUtensorMap* map, int64_t row, int head, bool tail) {
          ok = ok && tc::mbar_wait(&b->empty[slot], phase ^ 1u, &b->abort);
          if (!ok) return;
          uint64_t* bar = tail ? &b->raw[slot] : &b->full[slot];
          tc::mbar_expect_tx(bar, kTileBytes);
          if (tail) ++b->raw_issued[slot];
          else b->issued[slot] = phase + 1;
          load_rows(ring + slot * kTileBytes, map, bar, row, head, kChunks);
          if (++slot == kSlots) { slot = 0; phase ^= 1u; }
        };
        for (int64_t r = 0; ok && !stall && get_item(f, items, r, it); ++r) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const int blk = s ? it.blk1 : it.blk0;
            if (blk >= 0) {
              ok = ok && tc::mbar_wait(&b->q_empty[s], q_phase[s] ^ 1u, &b->abort);
              if (!ok) break;
              tc::mbar_expect_tx(&b->q_full[s], kTileBytes);
              b->q_issued[s] = q_phase[s] + 1;
              load_rows(sQ + s * kTileBytes, &f.q, &b->q_full[s], it.start + kTile * blk, s ? it.head1 : it.head0, kChunks);
              q_phase[s] ^= 1u;
            }
            if (s == 0) load(&f.k, it.start + static_cast<int64_t>(kTile) * it.top, it.kvh, false);
          }
          for (int j = it.top; j >= 0 && ok; --j) {
            const int64_t row = it.start + static_cast<int64_t>(kTile) * j;
            load(&f.v, row, it.kvh, kTile * (j + 1) > it.len);
            if (j > 0) load(&f.k, row - kTile, it.kvh, false);
          }
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      zero_padding(f.a, f.a.o, f.a.heads, blockIdx.x, gridDim.x, lane);
      const int64_t pad = f.a.tokens - f.a.total;
      for (int64_t i = 32 * static_cast<int64_t>(blockIdx.x) + lane; i < pad * f.a.heads; i += 32 * static_cast<int64_t>(gridDim.x))
        f.a.lse[(i / pad) * f.a.tokens + f.a.total + i % pad] = -INFINITY;
    } else if (warp == 10) {
      // ---------------- sequence ends: V's rows past them become zeros ----------------
      int next = 0;             // ring slot of the item's first tile
      uint32_t seen = 0;        // per slot, parity of its raw barrier
      for (int64_t r = 0; ok && get_item(f, items, r, it); ++r) {
        const int rows = it.len - kTile * it.top;
        if (rows < kTile) {
          const int slot = next + 1 == kSlots ? 0 : next + 1;
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&b->raw[slot], (seen >> slot) & 1u, &b->abort));
          seen ^= 1u << slot;
          if (!ok) break;
          zero_tail(ring + slot * kTileBytes, rows, kChunks, lane);
          if (lane == 0) tc::mbar_arrive(&b->full[slot]);
        }
        next = (next + 2 * (it.top + 1)) % kSlots;
      }
    } else {
      // ---------------- MMA of one tile (one thread) ----------------
      // A thread's MMAs run almost as it issues them, so that its waits would
      // idle the tensor cores: the two tiles are issued by two warps.  They
      // take turns, a tile's P V and next scores at a time, which keeps one
      // tile's softmax beside the other's products (left alone they fall into
      // step).  The turn passes before the last MMAs, to cover its latency.
      const int s = warp == 11;
      if (tc::elect_one()) {
        int slot = 0, acc = 0;
        uint32_t phase = 0, q_phase = 0, p_phase = 0, o_phase = 0, t_phase = s ? 0 : 1;
        const uint32_t sq = tc::su32(sQ + s * kTileBytes);
        auto tile = [&](int t) { return tc::su32(ring + t * kTileBytes); };
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          ok = ok && tc::mbar_wait(bar, parity, &b->abort);
          tc::fence_after();
          return ok;
        };
        auto my_turn = [&]() {
          wait(&b->turn[s], t_phase);
          t_phase ^= 1u;
          return ok;
        };
        auto pass_turn = [&]() { tc::mbar_arrive(&b->turn[s ^ 1]); };
        // next tile of the ring, once it has arrived
        auto take = [&]() {
          const int t = slot;
          wait(&b->full[t], phase);
          if (++slot == kSlots) { slot = 0; phase ^= 1u; }
          return t;
        };
        // S = Q K^T, and the turn is over
        auto scores = [&](int k) {
          product_ss<DP, 0, DP / 32>(s_col(s), sq, tile(k));
          pass_turn();
          product_ss<DP, DP / 32, DP / 16>(s_col(s), sq, tile(k));
          tc::mma_commit(&b->s_full[s]);
          tc::mma_commit(&b->empty[k]);
        };
        for (int64_t r = 0; ok && get_item(f, items, r, it); ++r) {
          const int blk = s ? it.blk1 : it.blk0;
          int k = take();
          if (blk >= 0 && !wait(&b->q_full[s], q_phase)) break;
          if (blk >= 0) q_phase ^= 1u;
          if (!ok || !my_turn()) break;
          if (it.top == blk) {
            scores(k);
            if (blk == 0) tc::mma_commit(&b->q_empty[s]);
          } else {
            tc::mbar_arrive(&b->empty[k]);
            pass_turn();
          }
          for (int j = it.top; j >= 0; --j) {
            const int v = take();
            if (j > 0) k = take();
            if (!ok) break;
            const uint32_t o = o_col(s, acc), p = s_col(s);
            if (j <= blk) {
              if (j == blk) {
                if (!wait(&b->o_empty[s][acc], ((o_phase >> acc) & 1u) ^ 1u)) break;
                o_phase ^= 1u << acc;
              }
              if (!my_turn() || !wait(&b->p_ready[s][0], p_phase)) break;
              product_ts<DP, 1, 0, 6>(o, p, tile(v), j == blk);
              if (!wait(&b->p_ready[s][1], p_phase)) break;
              product_ts<DP, 1, 6, 8>(o, p, tile(v), false);
              p_phase ^= 1u;
              tc::mma_commit(&b->pv_done[s]);
              tc::mma_commit(&b->empty[v]);
            } else {
              if (!my_turn()) break;
              tc::mbar_arrive(&b->empty[v]);
            }
            if (j > 0 && j - 1 <= blk) {
              scores(k);
              if (j == 1) tc::mma_commit(&b->q_empty[s]);
            } else {
              if (j > 0) tc::mbar_arrive(&b->empty[k]);
              pass_turn();
            }
          }
          if (blk >= 0 && kAcc == 2) acc ^= 1;
        }
        // every MMA issued has completed once `drain` fires
        tc::mma_commit(&b->drain[s]);
        int never = 0;
        tc::mbar_wait(&b->drain[s], 0, &never);
      }
      __syncwarp();
      ok = __all_sync(0xffffffffu, ok);
    }
  } else {
    // ---------------- softmax: warps 0-3 tile 0, warps 4-7 tile 1 ----------------
    tc::regs_more<200>();
    const int s = warp >> 2, q4 = warp & 3;
    const int row = 32 * q4 + lane;                       // of the tile
    const uint32_t lanes = static_cast<uint32_t>(q4 * 32) << 16;
    const uint32_t sc = s_col(s) + lanes;
    const float c = f.a.scale_log2;
    const uint64_t c2 = tc::pack2(c, c);
    uint32_t s_phase = 0, pv = 0;                         // products P V before this block
    int acc = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, &b->abort));
      tc::fence_after();
      return ok;
    };
    for (int64_t r = 0; ok && get_item(f, items, r, it); ++r) {
      const int blk = s ? it.blk1 : it.blk0;
      if (blk < 0) continue;
      const uint32_t oc = o_col(s, acc) + lanes;
      float m = -INFINITY, l = 0.f;
      for (int j = blk; j >= 0; --j) {
        if (!wait(&b->s_full[s], s_phase)) break;
        s_phase ^= 1u;
        uint32_t x[32];                 // a quarter of the row's scores
        uint32_t p[48];
        uint64_t sum[2] = {0, 0};
        float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto load = [&](int q) {
          tc::tmem_ld32(sc + 32 * q, x);
          tc::tmem_ld_wait();
        };
        auto mask = [&](int q) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (32 * q + i > row) x[i] = 0xFF800000u;
        };
        auto compare = [&]() {
#pragma unroll
          for (int i = 0; i < 32; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              t[e] = fmaxf(fmaxf(t[e], __uint_as_float(x[i + 2 * e])), __uint_as_float(x[i + 2 * e + 1]));
        };
        auto top = [&]() { return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])); };
        // the quarter's exponentials with the running maximum, as P and into the sum
        auto exps = [&](uint32_t* to) {
          const uint64_t m2 = tc::pack2(-m, -m);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float lo, hi;
            tc::unpack2(tc::mul2(tc::add2(tc::pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), m2), c2), lo, hi);
            lo = tc::exp2_fast(lo);
            hi = tc::exp2_fast(hi);
            sum[i & 1] = tc::add2(sum[i & 1], tc::pack2(lo, hi));
            to[i] = pack_bf16x2(lo, hi);
          }
        };
        auto release = [&](int part) {
          tc::tmem_st_drain();
          tc::fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&b->p_ready[s][part]);
        };
        // Three quarters of P go first: the products on them cover the rest.
        if (j == blk) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            load(q);
            mask(q);
            compare();
          }
          m = top();
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            load(q);
            mask(q);
            exps(p + 16 * q);
          }
          load(3);
          mask(3);
        } else {
          // A later block's maximum is needed only to see whether the running
          // one must be raised, which is rare: its comparisons run in the
          // shadow of the exponentials.
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            load(q);
            compare();
            exps(p + 16 * q);
          }
          load(3);
          compare();
          const float up = fmaxf(m, top());
          if (__any_sync(0xffffffffu, (up - m) * c > kGrow)) {
            const float keep = tc::exp2_fast((m - up) * c);
            m = up;
            l *= keep;
            if (!wait(&b->pv_done[s], (pv - 1) & 1u)) break;
#pragma unroll 1
            for (int i = 0; i < DP; i += 32) {
              uint32_t o[32];
              tc::tmem_ld32(oc + i, o);
              tc::tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
              tc::tmem_put32(oc + i, o);
            }
            sum[0] = sum[1] = 0;
#pragma unroll
            for (int q = 0; q < 3; ++q) {
              load(q);
              exps(p + 16 * q);
            }
            load(3);
          }
        }
        tc::tmem_put32(sc, p);
        tc::tmem_put16(sc + 32, p + 32);
        release(0);
        exps(p);
        tc::tmem_put16(sc + 48, p);
        release(1);
        float lo, hi;
        tc::unpack2(tc::add2(sum[0], sum[1]), lo, hi);
        l += lo + hi;
        ++pv;
      }
      if (!ok || !wait(&b->pv_done[s], (pv - 1) & 1u)) break;
      const float inv = 1.f / l;
      const int rows = it.len - kTile * blk;              // of the tile
      const int64_t at = it.start + static_cast<int64_t>(kTile) * blk;
      const int head = s ? it.head1 : it.head0;
      bf16* out = static_cast<bf16*>(f.a.o.p) + at * f.a.o.ts + head * f.a.o.hs;
#pragma unroll 1
      for (int d = 0; d < DP; d += 32) {
        uint32_t o[32];
        tc::tmem_ld32(oc + d, o);
        tc::tmem_ld_wait();
        store_rows<32>(out, f.a.o.ts, o, inv, 32 * q4, rows, d, f.a.dim, lane);
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&b->o_empty[s][acc]);
      if (kAcc == 2) acc ^= 1;
      if (row < rows)
        f.a.lse[static_cast<int64_t>(head) * f.a.tokens + at + row] = fmaf(m, f.a.scale, log2f(l) * 0.6931471805599453f);
    }
  }
  if (!ok && lane == 0) {
    *static_cast<volatile int*>(&b->abort) = 1;
    raise_host_flag(f.a.flags, kFlagTimeout);
  }

  __syncthreads();
  if (threadIdx.x == 0 && *static_cast<volatile int*>(&b->abort)) {
    // let every TMA copy still in flight land before the CTA exits
    int never = 0;
    for (int i = 0; i < kSlots; ++i) {
      if (b->issued[i]) tc::mbar_wait(&b->full[i], b->issued[i] - 1, &never);
      if (b->raw_issued[i]) tc::mbar_wait(&b->raw[i], (b->raw_issued[i] - 1) & 1u, &never);
    }
    for (int i = 0; i < 2; ++i)
      if (b->q_issued[i]) tc::mbar_wait(&b->q_full[i], b->q_issued[i] - 1, &never);
  }
  __syncthreads();
  if (warp == 9) {
    tc::fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
}

}  // namespace

template <int DP>
static cudaError_t launch(const FwdArgs& f, int64_t items, cudaStream_t s) {
  const cudaError_t e = allow_smem<k_attn_fwd_tc<DP>>(Fwd<DP>::kSmem);
  if (e) return e;
  k_attn_fwd_tc<DP><<<walk_grid(items), kThreads, Fwd<DP>::kSmem, s>>>(f);
  return cudaGetLastError();
}

cudaError_t launch_attn_forward_tc(const AttnArgs& a, cudaStream_t s, std::string* err) {
  FwdArgs f;
  f.a = a;
  if (!rows_map(&f.q, a.q, a.tokens, a.heads, a.dim, err) || !rows_map(&f.k, a.k, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.v, a.v, a.tokens, a.kv_heads, a.dim, err))
    return cudaErrorInvalidValue;
  f.pair_heads = attn_pair_heads(a.group);
  f.list = f.pair_heads ? a.by_query : a.by_pair;
  f.n_list = f.pair_heads ? a.n_blocks : a.n_pairs;
  const int64_t items = static_cast<int64_t>(f.n_list) * (f.pair_heads ? a.heads / 2 : a.heads);
  return a.dim <= 64 ? launch<64>(f, items, s) : launch<128>(f, items, s);
}

}  // namespace normpre
