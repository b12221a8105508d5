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
// Roundings to bf16: P once (the MMA operand; l sums the unrounded values) and
// the output once.
#include "attn_tc.cuh"

namespace normpre {
namespace {

constexpr int kThreads = 384;   // softmax 2 x 4 warps, TMA, MMA, two for the padding rows
constexpr float kGrow = 8.f;    // log2 of the growth that raises the maximum

template <int DP> struct Fwd {
  static constexpr int kChunks = DP / 64;
  static constexpr int kTileBytes = kChunks * kChunk;
  static constexpr int kSlots = DP == 128 ? 5 : 10;    // K / V ring
  static constexpr size_t kSmem = 1024 + (2 + kSlots) * kTileBytes + 512;
};

struct FwdArgs {
  AttnArgs a;
  CUtensorMap q, k, v;
  const AttnBlock* list;
  int n_list;      // blocks, or pairs of blocks
  int pair_heads;  // the two tiles are two heads of a group
};

struct Item {
  int64_t start;   // the sequence's first row
  int len;
  int blk[2];      // the tiles' block in the sequence, -1: no tile
  int head[2];
  int kvh;
};

__device__ __forceinline__ bool get_item(const FwdArgs& f, int64_t r, Item& it) {
  const int per = f.pair_heads ? f.a.heads / 2 : f.a.heads;
  const int64_t i = walk_item(r);
  if (i >= static_cast<int64_t>(f.n_list) * per) return false;
  const AttnBlock b = f.list[i / per];
  const int h = static_cast<int>(i % per);
  it.start = b.start;
  it.len = b.len;
  if (f.pair_heads) {
    it.blk[0] = it.blk[1] = b.blk;
    it.head[0] = 2 * h;
    it.head[1] = 2 * h + 1;
  } else {
    it.blk[0] = b.blk;
    it.blk[1] = (b.blk + 1) * kTile < b.len ? b.blk + 1 : -1;
    it.head[0] = it.head[1] = h;
  }
  it.kvh = it.head[0] / f.a.group;
  return true;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attn_fwd_tc(const __grid_constant__ FwdArgs f) {
  using F = Fwd<DP>;
  constexpr int kSlots = F::kSlots, kTileBytes = F::kTileBytes, kChunks = F::kChunks;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                          // [2]
  uint8_t* sKV = smem + 2 * kTileBytes;        // [kSlots]
  uint64_t* kv_full = reinterpret_cast<uint64_t*>(sKV + kSlots * kTileBytes);
  uint64_t* kv_empty = kv_full + kSlots;
  uint64_t* q_full = kv_empty + kSlots;        // [2], as the following ones
  uint64_t* q_empty = q_full + 2;
  uint64_t* s_full = q_empty + 2;
  uint64_t* p_ready = s_full + 2;
  uint64_t* pv_done = p_ready + 2;
  uint64_t* o_empty = pv_done + 2;
  uint64_t* drain = o_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* issued = tmem_slot + 2;            // [kSlots + 2]: last parity + 1 of kv_full and q_full

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      tc::mbar_init(&kv_full[i], 1);
      tc::mbar_init(&kv_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&q_full[i], 1);
      tc::mbar_init(&q_empty[i], 1);
      tc::mbar_init(&s_full[i], 1);
      tc::mbar_init(&p_ready[i], 4);
      tc::mbar_init(&pv_done[i], 1);
      tc::mbar_init(&o_empty[i], 4);
    }
    tc::mbar_init(drain, 1);
    for (int i = 0; i < kSlots + 2; ++i) issued[i] = 0;
    *abort_flag = 0;
    tc::fence_barrier_init();
    tc::prefetch_map(&f.q);
    tc::prefetch_map(&f.k);
    tc::prefetch_map(&f.v);
  }
  if (warp == 9) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = *tmem_slot;
  auto s_col = [&](int s) { return tmem + static_cast<uint32_t>(128 * s); };
  auto o_col = [&](int s) { return tmem + static_cast<uint32_t>(256 + DP * s); };
  bool ok = true;
  Item it;

  // of the launch's 384 * 168 registers: 256 * 200 + 128 * 96
  if (warp >= 8) {
    tc::regs_fewer<96>();
    if (warp == 8) {
      // ---------------- TMA ----------------
      int slot = 0;
      uint32_t phase = 0, q_phase[2] = {0, 0};
      auto load_kv = [&](const CUtensorMap* map, int64_t row, int head) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&kv_empty[slot], phase ^ 1u, abort_flag));
        if (!ok) return;
        if (lane == 0) {
          tc::mbar_expect_tx(&kv_full[slot], kTileBytes);
          issued[slot] = phase + 1;
          load_rows(sKV + slot * kTileBytes, map, &kv_full[slot], row, head, kChunks);
        }
        __syncwarp();
        if (++slot == kSlots) { slot = 0; phase ^= 1u; }
      };
      for (int64_t r = 0; ok && get_item(f, r, it); ++r) {
        for (int s = 0; s < 2 && ok; ++s) {
          if (it.blk[s] < 0) continue;
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&q_empty[s], q_phase[s] ^ 1u, abort_flag));
          if (!ok) break;
          if (lane == 0) {
            tc::mbar_expect_tx(&q_full[s], kTileBytes);
            issued[kSlots + s] = q_phase[s] + 1;
            load_rows(sQ + s * kTileBytes, &f.q, &q_full[s], it.start + kTile * it.blk[s], it.head[s], kChunks);
          }
          __syncwarp();
          q_phase[s] ^= 1u;
          if (s == 0) load_kv(&f.k, it.start + static_cast<int64_t>(kTile) * max(it.blk[0], it.blk[1]), it.kvh);
        }
        for (int j = max(it.blk[0], it.blk[1]); j >= 0 && ok; --j) {
          const int64_t row = it.start + static_cast<int64_t>(kTile) * j;
          load_kv(&f.v, row, it.kvh);
          if (j > 0 && ok) load_kv(&f.k, row - kTile, it.kvh);
        }
      }
      if (!ok && lane == 0) { *abort_flag = 1; raise_flag(f.a.flags, kFlagTimeout); }
    } else if (warp == 9) {
      // ---------------- MMA ----------------
      int slot = 0;
      uint32_t phase = 0;
      uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0}, o_phase[2] = {0, 0};
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort_flag));
        tc::fence_after();
        return ok;
      };
      // slot of the next tile of the ring, once it has arrived
      auto take_kv = [&]() {
        const int s = slot;
        wait(&kv_full[s], phase);
        if (++slot == kSlots) { slot = 0; phase ^= 1u; }
        return s;
      };
      auto scores = [&](int s, int kslot) {   // S_s = Q_s K^T
        if (tc::elect_one()) {
          product_ss<DP>(s_col(s), tc::su32(sQ + s * kTileBytes), tc::su32(sKV + kslot * kTileBytes));
          tc::mma_commit(&s_full[s]);
        }
        __syncwarp();
      };
      for (int64_t r = 0; ok && get_item(f, r, it); ++r) {
        const int top = max(it.blk[0], it.blk[1]);
        const int krows = min(kTile, it.len - kTile * top);   // keys of the topmost block
        int kslot = take_kv();
        for (int s = 0; s < 2 && ok; ++s) {
          if (it.blk[s] < 0) continue;
          if (!wait(&q_full[s], q_phase[s])) break;
          q_phase[s] ^= 1u;
          if (it.blk[s] == top) scores(s, kslot);
        }
        if (!ok) break;
        if (tc::elect_one()) {
          tc::mma_commit(&kv_empty[kslot]);
          if (top == 0)
            for (int s = 0; s < 2; ++s)
              if (it.blk[s] >= 0) tc::mma_commit(&q_empty[s]);
        }
        __syncwarp();
        for (int j = top; j >= 0 && ok; --j) {
          const int vslot = take_kv();
          if (!ok) break;
          if (j == top && krows < kTile) zero_tail(sKV + vslot * kTileBytes, krows, kChunks, lane);
          if (j > 0) {
            kslot = take_kv();
            if (!ok) break;
          }
          for (int s = 0; s < 2 && ok; ++s) {
            if (j <= it.blk[s]) {
              if (!wait(&p_ready[s], p_phase[s])) break;
              p_phase[s] ^= 1u;
              if (j == it.blk[s]) {
                if (!wait(&o_empty[s], o_phase[s] ^ 1u)) break;
                o_phase[s] ^= 1u;
              }
              if (tc::elect_one()) {   // O_s += P_s V
                product_ts<DP>(o_col(s), s_col(s), tc::su32(sKV + vslot * kTileBytes), j == it.blk[s], 0);
                tc::mma_commit(&pv_done[s]);
              }
              __syncwarp();
            }
            if (j > 0 && j - 1 <= it.blk[s]) scores(s, kslot);
          }
          if (!ok) break;
          if (tc::elect_one()) {
            tc::mma_commit(&kv_empty[vslot]);
            if (j > 0) tc::mma_commit(&kv_empty[kslot]);
            if (j == 1)
              for (int s = 0; s < 2; ++s)
                if (it.blk[s] >= 0) tc::mma_commit(&q_empty[s]);
          }
          __syncwarp();
        }
      }
      if (!ok && lane == 0) { *abort_flag = 1; raise_flag(f.a.flags, kFlagTimeout); }
      // every MMA issued has completed once `drain` fires
      if (tc::elect_one()) {
        tc::mma_commit(drain);
        volatile int never = 0;
        tc::mbar_wait(drain, 0, &never);
      }
      __syncwarp();
    } else if (warp >= 10) {
      // ---------------- rows past the sequences ----------------
      const int64_t w = static_cast<int64_t>(blockIdx.x) * 2 + warp - 10, n = 2 * static_cast<int64_t>(gridDim.x);
      zero_padding(f.a, f.a.o, f.a.heads, w, n, lane);
      const int64_t pad = f.a.tokens - f.a.total;
      for (int64_t i = w * 32 + lane; i < pad * f.a.heads; i += 32 * n)
        f.a.lse[(i / pad) * f.a.tokens + f.a.total + i % pad] = -INFINITY;
    }
  } else {
    // ---------------- softmax: warps 0-3 tile 0, warps 4-7 tile 1 ----------------
    tc::regs_more<200>();
    const int s = warp >> 2, q4 = warp & 3;
    const int row = 32 * q4 + lane;                       // of the tile
    const uint32_t lanes = static_cast<uint32_t>(q4 * 32) << 16;
    const uint32_t sc = s_col(s) + lanes, oc = o_col(s) + lanes;
    const float c = f.a.scale_log2;
    uint32_t s_phase = 0, pv = 0;                         // score tiles seen, products P V before this block
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort_flag));
      tc::fence_after();
      return ok;
    };
    for (int64_t r = 0; ok && get_item(f, r, it); ++r) {
      const int blk = it.blk[s];
      if (blk < 0) continue;
      float m = -INFINITY, l = 0.f;
      for (int j = blk; j >= 0; --j) {
        if (!wait(&s_full[s], s_phase)) break;
        s_phase ^= 1u;
        uint32_t x[128];
#pragma unroll
        for (int i = 0; i < 4; ++i) tc::tmem_ld32(sc + 32 * i, x + 32 * i);
        tc::tmem_ld_wait();
        if (j == blk) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i > row) x[i] = 0xFF800000u;
        }
        float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 128; i += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            t[e] = fmaxf(fmaxf(t[e], __uint_as_float(x[i + 2 * e])), __uint_as_float(x[i + 2 * e + 1]));
        const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        if (j == blk) {
          m = top;
        } else if (__any_sync(0xffffffffu, (top - m) * c > kGrow)) {
          const float up = fmaxf(m, top), keep = tc::exp2_fast((m - up) * c);
          m = up;
          l *= keep;
          if (!wait(&pv_done[s], (pv - 1) & 1u)) break;
#pragma unroll 1
          for (int i = 0; i < DP; i += 32) {
            uint32_t o[32];
            tc::tmem_ld32(oc + i, o);
            tc::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
            tc::tmem_st32(oc + i, o);
          }
        }
        const float mc = -m * c;
        const uint64_t c2 = tc::pack2(c, c), mc2 = tc::pack2(mc, mc);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float lo, hi;
            const int e = 64 * h + 2 * i;
            tc::unpack2(tc::fma2(tc::pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, mc2), lo, hi);
            lo = tc::exp2_fast(lo);
            hi = tc::exp2_fast(hi);
            sum[i & 1] = tc::add2(sum[i & 1], tc::pack2(lo, hi));
            p[i] = pack_bf16x2(lo, hi);
          }
          tc::tmem_st32(sc + 32 * h, p);
        }
        tc::tmem_st_drain();
        tc::fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&p_ready[s]);
        float lo, hi;
        tc::unpack2(tc::add2(sum[0], sum[1]), lo, hi);
        l += lo + hi;
        ++pv;
      }
      if (!ok || !wait(&pv_done[s], (pv - 1) & 1u)) break;
      const float inv = 1.f / l;
      const int i = kTile * blk + row;                    // of the sequence
      const int64_t at = it.start + i;
      bf16* out = static_cast<bf16*>(f.a.o.p) + at * f.a.o.ts + it.head[s] * f.a.o.hs;
#pragma unroll 1
      for (int d = 0; d < DP; d += 32) {
        uint32_t o[32];
        tc::tmem_ld32(oc + d, o);
        tc::tmem_ld_wait();
        if (i < it.len) store_row32(out, o, inv, d, f.a.dim);
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&o_empty[s]);
      if (i < it.len) f.a.lse[static_cast<int64_t>(it.head[s]) * f.a.tokens + at] = (m * c + log2f(l)) * 0.6931471805599453f;
    }
    if (!ok && lane == 0) { *abort_flag = 1; raise_flag(f.a.flags, kFlagTimeout); }
  }

  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {
    // let every TMA copy still in flight land before the CTA exits
    volatile int never = 0;
    for (int i = 0; i < kSlots + 2; ++i)
      if (issued[i]) tc::mbar_wait(i < kSlots ? &kv_full[i] : &q_full[i - kSlots], issued[i] - 1, &never);
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
  cudaError_t e = cudaFuncSetAttribute(k_attn_fwd_tc<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(Fwd<DP>::kSmem));
  if (e) return e;
  const int grid = static_cast<int>(std::min<int64_t>(std::max<int64_t>(items, 1), device_sm_count()));
  k_attn_fwd_tc<DP><<<grid, kThreads, Fwd<DP>::kSmem, s>>>(f);
  return cudaGetLastError();
}

cudaError_t launch_attn_forward_tc(const AttnArgs& a, cudaStream_t s, std::string* err) {
  FwdArgs f;
  f.a = a;
  if (!rows_map(&f.q, a.q, a.tokens, a.heads, a.dim, err) || !rows_map(&f.k, a.k, a.tokens, a.kv_heads, a.dim, err) ||
      !rows_map(&f.v, a.v, a.tokens, a.kv_heads, a.dim, err))
    return cudaErrorInvalidValue;
  f.pair_heads = a.group % 2 == 0;
  f.list = f.pair_heads ? a.by_query : a.by_pair;
  f.n_list = f.pair_heads ? a.n_blocks : a.n_pairs;
  const int64_t items = static_cast<int64_t>(f.n_list) * (f.pair_heads ? a.heads / 2 : a.heads);
  return a.dim <= 64 ? launch<64>(f, items, s) : launch<128>(f, items, s);
}

}  // namespace normpre
