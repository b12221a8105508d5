// Packed causal attention: plan, argument checks and launches of the
// normpre_attn_* entry points.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <iterator>
#include <memory>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/normpre.h"
#include "attn.h"
#include "internal.h"

using namespace normpre;

struct normpre_attn {
  normpre_attn_config cfg;
  int device = 0;
  int64_t max_blocks = 0;
  int n_blocks = 0, n_pairs = 0, n_keys = 0, n_split = 0;
  int64_t total = 0;
  // work lists of the current lengths, one block of memory: by_query, by_key,
  // by_pair, by_split, then the walks
  char* lists = nullptr;
  char* staging = nullptr;         // pinned, the same size
  cudaEvent_t copied = nullptr;    // the last copy out of `staging`
  cudaStream_t list_stream = nullptr;   // where it ran; calls there are in order with it
  int window = 0, sinks = 0;       // of the plan (0: none), and what the current lengths need of them
  int now_window = kNoWindow, now_sinks = 0;
  bool used = false, elsewhere = false;   // calls since: any, on other streams
  int64_t walk_at[3] = {-1, -1, -1};   // byte offsets of the walks, -1: none
  float* delta = nullptr;          // [n_heads][max_tokens]
  int chunk = 0, slots = 0;        // of split key blocks (see KeyPart): the least part, the most slots
  int now_chunk = 0;               // part of the current lengths
  float* partial = nullptr;
  int* flags = nullptr;            // pinned: set by kernels, read here between calls
};

namespace {

// Up to this many items a kernel's items are dealt out to the CTAs on the host;
// beyond it every CTA has dozens, and a fixed back-and-forth walk is as even.
constexpr int64_t kMaxDealt = 8192;
constexpr int64_t kWalkInts = kMaxDealt + 1024;   // most of one walk

int64_t list_bytes(const normpre_attn* a) {
  return (3 * a->max_blocks + 2 * a->slots) * static_cast<int64_t>(sizeof(AttnBlock)) +
         3 * kWalkInts * static_cast<int64_t>(sizeof(int));
}

// Most memory of the partial sums.
constexpr int64_t kMaxPartial = int64_t(64) << 20;

int64_t slot_bytes(const normpre_attn* a) {
  return static_cast<int64_t>(a->cfg.n_kv_heads) * 2 * 128 * a->cfg.head_dim * static_cast<int64_t>(sizeof(float));
}

// Parts of split key blocks: as long as a window's own walk, but long enough to
// be worth an item, and few enough for their memory.
void plan_parts(normpre_attn* a) {
  if (!a->window || !a->sinks) return;
  const int64_t most = std::min<int64_t>(kMaxSlots, kMaxPartial / slot_bytes(a));
  const int64_t blocks = cdiv(a->cfg.max_tokens, 128), sinks = std::min<int64_t>(cdiv(a->sinks, 128), blocks);
  // fp32 items are tiles of 64 rows and run in rounds whose longest item counts: one
  // block less than a window's own walk (2000 tokens, 12 heads of 64, window 100, 3
  // sinks: 165 us against 177; with 8 heads of 128 and 640 tokens 196 against 223)
  const int64_t walk = (126 + a->window) / 128 + 1;
  for (int64_t chunk = a->cfg.dtype == NORMPRE_BF16 ? std::max<int64_t>(8, walk) : std::max<int64_t>(1, walk - 1); chunk < blocks;
       chunk *= 2) {
    // a sequence of n > chunk blocks has at most 2 n / chunk parts for each of its sink blocks
    const int64_t slots = sinks * 2 * (blocks + blocks / chunk + 1) / chunk;
    if (slots > most) continue;
    a->chunk = static_cast<int>(chunk);
    a->slots = static_cast<int>(slots);
    return;
  }
}

int fail(int code, const std::string& msg) {
  set_thread_error(msg);
  return code;
}
int cuda_fail(cudaError_t e, const char* what) {
  return fail(NORMPRE_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

void release(normpre_attn* a) {
  cudaFree(a->lists);
  if (a->staging) cudaFreeHost(a->staging);
  if (a->copied) cudaEventDestroy(a->copied);
  cudaFree(a->delta);
  cudaFree(a->partial);
  if (a->flags) cudaFreeHost(a->flags);
  delete a;
}
struct Release {
  void operator()(normpre_attn* a) const { release(a); }
};

int take(const normpre_attn* a, const normpre_heads* t, int64_t tokens, int heads, const char* name, bool output,
         AttnTensor* out) {
  return take_heads(t, tokens, heads, a->cfg.head_dim, a->cfg.dtype, name, output, out);
}

AttnArgs base_args(const normpre_attn* a, int64_t tokens) {
  AttnArgs g = {};
  g.by_query = reinterpret_cast<const AttnBlock*>(a->lists);
  g.by_key = g.by_query + a->n_blocks;
  g.by_pair = g.by_key + a->n_keys;
  g.by_split = g.by_pair + a->n_pairs;
  const int** walks[3] = {&g.walk_fwd, &g.walk_dkdv, &g.walk_dq};
  for (int i = 0; i < 3; ++i)
    *walks[i] = a->walk_at[i] < 0 ? nullptr : reinterpret_cast<const int*>(a->lists + a->walk_at[i]);
  g.n_blocks = a->n_blocks;
  g.n_pairs = a->n_pairs;
  g.n_keys = a->n_keys;
  g.n_split = a->n_split;
  g.chunk = a->now_chunk;
  g.slots = a->slots;
  g.partial = a->partial;
  g.total = static_cast<int>(a->total);
  g.tokens = static_cast<int>(tokens);
  g.heads = a->cfg.n_heads;
  g.kv_heads = a->cfg.n_kv_heads;
  g.group = a->cfg.n_heads / a->cfg.n_kv_heads;
  g.dim = a->cfg.head_dim;
  g.window = a->now_window;
  g.sinks = a->now_sinks;
  g.scale = a->cfg.scale;
  g.scale_log2 = a->cfg.scale * 1.4426950408889634f;
  g.delta = a->delta;
  g.flags = a->flags;
  g.test_stall = a->cfg.test_stall;
  return g;
}

int flags_of(const normpre_attn* a) { return *static_cast<const volatile int*>(a->flags); }

constexpr char kOtherLists[] = "a captured call ran with the lists of other lengths than its own; its outputs have no meaning";

// Puts a call's stream behind the copy of the lists.
cudaError_t order(normpre_attn* a, cudaStream_t s) {
  a->used = true;
  if (s == a->list_stream) return cudaSuccess;
  a->elsewhere = true;
  cudaStreamCaptureStatus capture;
  cudaError_t e = cudaStreamIsCapturing(s, &capture);
  if (e) return e;
  if (capture == cudaStreamCaptureStatusNone) return cudaStreamWaitEvent(s, a->copied, 0);
  // a capture cannot depend on work outside it: the copy is waited for here
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  if ((e = cudaThreadExchangeStreamCaptureMode(&mode))) return e;
  e = cudaEventSynchronize(a->copied);
  const cudaError_t back = cudaThreadExchangeStreamCaptureMode(&mode);
  return e ? e : back;
}

int check_call(const normpre_attn* a, int64_t tokens) {
  if (flags_of(a) & kFlagTimeout)
    return fail(NORMPRE_ERR_TIMEOUT, "a bounded device wait of an earlier call of this plan gave up: what that call wrote "
                                     "has no meaning (normpre_attn_sync_status clears this)");
  if (flags_of(a) & kFlagLists) return fail(NORMPRE_ERR_ARG, kOtherLists);
  if (tokens < a->total || tokens > a->cfg.max_tokens)
    return fail(NORMPRE_ERR_SHAPE, "tokens must be between the sum of the lengths and max_tokens");
  return NORMPRE_OK;
}

// Deals out the items of a walk, given in falling order of cost (`per` items
// for each entry of `costs`): each goes to the CTA with the least so far.  loads:
// what the CTAs have already, a pair of load and CTA for each.
typedef std::vector<std::pair<int64_t, int>> Loads;
Loads no_loads(int grid) {
  Loads loads;
  for (int c = 0; c < grid; ++c) loads.push_back({0, c});
  return loads;
}
void deal(const std::vector<int>& costs, int per, Loads* loads, std::vector<int>* out) {
  const int64_t items = static_cast<int64_t>(costs.size()) * per;
  Loads& heap = *loads;                                      // the least on top
  const int grid = static_cast<int>(heap.size());
  const auto more = std::greater<std::pair<int64_t, int>>();
  std::make_heap(heap.begin(), heap.end(), more);
  std::vector<int> owner(items), count(grid + 1, 0);
  for (int64_t i = 0; i < items; ++i) {
    std::pop_heap(heap.begin(), heap.end(), more);
    owner[i] = heap.back().second;
    heap.back().first += costs[i / per];
    ++count[owner[i] + 1];
    std::push_heap(heap.begin(), heap.end(), more);
  }
  for (int c = 0; c < grid; ++c) count[c + 1] += count[c];
  out->assign(grid + 1 + items, 0);
  std::copy(count.begin(), count.end(), out->begin());
  for (int64_t i = 0; i < items; ++i) (*out)[grid + 1 + count[owner[i]]++] = static_cast<int>(i);
}

int set_lengths(normpre_attn* a, int n_seqs, const int64_t* lengths, cudaStream_t s) {
  int64_t total = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (lengths[i] < 0) return fail(NORMPRE_ERR_ARG, "lengths[" + std::to_string(i) + "] is negative");
    if (lengths[i] > a->cfg.max_tokens - total) return fail(NORMPRE_ERR_SHAPE, "the lengths exceed max_tokens");
    total += lengths[i];
  }
  // a window that no sequence is longer than hides nothing
  int64_t longest = 0;
  for (int i = 0; i < n_seqs; ++i) longest = std::max(longest, lengths[i]);
  const bool windowed = a->window && a->window < longest;
  const int window = windowed ? a->window : kNoWindow, sinks = windowed ? a->sinks : 0;
  std::vector<AttnBlock> blocks;
  int64_t start = 0;
  for (int i = 0; i < n_seqs; ++i) {
    for (int64_t b = 0; b * 128 < lengths[i]; ++b)
      blocks.push_back(AttnBlock{static_cast<int>(start), static_cast<int>(lengths[i]), static_cast<int>(b), 0});
    start += lengths[i];
  }
  // longest work first
  auto keys = [&](const AttnBlock& b, int top) { return key_span(b.blk, window, sinks).count(top); };
  auto queries = [&](const AttnBlock& b) { return last_query(b.blk, b.len, window, sinks) - b.blk; };
  std::stable_sort(blocks.begin(), blocks.end(),
                   [&](const AttnBlock& x, const AttnBlock& y) { return keys(x, x.blk) > keys(y, y.blk); });
  // A block that is no more than about half of what a CTA gets in all is dealt
  // out well as it is: 8 x 2432 tokens, window 1024, 450 us without parts, 475 with.
  int chunk = 0, slots = 0;
  if (windowed && a->chunk) {
    int64_t all = 0;
    for (const AttnBlock& b : blocks) all += queries(b) + 1;
    const int64_t ctas = device_sm_count() * (a->cfg.dtype == NORMPRE_BF16 ? 1 : 2);
    chunk = static_cast<int>(std::max<int64_t>(a->chunk, all * a->cfg.n_kv_heads / (2 * ctas)));
  }
  std::vector<AttnBlock> by_key, pairs, by_split;
  for (AttnBlock b : blocks) {
    const int count = queries(b) + 1, parts = chunk ? key_parts(count, chunk) : 1;
    if (128 * b.blk >= sinks || parts < 2 || slots + parts > a->slots) {
      by_key.push_back(b);
      continue;
    }
    b.part = slots;
    by_split.push_back(b);
    for (int i = 0; i < parts; ++i) {
      b.part = i << 12 | (slots++ + 1);
      by_key.push_back(b);
    }
  }
  auto walked = [&](const AttnBlock& b) {
    const KeyPart p = key_part(b, window, sinks, chunk, a->slots);
    return p.end - p.first;
  };
  std::stable_sort(by_key.begin(), by_key.end(),
                   [&](const AttnBlock& x, const AttnBlock& y) { return walked(x) > walked(y); });
  std::copy_if(blocks.begin(), blocks.end(), std::back_inserter(pairs), [](const AttnBlock& b) { return b.blk % 2 == 0; });
  const int h = a->cfg.n_heads, hk = a->cfg.n_kv_heads, group = h / hk;
  const int64_t n = static_cast<int64_t>(blocks.size());
  std::vector<int> walk[3];
  if (a->cfg.dtype == NORMPRE_BF16 && n && n * h <= kMaxDealt && static_cast<int64_t>(by_key.size()) * hk <= kMaxDealt) {
    // costs in tiles, with about what an item's start and end take
    std::vector<int> fwd, dkdv, dq;
    const bool heads = attn_pair_heads(group);
    for (const AttnBlock& b : heads ? blocks : pairs)
      fwd.push_back(2 * keys(b, heads || (b.blk + 1) * 128 >= b.len ? b.blk : b.blk + 1) + 2);
    // four products a tile against three
    for (const AttnBlock& b : by_key) dkdv.push_back(5 * (group * walked(b) + 1));
    for (const AttnBlock& b : blocks) dq.push_back(4 * (keys(b, b.blk) + 1));
    const int64_t of_fwd = static_cast<int64_t>(fwd.size()) * (heads ? h / 2 : h), of_keys = static_cast<int64_t>(by_key.size()) * hk;
    const int64_t of_queries = n * h;
    Loads loads = no_loads(walk_grid(of_fwd));
    deal(fwd, heads ? h / 2 : h, &loads, &walk[0]);
    // with a window the two walks of the backward pass are one launch
    loads = no_loads(walk_grid(windowed ? std::max(of_keys, of_queries) : of_keys));
    deal(dkdv, hk, &loads, &walk[1]);
    if (!windowed) loads = no_loads(walk_grid(of_queries));
    deal(dq, h, &loads, &walk[2]);
  }
  // one copy; the staging memory is free once the last one has left it, the
  // lists once the calls that read them are done
  cudaError_t e = cudaEventSynchronize(a->copied);
  if (!e && (a->elsewhere || (a->used && s != a->list_stream))) e = cudaDeviceSynchronize();
  if (e) return cuda_fail(e, "normpre_attn_set_lengths");
  a->list_stream = s;
  a->used = a->elsewhere = false;
  int64_t at = 0, walk_at[3];
  auto put = [&](const void* src, size_t bytes) {
    if (bytes) std::memcpy(a->staging + at, src, bytes);
    at += static_cast<int64_t>(bytes);
  };
  put(blocks.data(), blocks.size() * sizeof(AttnBlock));
  put(by_key.data(), by_key.size() * sizeof(AttnBlock));
  put(pairs.data(), pairs.size() * sizeof(AttnBlock));
  put(by_split.data(), by_split.size() * sizeof(AttnBlock));
  for (int i = 0; i < 3; ++i) {
    walk_at[i] = walk[i].empty() ? -1 : at;
    put(walk[i].data(), walk[i].size() * sizeof(int));
  }
  if (at) e = cudaMemcpyAsync(a->lists, a->staging, static_cast<size_t>(at), cudaMemcpyHostToDevice, s);
  if (!e) e = cudaEventRecord(a->copied, s);
  if (e) return cuda_fail(e, "cudaMemcpyAsync");
  a->n_blocks = static_cast<int>(n);
  a->n_pairs = static_cast<int>(pairs.size());
  a->n_keys = static_cast<int>(by_key.size());
  a->n_split = static_cast<int>(by_split.size());
  std::copy(walk_at, walk_at + 3, a->walk_at);
  a->total = total;
  a->now_chunk = chunk;
  a->now_window = window;
  a->now_sinks = sinks;
  return NORMPRE_OK;
}

}  // namespace

extern "C" {

int normpre_attn_init(const normpre_attn_config* cfg, normpre_attn** out) {
  return normpre_attn_init_window(cfg, 0, 0, out);
}

int normpre_attn_init_window(const normpre_attn_config* cfg, int64_t window, int64_t sinks, normpre_attn** out) {
  if (!cfg || !out) return fail(NORMPRE_ERR_ARG, "null argument");
  *out = nullptr;
  if (cfg->dtype != NORMPRE_F32 && cfg->dtype != NORMPRE_BF16)
    return fail(NORMPRE_ERR_DTYPE, "dtype must be NORMPRE_F32 or NORMPRE_BF16");
  if (cfg->n_heads < 1 || cfg->n_kv_heads < 1 || cfg->n_heads > 65535 || cfg->n_heads % cfg->n_kv_heads)
    return fail(NORMPRE_ERR_SHAPE, "n_heads must be in [1, 65535] and a multiple of n_kv_heads");
  if (cfg->head_dim < 8 || cfg->head_dim > 128 || cfg->head_dim % 8)
    return fail(NORMPRE_ERR_SHAPE, "head_dim must be a multiple of 8 in [8, 128]");
  if (cfg->max_tokens < 1 || cfg->max_tokens > (int64_t(1) << 24) || cfg->max_seqs < 1 || cfg->max_seqs > 65536)
    return fail(NORMPRE_ERR_SHAPE, "max_tokens must be in [1, 2^24] and max_seqs in [1, 65536]");
  if (!std::isfinite(cfg->scale) || cfg->scale < 0.f) return fail(NORMPRE_ERR_ARG, "scale must be finite and >= 0");
  if (window < 0 || sinks < 0) return fail(NORMPRE_ERR_ARG, "window and sinks must be >= 0");
  if (cfg->test_stall < 0 || cfg->test_stall > 2) return fail(NORMPRE_ERR_ARG, "test_stall must be 0, 1 or 2");
  try {
    std::unique_ptr<normpre_attn, Release> a(new normpre_attn());
    a->cfg = *cfg;
    // beyond max_tokens there is nothing that a window hides or a sink shows
    a->window = window < cfg->max_tokens ? static_cast<int>(window) : 0;
    a->sinks = a->window ? static_cast<int>(std::min(sinks, cfg->max_tokens)) : 0;
    if (a->cfg.scale == 0.f) a->cfg.scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(cfg->head_dim)));
    a->max_blocks = cfg->max_tokens / 128 + std::min<int64_t>(cfg->max_seqs, cfg->max_tokens);
    plan_parts(a.get());
    cudaError_t e = cudaGetDevice(&a->device);
    if (!e) e = cudaMalloc(&a->lists, list_bytes(a.get()));
    if (!e) e = cudaHostAlloc(&a->staging, list_bytes(a.get()), cudaHostAllocDefault);
    if (!e) e = cudaEventCreateWithFlags(&a->copied, cudaEventDisableTiming);
    if (!e) e = cudaMalloc(&a->delta, static_cast<size_t>(cfg->n_heads) * cfg->max_tokens * sizeof(float));
    if (!e && a->slots) e = cudaMalloc(&a->partial, static_cast<size_t>(a->slots) * slot_bytes(a.get()));
    if (!e) e = cudaHostAlloc(&a->flags, sizeof(int), cudaHostAllocDefault);
    if (e) return cuda_fail(e, "normpre_attn_init");
    *a->flags = 0;
    *out = a.release();
  } catch (const std::bad_alloc&) {
    return fail(NORMPRE_ERR_CUDA, "out of host memory");
  }
  return NORMPRE_OK;
}

int normpre_attn_set_lengths(normpre_attn* a, int n_seqs, const int64_t* lengths, void* stream) {
  if (!a || (n_seqs > 0 && !lengths)) return fail(NORMPRE_ERR_ARG, "null argument");
  if (n_seqs < 0) return fail(NORMPRE_ERR_ARG, "n_seqs is negative");
  if (n_seqs > a->cfg.max_seqs) return fail(NORMPRE_ERR_SHAPE, "more sequences than max_seqs");
  DeviceGuard device_guard(a->device);
  try {
    return set_lengths(a, n_seqs, lengths, static_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return fail(NORMPRE_ERR_CUDA, "out of host memory");
  }
}

int normpre_attn_forward(normpre_attn* a, int64_t tokens, const normpre_heads* q, const normpre_heads* k,
                         const normpre_heads* v, const normpre_heads* out, float* lse, void* stream) {
  if (!a) return fail(NORMPRE_ERR_ARG, "null plan");
  int rc = check_call(a, tokens);
  if (rc || !tokens) return rc;
  AttnArgs g = base_args(a, tokens);
  const int h = a->cfg.n_heads, hk = a->cfg.n_kv_heads;
  if ((rc = take(a, q, tokens, h, "q", false, &g.q)) || (rc = take(a, k, tokens, hk, "k", false, &g.k)) ||
      (rc = take(a, v, tokens, hk, "v", false, &g.v)) || (rc = take(a, out, tokens, h, "out", true, &g.o)))
    return rc;
  if (!lse) return fail(NORMPRE_ERR_ARG, "lse: null");
  g.lse = lse;
  DeviceGuard device_guard(a->device);
  std::string err;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = order(a, s);
  if (!e) e = a->cfg.dtype == NORMPRE_BF16 ? launch_attn_forward_tc(g, s, &err) : launch_attn_forward_simt(g, s);
  return e ? cuda_fail(e, err.empty() ? "attention forward" : err.c_str()) : NORMPRE_OK;
}

int normpre_attn_backward(normpre_attn* a, int64_t tokens, const normpre_heads* q, const normpre_heads* k,
                          const normpre_heads* v, const normpre_heads* out, const float* lse,
                          const normpre_heads* dout, const normpre_heads* dq, const normpre_heads* dk,
                          const normpre_heads* dv, void* stream) {
  if (!a) return fail(NORMPRE_ERR_ARG, "null plan");
  int rc = check_call(a, tokens);
  if (rc || !tokens) return rc;
  AttnArgs g = base_args(a, tokens);
  const int h = a->cfg.n_heads, hk = a->cfg.n_kv_heads;
  if ((rc = take(a, q, tokens, h, "q", false, &g.q)) || (rc = take(a, k, tokens, hk, "k", false, &g.k)) ||
      (rc = take(a, v, tokens, hk, "v", false, &g.v)) || (rc = take(a, out, tokens, h, "out", false, &g.o)) ||
      (rc = take(a, dout, tokens, h, "dout", false, &g.dout)) || (rc = take(a, dq, tokens, h, "dq", true, &g.dq)) ||
      (rc = take(a, dk, tokens, hk, "dk", true, &g.dk)) || (rc = take(a, dv, tokens, hk, "dv", true, &g.dv)))
    return rc;
  if (!lse) return fail(NORMPRE_ERR_ARG, "lse: null");
  g.lse = const_cast<float*>(lse);
  DeviceGuard device_guard(a->device);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = order(a, s);
  if (!e) e = launch_attn_delta(g, a->cfg.dtype, s);
  std::string err;
  if (!e) e = a->cfg.dtype == NORMPRE_BF16 ? launch_attn_backward_tc(g, s, &err) : launch_attn_backward_simt(g, s);
  if (!e) e = launch_attn_join(g, a->cfg.dtype, s);
  return e ? cuda_fail(e, err.empty() ? "attention backward" : err.c_str()) : NORMPRE_OK;
}

int normpre_attn_sync_status(normpre_attn* a, void* stream) {
  if (!a) return fail(NORMPRE_ERR_ARG, "null plan");
  DeviceGuard device_guard(a->device);
  const cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e) return cuda_fail(e, "normpre_attn_sync_status");
  const int flags = flags_of(a);
  if (flags) *static_cast<volatile int*>(a->flags) = 0;
  if (flags & kFlagTimeout) return fail(NORMPRE_ERR_TIMEOUT, "a bounded device wait gave up");
  if (flags & kFlagLists) return fail(NORMPRE_ERR_ARG, kOtherLists);
  return NORMPRE_OK;
}

void normpre_attn_free(normpre_attn* a) {
  if (!a) return;
  DeviceGuard device_guard(a->device);
  cudaDeviceSynchronize();
  release(a);
}

}  // extern "C"
