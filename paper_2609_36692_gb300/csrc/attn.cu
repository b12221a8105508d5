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
  int n_blocks = 0, n_pairs = 0;
  int64_t total = 0;
  // work lists of the current lengths, one block of memory: by_query, by_key,
  // by_pair, then the walks
  char* lists = nullptr;
  char* staging = nullptr;         // pinned, the same size
  cudaEvent_t copied = nullptr;    // the last copy out of `staging`
  cudaStream_t list_stream = nullptr;   // where it ran; calls there are in order with it
  bool used = false, elsewhere = false;   // calls since: any, on other streams
  int64_t walk_at[3] = {-1, -1, -1};   // byte offsets of the walks, -1: none
  float* delta = nullptr;          // [n_heads][max_tokens]
  int* flags = nullptr;            // pinned: set by kernels, read here between calls
};

namespace {

// Up to this many items a kernel's items are dealt out to the CTAs on the host;
// beyond it every CTA has dozens, and a fixed back-and-forth walk is as even.
constexpr int64_t kMaxDealt = 8192;
constexpr int64_t kWalkInts = kMaxDealt + 1024;   // most of one walk

int64_t list_bytes(const normpre_attn* a) {
  return 3 * (a->max_blocks * static_cast<int64_t>(sizeof(AttnBlock)) + kWalkInts * static_cast<int64_t>(sizeof(int)));
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
  if (a->flags) cudaFreeHost(a->flags);
  delete a;
}
struct Release {
  void operator()(normpre_attn* a) const { release(a); }
};

// Checks one tensor argument and copies it; a stride that no address uses (a
// single row or head) is replaced by a valid one.
int take(const normpre_attn* a, const normpre_heads* t, int64_t tokens, int heads, const char* name, bool output,
         AttnTensor* out) {
  if (!t || !t->data) return fail(NORMPRE_ERR_ARG, std::string(name) + ": null");
  const int64_t d = a->cfg.head_dim, per16 = a->cfg.dtype == NORMPRE_BF16 ? 8 : 4;
  int64_t ts = tokens > 1 ? t->token_stride : 0, hs = heads > 1 ? t->head_stride : 0;
  if (tokens > 1 && (ts < d || ts > (int64_t(1) << 30)))
    return fail(NORMPRE_ERR_SHAPE, std::string(name) + ": token stride must be in [head_dim, 2^30]");
  if (heads > 1 && (hs < d || hs > (int64_t(1) << 36)))
    return fail(NORMPRE_ERR_SHAPE, std::string(name) + ": head stride must be in [head_dim, 2^36]");
  if ((reinterpret_cast<uintptr_t>(t->data) & 15u) || ts % per16 || hs % per16)
    return fail(NORMPRE_ERR_ALIGN, std::string(name) + ": data and strides must be multiples of 16 bytes");
  if (output && tokens > 1 && heads > 1) {
    const bool by_token = ts >= hs;   // rows outermost, or heads
    const int64_t inner = by_token ? (heads - 1) * hs + d : (tokens - 1) * ts + d;
    if ((by_token ? ts : hs) < inner) return fail(NORMPRE_ERR_SHAPE, std::string(name) + ": overlapping strides");
  }
  if (!ts) ts = round_up(d, 8);
  if (!hs) hs = round_up(d, 8);
  *out = AttnTensor{t->data, ts, hs};
  return NORMPRE_OK;
}

AttnArgs base_args(const normpre_attn* a, int64_t tokens) {
  AttnArgs g = {};
  g.by_query = reinterpret_cast<const AttnBlock*>(a->lists);
  g.by_key = g.by_query + a->n_blocks;
  g.by_pair = g.by_key + a->n_blocks;
  const int** walks[3] = {&g.walk_fwd, &g.walk_dkdv, &g.walk_dq};
  for (int i = 0; i < 3; ++i)
    *walks[i] = a->walk_at[i] < 0 ? nullptr : reinterpret_cast<const int*>(a->lists + a->walk_at[i]);
  g.n_blocks = a->n_blocks;
  g.n_pairs = a->n_pairs;
  g.total = static_cast<int>(a->total);
  g.tokens = static_cast<int>(tokens);
  g.heads = a->cfg.n_heads;
  g.kv_heads = a->cfg.n_kv_heads;
  g.group = a->cfg.n_heads / a->cfg.n_kv_heads;
  g.dim = a->cfg.head_dim;
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

// Deals out the items of a kernel, given in falling order of cost (`per` items
// for each entry of `costs`): each goes to the CTA with the least so far.
void deal(const std::vector<int>& costs, int per, std::vector<int>* out) {
  const int64_t items = static_cast<int64_t>(costs.size()) * per;
  const int grid = walk_grid(items);
  std::vector<std::pair<int64_t, int>> heap;                 // load, CTA; the least on top
  for (int c = 0; c < grid; ++c) heap.push_back({0, c});
  const auto more = std::greater<std::pair<int64_t, int>>();
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
  std::vector<AttnBlock> blocks;
  int64_t start = 0;
  for (int i = 0; i < n_seqs; ++i) {
    for (int64_t b = 0; b * 128 < lengths[i]; ++b)
      blocks.push_back(AttnBlock{static_cast<int>(start), static_cast<int>(lengths[i]), static_cast<int>(b), 0});
    start += lengths[i];
  }
  // longest work first
  auto queries = [](const AttnBlock& b) { return (b.len - 1) / 128 - b.blk; };
  std::stable_sort(blocks.begin(), blocks.end(), [](const AttnBlock& x, const AttnBlock& y) { return x.blk > y.blk; });
  std::vector<AttnBlock> by_key = blocks, pairs;
  std::stable_sort(by_key.begin(), by_key.end(),
                   [&](const AttnBlock& x, const AttnBlock& y) { return queries(x) > queries(y); });
  std::copy_if(blocks.begin(), blocks.end(), std::back_inserter(pairs), [](const AttnBlock& b) { return b.blk % 2 == 0; });
  const int h = a->cfg.n_heads, hk = a->cfg.n_kv_heads, group = h / hk;
  const int64_t n = static_cast<int64_t>(blocks.size());
  std::vector<int> walk[3];
  if (a->cfg.dtype == NORMPRE_BF16 && n && n * h <= kMaxDealt) {
    // costs in tiles, with about what an item's start and end take
    std::vector<int> fwd, dkdv, dq;
    const bool heads = attn_pair_heads(group);
    for (const AttnBlock& b : heads ? blocks : pairs)
      fwd.push_back(2 * (b.blk + 1) + (heads ? 2 : (b.blk + 1) * 128 < b.len ? 4 : 2));
    for (const AttnBlock& b : by_key) dkdv.push_back(group * (queries(b) + 1) + 1);
    for (const AttnBlock& b : blocks) dq.push_back(b.blk + 2);
    deal(fwd, heads ? h / 2 : h, &walk[0]);
    deal(dkdv, hk, &walk[1]);
    deal(dq, h, &walk[2]);
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
  for (int i = 0; i < 3; ++i) {
    walk_at[i] = walk[i].empty() ? -1 : at;
    put(walk[i].data(), walk[i].size() * sizeof(int));
  }
  if (at) e = cudaMemcpyAsync(a->lists, a->staging, static_cast<size_t>(at), cudaMemcpyHostToDevice, s);
  if (!e) e = cudaEventRecord(a->copied, s);
  if (e) return cuda_fail(e, "cudaMemcpyAsync");
  a->n_blocks = static_cast<int>(n);
  a->n_pairs = static_cast<int>(pairs.size());
  std::copy(walk_at, walk_at + 3, a->walk_at);
  a->total = total;
  return NORMPRE_OK;
}

}  // namespace

extern "C" {

int normpre_attn_init(const normpre_attn_config* cfg, normpre_attn** out) {
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
  if (cfg->test_stall != 0 && cfg->test_stall != 1) return fail(NORMPRE_ERR_ARG, "test_stall must be 0 or 1");
  try {
    std::unique_ptr<normpre_attn, Release> a(new normpre_attn());
    a->cfg = *cfg;
    if (a->cfg.scale == 0.f) a->cfg.scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(cfg->head_dim)));
    a->max_blocks = cfg->max_tokens / 128 + std::min<int64_t>(cfg->max_seqs, cfg->max_tokens);
    cudaError_t e = cudaGetDevice(&a->device);
    if (!e) e = cudaMalloc(&a->lists, list_bytes(a.get()));
    if (!e) e = cudaHostAlloc(&a->staging, list_bytes(a.get()), cudaHostAllocDefault);
    if (!e) e = cudaEventCreateWithFlags(&a->copied, cudaEventDisableTiming);
    if (!e) e = cudaMalloc(&a->delta, static_cast<size_t>(cfg->n_heads) * cfg->max_tokens * sizeof(float));
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
