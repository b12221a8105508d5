// The norm of many gradients taken as one vector, and clipping by it: the
// normpre_grad_* entry points.
//
//   n = sqrt(sum g^2),   c = min(1, max_norm / (n + eps)),   g' = c g
//
// Two launches for a table of tensors: k_grad_squares sums the squares, one
// partial sum per CTA; k_grad_scale folds the partial sums in each CTA (a few
// kilobytes from L2), and writes the clipped values.  In place and with c = 1 it
// changes nothing and reads nothing more.  The partial sums have fixed shares
// and a fixed order: the same inputs give the same bits.  The tables travel as
// launch arguments, so that a call copies nothing to the device and can be
// captured.
//
// Bound by HBM: the norm must be known before the first value is written, so
// that what does not stay in L2 is read twice.  Each CTA therefore scales its
// share backwards, from what it read last.  405 M fp32 values to bf16: 1.62 GB
// read twice, 0.81 written, 0.600 ms (6.75 TB/s).  16 tensors of 5.4 MB: 16 us, two
// launches and the latency of the tables, the loads and the sums, behind 40 us of
// the host's.
//
// Range and precision: a thread sums 16 KB / 256 threads = 64 bytes of values
// in fp32, four sums of 16 bytes side by side, where squares cannot overflow or vanish, else in fp64; everything
// beyond is fp64.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/normpre.h"
#include "common.cuh"
#include "internal.h"

namespace normpre {
namespace {

constexpr int kThreads = 256;
constexpr int kChunkBytes = 16384;   // of the input: what a CTA takes at once
constexpr int kPerSm = 4;            // CTAs
constexpr int kMaxCtas = 1024;       // of one launch

struct Entry {
  const void* in;
  void* out;
  int64_t size;        // elements
  uint32_t first;      // the tensor's first chunk of the table
  uint16_t in_bf16, out_bf16;
};
template <int N> struct Table {
  Entry e[N];
  int n;
  uint32_t chunks;
};
constexpr int kSmall = 64, kLarge = 960;   // 2 KB and 30 KB of launch arguments

// The entry that holds a chunk.
template <int N>
__device__ __forceinline__ int find(const Table<N>& t, uint32_t chunk) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Sixteen bytes of a tensor as fp32 values.
template <typename T> struct Piece {
  static constexpr int kN = 16 / sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return i & 1 ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]);
  }
  // elements i .. of the tensor's n, i a multiple of 16 bytes' worth before its
  // first one or behind it: zeros outside.  ONLY_READ: the launch writes nothing of
  // the memory, which the read-only path asks for; clipping in place does.
  template <bool ONLY_READ> __device__ __forceinline__ void load(const T* p, int64_t i, int64_t n) {
    auto get = [](const auto* at) { return ONLY_READ ? __ldg(at) : *at; };
    if (i >= 0 && i + kN <= n) {
      const uint4 q = get(reinterpret_cast<const uint4*>(p + i));
      w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = 0;
#pragma unroll
      for (int e = 0; e < kN; ++e)
        if (i + e >= 0 && i + e < n) {
          if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(get(p + i + e));
          else w[e >> 1] |= static_cast<uint32_t>(get(reinterpret_cast<const unsigned short*>(p) + i + e)) << (16 * (e & 1));
        }
    }
  }
  template <typename U> __device__ __forceinline__ void store(U* p, int64_t i, int64_t n, float c, bool aligned) const {
    if (i >= 0 && i + kN <= n && aligned) {
      uint32_t o[kN * sizeof(U) / 4];
#pragma unroll
      for (int e = 0; e < kN; e += 2) {
        if constexpr (sizeof(U) == 4) {
          o[e] = __float_as_uint(at(e) * c);
          o[e + 1] = __float_as_uint(at(e + 1) * c);
        } else {
          o[e >> 1] = pack_bf16x2(at(e) * c, at(e + 1) * c);
        }
      }
      if constexpr (kN * sizeof(U) == 8) {
        *reinterpret_cast<uint2*>(p + i) = make_uint2(o[0], o[1]);
      } else {
#pragma unroll
        for (int e = 0; e < static_cast<int>(kN * sizeof(U) / 4); e += 4)
          *reinterpret_cast<uint4*>(p + i + e * (4 / sizeof(U))) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e)
        if (i + e >= 0 && i + e < n) p[i + e] = from_f32<U>(at(e) * c);
    }
  }
};

// A thread's share of a chunk: four pieces, neighbours in neighbouring threads.
// Chunks start on 16-byte boundaries, the first one at or before the tensor.
template <typename T> struct Share {
  Piece<T> q[4];
  static __device__ __forceinline__ int64_t index(const Entry& e, uint32_t chunk, int i) {
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(e.in) % 16 / sizeof(T));
    return (static_cast<int64_t>(chunk - e.first) * (kChunkBytes / 16) + i * kThreads + static_cast<int>(threadIdx.x)) *
               Piece<T>::kN - lead;
  }
  template <bool ONLY_READ> __device__ __forceinline__ void load(const Entry& e, uint32_t chunk) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i].template load<ONLY_READ>(static_cast<const T*>(e.in), index(e, chunk, i), e.size);
  }
  __device__ __forceinline__ double squares() const {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = q[i].at(0) * q[i].at(0);
#pragma unroll
      for (int e = 1; e < Piece<T>::kN; ++e) p[i] = fmaf(q[i].at(e), q[i].at(e), p[i]);
    }
    const float s = (p[0] + p[1]) + (p[2] + p[3]);
    if (s > 0x1p-100f && s < 0x1p120f) return s;
    // squares near the ends of fp32's range
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= q[i].w[e];
    if (!any) return 0.;
    double d = 0.;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < Piece<T>::kN; ++e) d = fma(static_cast<double>(q[i].at(e)), static_cast<double>(q[i].at(e)), d);
    return d;
  }
  template <typename U> __device__ __forceinline__ void store(const Entry& e, uint32_t chunk, float c) const {
    constexpr int kOut = Piece<T>::kN * sizeof(U) < 16 ? 8 : 16;
    // whether the output's pieces start on their boundaries too
    const bool aligned = reinterpret_cast<uintptr_t>(static_cast<U*>(e.out) + index(e, e.first, 0)) % kOut == 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i].store(static_cast<U*>(e.out), index(e, chunk, i), e.size, c, aligned);
  }
};

template <typename T>
__device__ __forceinline__ double chunk_squares(const Entry& e, uint32_t chunk) {
  Share<T> x;
  x.template load<true>(e, chunk);
  return x.squares();
}

template <int N>
__global__ void __launch_bounds__(kThreads, kPerSm) k_grad_squares(const __grid_constant__ Table<N> t, double* part) {
  __shared__ double red[kThreads / 32];
  uint32_t c = static_cast<uint32_t>(static_cast<uint64_t>(t.chunks) * blockIdx.x / gridDim.x);
  const uint32_t end = static_cast<uint32_t>(static_cast<uint64_t>(t.chunks) * (blockIdx.x + 1) / gridDim.x);
  double sum = 0.;
  if (c < end) {
    int i = find(t, c);
    for (; c < end; ++c) {
      while (i + 1 < t.n && t.e[i + 1].first <= c) ++i;
      sum += t.e[i].in_bf16 ? chunk_squares<bf16>(t.e[i], c) : chunk_squares<float>(t.e[i], c);
    }
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The sum of all partial sums; every thread gets it.
__device__ __forceinline__ double fold(const double* part, int parts, double* red) {
  double sum = 0.;
  for (int i = threadIdx.x; i < parts; i += kThreads) sum += part[i];
  return block_sum(sum, red);
}

// The root of a sum in fp64.  Where fp32's range allows, its fp32 root f and one
// step of Heron's method, f + (sum - f^2) / (2 f), whose last quotient needs fp32
// only: off by 2^-46 (the fp64 root takes a microsecond).
__device__ __forceinline__ double root(double sum) {
  if (!(sum > 0x1p-120 && sum < 0x1p120)) return sqrt(sum);
  const float f = sqrtf(static_cast<float>(sum));
  const double n = f;
  return fma(fma(-n, n, sum), static_cast<double>(0.5f / f), n);
}

// min(1, limit / (n + eps)), rounded once: the fp32 quotient q and one step of its
// refinement, q + (limit - q to) / to, where fp32's range allows.  A norm that is
// NaN gives NaN; all zeros are left as they are.
__device__ __forceinline__ float clip_factor(double n, float max_norm, float eps) {
  const double to = n + static_cast<double>(eps), limit = max_norm;
  if (to <= limit) return 1.f;
  if (!(to > 0x1p-60 && to < 0x1p60 && limit > 0x1p-60)) return static_cast<float>(limit / to);
  const float f = static_cast<float>(to), inv = 1.f / f;
  const double q = max_norm * inv;
  return static_cast<float>(fma(fma(-q, to, limit), static_cast<double>(inv), q));
}

template <typename T, typename U>
__device__ __forceinline__ void scale_chunk(const Entry& e, uint32_t chunk, float c) {
  Share<T> x;
  x.template load<false>(e, chunk);
  x.template store<U>(e, chunk, c);
}

template <int N>
__global__ void __launch_bounds__(kThreads, kPerSm) k_grad_scale(const __grid_constant__ Table<N> t, const double* part, int parts,
                                                         float max_norm, float eps, int in_place, float* norm) {
  __shared__ double red[kThreads / 32];
  __shared__ float factor;
  const double sum = fold(part, parts, red);
  if (threadIdx.x == 0) {
    const double n = root(sum);
    factor = clip_factor(n, max_norm, eps);
    if (norm && blockIdx.x == 0) *norm = static_cast<float>(n);
  }
  __syncthreads();
  const float f = factor;
  if (in_place && f == 1.f) return;
  const uint32_t first = static_cast<uint32_t>(static_cast<uint64_t>(t.chunks) * blockIdx.x / gridDim.x);
  uint32_t c = static_cast<uint32_t>(static_cast<uint64_t>(t.chunks) * (blockIdx.x + 1) / gridDim.x);
  if (c <= first) return;
  int i = find(t, c - 1);
  while (c-- > first) {
    while (t.e[i].first > c) --i;
    const Entry& e = t.e[i];
    if (e.in_bf16) {
      if (e.out_bf16) scale_chunk<bf16, bf16>(e, c, f);
      else scale_chunk<bf16, float>(e, c, f);
    } else {
      if (e.out_bf16) scale_chunk<float, bf16>(e, c, f);
      else scale_chunk<float, float>(e, c, f);
    }
  }
}

__global__ void __launch_bounds__(kThreads) k_grad_norm(const double* part, int parts, float* norm) {
  __shared__ double red[kThreads / 32];
  const double sum = fold(part, parts, red);
  if (threadIdx.x == 0) *norm = static_cast<float>(root(sum));
}

int fail(int code, const std::string& msg) {
  set_thread_error(msg);
  return code;
}
int done(cudaError_t e, const char* what) {
  return e ? fail(NORMPRE_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e)) : NORMPRE_OK;
}

int64_t max_launches(int n) { return cdiv(n < 1 ? 1 : n, kLarge); }

int check_list(int n, const void* const* grads, const int* dtypes, const int64_t* sizes) {
  if (n < 0 || n > (1 << 20)) return fail(NORMPRE_ERR_ARG, "the number of gradients must be in [0, 2^20]");
  if (n && (!grads || !dtypes || !sizes)) return fail(NORMPRE_ERR_ARG, "null argument");
  int64_t total = 0;
  auto refuse = [](int code, int i, const char* what) { return fail(code, "gradient " + std::to_string(i) + what); };
  for (int i = 0; i < n; ++i) {
    if (dtypes[i] != NORMPRE_F32 && dtypes[i] != NORMPRE_BF16)
      return refuse(NORMPRE_ERR_DTYPE, i, ": dtype must be NORMPRE_F32 or NORMPRE_BF16");
    // a table's chunks are counted in 32 bits
    if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 40) - total)
      return refuse(NORMPRE_ERR_SHAPE, i, ": size must be >= 0, and all together at most 2^40");
    total += sizes[i];
    if (!sizes[i]) continue;
    if (!grads[i]) return refuse(NORMPRE_ERR_ARG, i, ": null");
    if (reinterpret_cast<uintptr_t>(grads[i]) % (dtypes[i] == NORMPRE_BF16 ? 2 : 4))
      return refuse(NORMPRE_ERR_ALIGN, i, " must be aligned to its elements");
  }
  return NORMPRE_OK;
}

// Refuses outputs that share memory with another output or with another input
// (or with their own, unless they are it).
int check_overlap(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
                  const int* out_dtypes) {
  struct Span {
    uintptr_t at, end;
    int i;
    bool out;
  };
  std::vector<Span> spans;
  spans.reserve(2 * static_cast<size_t>(n));
  auto bytes = [](int dtype) { return dtype == NORMPRE_BF16 ? 2 : 4; };
  for (int i = 0; i < n; ++i) {
    if (!sizes[i]) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(grads[i]), b = reinterpret_cast<uintptr_t>(out[i]);
    if (a != b || dtypes[i] != out_dtypes[i]) spans.push_back({a, a + sizes[i] * bytes(dtypes[i]), i, false});
    spans.push_back({b, b + sizes[i] * bytes(out_dtypes[i]), i, true});
  }
  auto less = [](const Span& x, const Span& y) { return x.at < y.at; };
  if (!std::is_sorted(spans.begin(), spans.end(), less)) std::sort(spans.begin(), spans.end(), less);
  uintptr_t end = 0, out_end = 0;   // of all spans, of outputs
  for (const Span& s : spans) {
    if (s.at < (s.out ? end : out_end))
      return fail(NORMPRE_ERR_ARG, std::string("the clipped values of a gradient share memory with another tensor (gradient ") +
                                       std::to_string(s.i) + ")");
    end = std::max(end, s.end);
    if (s.out) out_end = std::max(out_end, s.end);
  }
  return NORMPRE_OK;
}

template <int N>
void fill(Table<N>* t, int first, int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
          const int* out_dtypes) {
  t->n = 0;
  uint64_t chunks = 0;
  for (int i = first; i < first + n; ++i) {
    if (!sizes[i]) continue;
    const int in_bf16 = dtypes[i] == NORMPRE_BF16;
    t->e[t->n++] = Entry{grads[i], out ? out[i] : nullptr, sizes[i], static_cast<uint32_t>(chunks), static_cast<uint16_t>(in_bf16),
                         static_cast<uint16_t>(out && out_dtypes[i] == NORMPRE_BF16)};
    const int64_t lead = static_cast<int64_t>(reinterpret_cast<uintptr_t>(grads[i]) % 16);
    chunks += static_cast<uint64_t>(cdiv(lead + sizes[i] * (in_bf16 ? 2 : 4), kChunkBytes));
  }
  t->chunks = static_cast<uint32_t>(chunks);
}

int grid_of(uint32_t chunks) {
  const int64_t most = std::min<int64_t>(kMaxCtas, static_cast<int64_t>(device_sm_count()) * kPerSm);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, chunks)));
}

// One launch per table; `scale`: the second pass, which needs all partial sums.
template <int N, typename F>
cudaError_t each_table(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
                       const int* out_dtypes, F launch) {
  Table<N> t;
  for (int first = 0; first == 0 || first < n; first += N) {
    fill(&t, first, std::min(N, n - first), grads, dtypes, sizes, out, out_dtypes);
    launch(t, grid_of(t.chunks));
    const cudaError_t e = cudaGetLastError();
    if (e) return e;
  }
  return cudaSuccess;
}

template <int N>
cudaError_t run(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
                const int* out_dtypes, float max_norm, float eps, float* norm, double* part, cudaStream_t s) {
  int parts = 0;
  cudaError_t e = each_table<N>(n, grads, dtypes, sizes, out, out_dtypes, [&](const Table<N>& t, int grid) {
    k_grad_squares<N><<<grid, kThreads, 0, s>>>(t, part + parts);
    parts += grid;
  });
  if (e) return e;
  if (!out) {
    k_grad_norm<<<1, kThreads, 0, s>>>(part, parts, norm);
    return cudaGetLastError();
  }
  bool in_place = true;
  for (int i = 0; i < n && in_place; ++i) in_place = !sizes[i] || (grads[i] == out[i] && dtypes[i] == out_dtypes[i]);
  return each_table<N>(n, grads, dtypes, sizes, out, out_dtypes, [&](const Table<N>& t, int grid) {
    k_grad_scale<N><<<grid, kThreads, 0, s>>>(t, part, parts, max_norm, eps, in_place, norm);
  });
}

cudaError_t run_any(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
                    const int* out_dtypes, float max_norm, float eps, float* norm, void* workspace, void* stream) {
  double* part = static_cast<double*>(workspace);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return n <= kSmall ? run<kSmall>(n, grads, dtypes, sizes, out, out_dtypes, max_norm, eps, norm, part, s)
                     : run<kLarge>(n, grads, dtypes, sizes, out, out_dtypes, max_norm, eps, norm, part, s);
}

int check_device(float* norm, void* workspace) {
  if (!norm || !workspace) return fail(NORMPRE_ERR_ARG, "norm or workspace: null");
  if (reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(NORMPRE_ERR_ALIGN, "norm must be aligned to 4 bytes and workspace to 16");
  return NORMPRE_OK;
}

}  // namespace
}  // namespace normpre

using namespace normpre;

extern "C" {

int normpre_grad_bytes(int n, int64_t* bytes) {
  if (!bytes) return fail(NORMPRE_ERR_ARG, "null argument");
  if (n < 0 || n > (1 << 20)) return fail(NORMPRE_ERR_ARG, "the number of gradients must be in [0, 2^20]");
  *bytes = max_launches(n) * kMaxCtas * static_cast<int64_t>(sizeof(double));
  return NORMPRE_OK;
}

int normpre_grad_norm(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, float* norm,
                      void* workspace, void* stream) {
  int rc = check_list(n, grads, dtypes, sizes);
  if (rc || (rc = check_device(norm, workspace))) return rc;
  return done(run_any(n, grads, dtypes, sizes, nullptr, nullptr, 0.f, 0.f, norm, workspace, stream), "gradient norm");
}

int normpre_grad_clip(int n, const void* const* grads, const int* dtypes, const int64_t* sizes, void* const* out,
                      const int* out_dtypes, float max_norm, float eps, float* norm, void* workspace, void* stream) {
  int rc = check_list(n, grads, dtypes, sizes);
  if (rc || (rc = check_device(norm, workspace))) return rc;
  if (n && (!out || !out_dtypes)) return fail(NORMPRE_ERR_ARG, "null argument");
  if (!(max_norm >= 0.f) || max_norm == INFINITY) return fail(NORMPRE_ERR_ARG, "max_norm must be finite and >= 0");
  if (!(eps >= 0.f) || eps == INFINITY) return fail(NORMPRE_ERR_ARG, "eps must be finite and >= 0");
  try {
    if ((rc = check_list(n, const_cast<const void* const*>(out), out_dtypes, sizes)) ||
        (rc = check_overlap(n, grads, dtypes, sizes, out, out_dtypes)))
      return rc;
  } catch (const std::bad_alloc&) {
    return fail(NORMPRE_ERR_CUDA, "out of host memory");
  }
  return done(run_any(n, grads, dtypes, sizes, out, out_dtypes, max_norm, eps, norm, workspace, stream), "gradient clipping");
}

}  // extern "C"
