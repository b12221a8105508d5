// 8-bit activation checkpoints: pack, restore and the gated activation that
// writes and reads them, with the normpre_ckpt_* entry points.
//
// All of these stream: each value is read once and each result written once.
// A CTA takes 128 features (a panel) of 64 rows; 8 lanes share a row, 16
// features each, so that a warp reads and writes whole 32-byte sectors of 4
// rows, the maximum of a 32-element block needs one shuffle, and the steps of
// consecutive rows (one 32-bit word per row and panel) leave in whole sectors.
// Bound by HBM: 16384 x 6144 bf16, pack and restore 0.102 ms (6.0 TB/s), the
// gated activation and its gradient 0.268 ms (6.1 TB/s; a copy runs at 6.8).
// Small calls are bound by the launch.
#include <atomic>
#include <cstring>
#include <string>

#include "../../include/normpre.h"
#include "ckpt.h"
#include "common.cuh"
#include "internal.h"

namespace normpre {
namespace {

constexpr int kRows = 64;        // rows of a CTA
constexpr int kThreads = 256;

// 16 consecutive elements as they lie in memory, `n` of which exist.  A thread
// fetches all that it will work on before it converts any of it, so that its
// reads are in flight together.
template <bool VEC, typename T> struct Raw16 {
  uint4 q[sizeof(T)];   // 16 elements: 16 sizeof(T) bytes
  __device__ __forceinline__ void fetch(const T* p, int n) {
    if (VEC && n >= 16) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) q[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    } else {
      T v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = i < n ? p[i] : from_f32<T>(0.f);
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) q[i] = pack(v + 16 / sizeof(T) * i);
    }
  }
  __device__ __forceinline__ void values(float (&v)[16]) const {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) {
      const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
          v[4 * i + e] = __uint_as_float(w[e]);
        } else {
          v[8 * i + 2 * e] = bf16lo(w[e]);
          v[8 * i + 2 * e + 1] = bf16hi(w[e]);
        }
      }
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ __forceinline__ uint4 pack(const bf16* v) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = static_cast<uint32_t>(__bfloat16_as_ushort(v[2 * e])) |
             (static_cast<uint32_t>(__bfloat16_as_ushort(v[2 * e + 1])) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <bool VEC, typename T>
__device__ __forceinline__ void store16(T* p, int n, const float (&v)[16]) {
  if (VEC && n >= 16) {
    store8(p, v);
    store8(p + 8, v + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// Rounds a lane's 16 elements of a row to codes and returns the row's step
// word of the panel in the first of its 8 lanes.  The step exponent e is the
// least with max |x| <= 127 * 2^e: with 2^f <= max < 2^(f+1), f - 6 if the
// significand is at most 127/64, else f - 5.
__device__ __forceinline__ uint32_t encode16(const float (&v)[16], uint4& codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const bool finite = top < 0x7F800000u;
  const int byte = finite ? max(1, static_cast<int>(top >> 23) - 6 + ((top & 0x7FFFFFu) > 0x7E0000u ? 1 : 0)) : 255;
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - byte) << 23);   // 2^-e
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = static_cast<uint32_t>(__float2int_rn(v[4 * i + j] * inv)) & 0xFFu;
    w[i] = finite ? b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24) : 0u;
  }
  codes = make_uint4(w[0], w[1], w[2], w[3]);
  // lanes 0, 2, 4, 6 of the row hold its four blocks
  uint32_t word = static_cast<uint32_t>(byte);
  word |= __shfl_down_sync(0xffffffffu, word, 2) << 8;
  word |= __shfl_down_sync(0xffffffffu, word, 4) << 16;
  return word;
}

__device__ __forceinline__ void decode16(const uint4& codes, float step, float (&v)[16]) {
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(static_cast<int8_t>(w[i >> 2] >> (8 * (i & 3)))) * step;
}

// A lane's place: row of the CTA's pass, feature, and what exists there.
struct Place {
  int64_t row;
  int64_t feature;
  int64_t word;   // index of the row's step word of the panel
  int n;          // elements of the lane's 16 that exist
  bool codes;     // the lane's codes (padding included) exist
};
__device__ __forceinline__ Place place(int64_t tokens, int64_t features, int64_t ld, int pass) {
  Place p;
  const unsigned panels = static_cast<unsigned>((features + kCkptPanel - 1) / kCkptPanel);
  const unsigned range = blockIdx.x / panels, panel = blockIdx.x - range * panels;
  p.row = static_cast<int64_t>(range) * kRows + pass * 32 + (threadIdx.x >> 3);
  p.feature = static_cast<int64_t>(panel) * kCkptPanel + (threadIdx.x & 7) * 16;
  p.word = panel * tokens + p.row;
  const bool in = p.row < tokens;
  p.codes = in && p.feature < ld;
  p.n = in ? static_cast<int>(max(int64_t(0), min(int64_t(16), features - p.feature))) : 0;
  return p;
}

struct PackArgs {
  int64_t tokens, features, ld;
  const void* x;
  int64_t x_ld;
  int8_t* codes;
  uint32_t* steps;
};

constexpr int kPasses = kRows / 32;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_ckpt_pack(const __grid_constant__ PackArgs a) {
  Place p[kPasses];
  Raw16<VEC, T> x[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    p[i] = place(a.tokens, a.features, a.ld, i);
    x[i].fetch(static_cast<const T*>(a.x) + p[i].row * a.x_ld + p[i].feature, p[i].n);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    float v[16];
    x[i].values(v);
    uint4 codes;
    const uint32_t word = encode16(v, codes);
    if (p[i].codes) *reinterpret_cast<uint4*>(a.codes + p[i].row * a.ld + p[i].feature) = codes;
    if ((threadIdx.x & 7) == 0 && p[i].row < a.tokens) a.steps[p[i].word] = word;
  }
}

// The codes and step of a lane's 16 elements.
struct Coded {
  uint4 codes;
  uint32_t word;
  __device__ __forceinline__ void fetch(const int8_t* codes_, const uint32_t* steps, int64_t ld, const Place& p) {
    codes = make_uint4(0, 0, 0, 0);
    word = 0;
    if (!p.n) return;
    codes = __ldcs(reinterpret_cast<const uint4*>(codes_ + p.row * ld + p.feature));
    word = __ldg(steps + p.word);
  }
  __device__ __forceinline__ void values(float (&v)[16]) const { decode16(codes, ckpt_step(word, (threadIdx.x & 7) >> 1), v); }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_ckpt_restore(const __grid_constant__ PackArgs a, T* y) {
  Place p[kPasses];
  Coded c[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    p[i] = place(a.tokens, a.features, a.ld, i);
    c[i].fetch(a.codes, a.steps, a.ld, p[i]);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    float v[16];
    c[i].values(v);
    if (p[i].n) store16<VEC>(y + p[i].row * a.x_ld + p[i].feature, p[i].n, v);
  }
}

struct SwigluArgs {
  int64_t tokens, features, ld;
  const void *gate, *up, *dh;
  void *h, *dgate, *dup;
  int64_t gate_ld, up_ld, h_ld, dgate_ld, dup_ld, dh_ld;
  int8_t *gate_codes, *up_codes;
  uint32_t *gate_steps, *up_steps;
};

// s = 1 / (1 + exp(-x)) in x, 1 - s in y, to a few units in the last place: from
// exp(-|x|), which cannot overflow, and a divisor in [1, 2].
__device__ __forceinline__ float2 sigmoids(float x) {
  const float e = expf(-fabsf(x)), r = __fdividef(1.f, 1.f + e);
  return x < 0.f ? make_float2(e * r, r) : make_float2(r, e * r);
}
// bf16 takes the hardware's exponential, whose relative error (1e-5 at |x| = 88)
// is far below the rounding that follows; the exact one makes its kernels 12 %
// slower (16384 x 6144, both passes: 301 us, not 268).
template <typename T> __device__ __forceinline__ float sigmoid(float x) {
  if constexpr (sizeof(T) == 4) return sigmoids(x).x;
  else return __fdividef(1.f, 1.f + __expf(-x));
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_ckpt_swiglu(const __grid_constant__ SwigluArgs a) {
  Place p[kPasses];
  Raw16<VEC, T> gr[kPasses], ur[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    p[i] = place(a.tokens, a.features, a.ld, i);
    gr[i].fetch(static_cast<const T*>(a.gate) + p[i].row * a.gate_ld + p[i].feature, p[i].n);
    ur[i].fetch(static_cast<const T*>(a.up) + p[i].row * a.up_ld + p[i].feature, p[i].n);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    float g[16], u[16];
    gr[i].values(g);
    ur[i].values(u);
    uint4 gc, uc;
    const uint32_t gw = encode16(g, gc), uw = encode16(u, uc);
    if (p[i].codes) {
      *reinterpret_cast<uint4*>(a.gate_codes + p[i].row * a.ld + p[i].feature) = gc;
      *reinterpret_cast<uint4*>(a.up_codes + p[i].row * a.ld + p[i].feature) = uc;
    }
    if ((threadIdx.x & 7) == 0 && p[i].row < a.tokens) {
      a.gate_steps[p[i].word] = gw;
      a.up_steps[p[i].word] = uw;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) u[e] *= g[e] * sigmoid<T>(g[e]);
    store16<VEC>(static_cast<T*>(a.h) + p[i].row * a.h_ld + p[i].feature, p[i].n, u);
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_ckpt_swiglu_bwd(const __grid_constant__ SwigluArgs a) {
  Place p[kPasses];
  Raw16<VEC, T> dr[kPasses];
  Coded gr[kPasses], ur[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    p[i] = place(a.tokens, a.features, a.ld, i);
    dr[i].fetch(static_cast<const T*>(a.dh) + p[i].row * a.dh_ld + p[i].feature, p[i].n);
    gr[i].fetch(a.gate_codes, a.gate_steps, a.ld, p[i]);
    ur[i].fetch(a.up_codes, a.up_steps, a.ld, p[i]);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    float g[16], u[16], d[16];
    dr[i].values(d);
    gr[i].values(g);
    ur[i].values(u);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float s = sigmoid<T>(g[e]);
      u[e] *= d[e] * s * fmaf(g[e], sizeof(T) == 4 ? sigmoids(g[e]).y : 1.f - s, 1.f);
      g[e] *= d[e] * s;
    }
    store16<VEC>(static_cast<T*>(a.dgate) + p[i].row * a.dgate_ld + p[i].feature, p[i].n, u);
    store16<VEC>(static_cast<T*>(a.dup) + p[i].row * a.dup_ld + p[i].feature, p[i].n, g);
  }
}

// A word of flags per device in pinned memory: kernels set it, the entry points
// read it.  The first call of a process that needs one allocates them (also
// within a stream capture, where an allocation otherwise counts as unsafe).
constexpr int kMaxDevices = 64;
std::atomic<int*> g_flags{nullptr};

cudaError_t ckpt_flags(int** out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e) return e;
  if (dev >= kMaxDevices) return cudaErrorInvalidDevice;
  int* p = g_flags.load(std::memory_order_acquire);
  if (!p) {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    if ((e = cudaThreadExchangeStreamCaptureMode(&mode))) return e;
    void* v = nullptr;
    e = cudaHostAlloc(&v, kMaxDevices * sizeof(int), cudaHostAllocPortable);
    if (!e) {
      std::memset(v, 0, kMaxDevices * sizeof(int));
      if (g_flags.compare_exchange_strong(p, static_cast<int*>(v), std::memory_order_acq_rel)) p = static_cast<int*>(v);
      else cudaFreeHost(v);   // another thread was first: p is its words
    }
    cudaThreadExchangeStreamCaptureMode(&mode);
    if (e) return e;
  }
  *out = p + dev;
  return cudaSuccess;
}
int flags_now(const int* p) { return *static_cast<const volatile int*>(p); }

int fail(int code, const std::string& msg) {
  set_thread_error(msg);
  return code;
}
int done(cudaError_t e, const char* what) {
  return e ? fail(NORMPRE_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e)) : NORMPRE_OK;
}

// One CTA per panel and kRows rows, the panels of a row range next to each other.
int64_t panel_ctas(int64_t tokens, int64_t features) { return ckpt_panels(features) * cdiv(tokens, kRows); }

int check_shape(int64_t tokens, int64_t features) {
  if (tokens < 0 || tokens >= (int64_t(1) << 31) || features < 1 || features > (int64_t(1) << 20))
    return fail(NORMPRE_ERR_SHAPE, "tokens must be in [0, 2^31) and features in [1, 2^20]");
  if (panel_ctas(tokens, features) >= (int64_t(1) << 31)) return fail(NORMPRE_ERR_SHAPE, "the matrix is too large");
  return NORMPRE_OK;
}
int check_dtype(int dtype, const char* name) {
  if (dtype != NORMPRE_F32 && dtype != NORMPRE_BF16)
    return fail(NORMPRE_ERR_DTYPE, std::string(name) + ": dtype must be NORMPRE_F32 or NORMPRE_BF16");
  return NORMPRE_OK;
}
int check_ptr(const void* p, const char* name) {
  if (!p) return fail(NORMPRE_ERR_ARG, std::string(name) + ": null");
  if (reinterpret_cast<uintptr_t>(p) & 15u) return fail(NORMPRE_ERR_ALIGN, std::string(name) + " must be 16-byte aligned");
  return NORMPRE_OK;
}
int check_matrix(const void* p, int64_t ld, int64_t cols, const char* name) {
  if (ld < cols || ld > (int64_t(1) << 31))
    return fail(NORMPRE_ERR_SHAPE, std::string(name) + ": the row stride must be in [columns, 2^31]");
  return check_ptr(p, name);
}
// Rows on 16-byte boundaries: whole-vector accesses.
bool vec_rows(int64_t ld, int dtype) { return ld % (dtype == NORMPRE_BF16 ? 8 : 4) == 0; }

}  // namespace
}  // namespace normpre

using namespace normpre;

#define CKPT_TRY(x)      \
  do {                   \
    const int rc_ = (x); \
    if (rc_) return rc_; \
  } while (0)

// kernel<T, VEC> for a dtype and whether every row starts on 16 bytes
#define CKPT_DISPATCH(kernel, dtype, vec, ...)                                   \
  do {                                                                           \
    if ((dtype) == NORMPRE_F32) {                                                \
      if (vec) kernel<float, true> __VA_ARGS__; else kernel<float, false> __VA_ARGS__; \
    } else {                                                                     \
      if (vec) kernel<bf16, true> __VA_ARGS__; else kernel<bf16, false> __VA_ARGS__;   \
    }                                                                            \
  } while (0)

extern "C" {

int normpre_ckpt_bytes(int64_t tokens, int64_t features, int64_t* codes_bytes, int64_t* steps_bytes) {
  CKPT_TRY(check_shape(tokens, features));
  if (!codes_bytes || !steps_bytes) return fail(NORMPRE_ERR_ARG, "null argument");
  *codes_bytes = tokens * ckpt_ld(features);
  *steps_bytes = 4 * tokens * ckpt_panels(features);
  return NORMPRE_OK;
}

int normpre_ckpt_pack(int64_t tokens, int64_t features, const void* x, int x_dtype, int64_t x_ld, void* codes,
                      void* steps, void* stream) {
  CKPT_TRY(check_shape(tokens, features));
  CKPT_TRY(check_dtype(x_dtype, "x"));
  if (!tokens) return NORMPRE_OK;
  CKPT_TRY(check_matrix(x, x_ld, features, "x"));
  CKPT_TRY(check_ptr(codes, "codes"));
  CKPT_TRY(check_ptr(steps, "steps"));
  PackArgs a = {tokens, features, ckpt_ld(features), x, x_ld, static_cast<int8_t*>(codes), static_cast<uint32_t*>(steps)};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(panel_ctas(tokens, features));
  CKPT_DISPATCH(k_ckpt_pack, x_dtype, vec_rows(x_ld, x_dtype), <<<grid, kThreads, 0, s>>>(a));
  return done(cudaGetLastError(), "checkpoint pack");
}

int normpre_ckpt_restore(int64_t tokens, int64_t features, const void* codes, const void* steps, void* y,
                         int y_dtype, int64_t y_ld, void* stream) {
  CKPT_TRY(check_shape(tokens, features));
  CKPT_TRY(check_dtype(y_dtype, "y"));
  if (!tokens) return NORMPRE_OK;
  CKPT_TRY(check_ptr(codes, "codes"));
  CKPT_TRY(check_ptr(steps, "steps"));
  CKPT_TRY(check_matrix(y, y_ld, features, "y"));
  PackArgs a = {tokens, features, ckpt_ld(features), nullptr, y_ld,
                const_cast<int8_t*>(static_cast<const int8_t*>(codes)),
                const_cast<uint32_t*>(static_cast<const uint32_t*>(steps))};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(panel_ctas(tokens, features));
  const bool vec = vec_rows(y_ld, y_dtype);
  if (y_dtype == NORMPRE_F32) {
    if (vec) k_ckpt_restore<float, true><<<grid, kThreads, 0, s>>>(a, static_cast<float*>(y));
    else k_ckpt_restore<float, false><<<grid, kThreads, 0, s>>>(a, static_cast<float*>(y));
  } else {
    if (vec) k_ckpt_restore<bf16, true><<<grid, kThreads, 0, s>>>(a, static_cast<bf16*>(y));
    else k_ckpt_restore<bf16, false><<<grid, kThreads, 0, s>>>(a, static_cast<bf16*>(y));
  }
  return done(cudaGetLastError(), "checkpoint restore");
}

int normpre_ckpt_wgrad(int64_t tokens, int64_t out_features, int64_t features, const void* dy, int dy_dtype,
                       int64_t dy_ld, const void* codes, const void* steps, void* dw, int dw_dtype, int64_t dw_ld,
                       int accumulate, void* stream) {
  CKPT_TRY(check_shape(tokens, features));
  if (out_features < 1 || out_features > (int64_t(1) << 20))
    return fail(NORMPRE_ERR_SHAPE, "out_features must be in [1, 2^20]");
  CKPT_TRY(check_dtype(dy_dtype, "dy"));
  CKPT_TRY(check_dtype(dw_dtype, "dw"));
  if (accumulate != 0 && accumulate != 1) return fail(NORMPRE_ERR_ARG, "accumulate must be 0 or 1");
  CKPT_TRY(check_matrix(dw, dw_ld, features, "dw"));
  if (tokens) {
    CKPT_TRY(check_matrix(dy, dy_ld, out_features, "dy"));
    CKPT_TRY(check_ptr(codes, "codes"));
    CKPT_TRY(check_ptr(steps, "steps"));
  } else if (accumulate) {
    return NORMPRE_OK;
  }
  WgradArgs a = {};
  a.dy = dy;
  a.dy_ld = dy_ld;
  a.x = CkptView{static_cast<const int8_t*>(codes), static_cast<const uint32_t*>(steps)};
  a.x_ld = ckpt_ld(features);
  a.dw = dw;
  a.dw_ld = dw_ld;
  a.tokens = tokens;
  a.n = static_cast<int>(out_features);
  a.k = static_cast<int>(features);
  a.accumulate = accumulate;
  cudaError_t e = ckpt_flags(&a.flags);
  if (!e && (flags_now(a.flags) & kFlagTimeout))
    return fail(NORMPRE_ERR_TIMEOUT, "a bounded device wait of an earlier weight gradient gave up: what that call wrote has "
                                     "no meaning (normpre_ckpt_sync_status clears this)");
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  std::string err;
  if (!e) e = tokens && dy_dtype == NORMPRE_BF16 && vec_rows(dy_ld, dy_dtype)
                  ? launch_ckpt_wgrad_tc(a, dw_dtype, s, &err)
                  : launch_ckpt_wgrad_simt(a, dy_dtype, dw_dtype, s);
  return done(e, err.empty() ? "checkpoint weight gradient" : err.c_str());
}

int normpre_ckpt_swiglu(int64_t tokens, int64_t features, int dtype, const void* gate, int64_t gate_ld,
                        const void* up, int64_t up_ld, void* h, int64_t h_ld, void* gate_codes, void* gate_steps,
                        void* up_codes, void* up_steps, void* stream) {
  CKPT_TRY(check_shape(tokens, features));
  CKPT_TRY(check_dtype(dtype, "gate, up and h"));
  if (!tokens) return NORMPRE_OK;
  CKPT_TRY(check_matrix(gate, gate_ld, features, "gate"));
  CKPT_TRY(check_matrix(up, up_ld, features, "up"));
  CKPT_TRY(check_matrix(h, h_ld, features, "h"));
  CKPT_TRY(check_ptr(gate_codes, "gate_codes"));
  CKPT_TRY(check_ptr(gate_steps, "gate_steps"));
  CKPT_TRY(check_ptr(up_codes, "up_codes"));
  CKPT_TRY(check_ptr(up_steps, "up_steps"));
  SwigluArgs a = {};
  a.tokens = tokens; a.features = features; a.ld = ckpt_ld(features);
  a.gate = gate; a.gate_ld = gate_ld;
  a.up = up; a.up_ld = up_ld;
  a.h = h; a.h_ld = h_ld;
  a.gate_codes = static_cast<int8_t*>(gate_codes); a.gate_steps = static_cast<uint32_t*>(gate_steps);
  a.up_codes = static_cast<int8_t*>(up_codes); a.up_steps = static_cast<uint32_t*>(up_steps);
  const bool vec = vec_rows(gate_ld, dtype) && vec_rows(up_ld, dtype) && vec_rows(h_ld, dtype);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(panel_ctas(tokens, features));
  CKPT_DISPATCH(k_ckpt_swiglu, dtype, vec, <<<grid, kThreads, 0, s>>>(a));
  return done(cudaGetLastError(), "checkpoint swiglu");
}

int normpre_ckpt_swiglu_backward(int64_t tokens, int64_t features, int dtype, const void* gate_codes,
                                 const void* gate_steps, const void* up_codes, const void* up_steps, const void* dh,
                                 int64_t dh_ld, void* dgate, int64_t dgate_ld, void* dup, int64_t dup_ld,
                                 void* stream) {
  CKPT_TRY(check_shape(tokens, features));
  CKPT_TRY(check_dtype(dtype, "dh, dgate and dup"));
  if (!tokens) return NORMPRE_OK;
  CKPT_TRY(check_matrix(dh, dh_ld, features, "dh"));
  CKPT_TRY(check_matrix(dgate, dgate_ld, features, "dgate"));
  CKPT_TRY(check_matrix(dup, dup_ld, features, "dup"));
  CKPT_TRY(check_ptr(gate_codes, "gate_codes"));
  CKPT_TRY(check_ptr(gate_steps, "gate_steps"));
  CKPT_TRY(check_ptr(up_codes, "up_codes"));
  CKPT_TRY(check_ptr(up_steps, "up_steps"));
  SwigluArgs a = {};
  a.tokens = tokens; a.features = features; a.ld = ckpt_ld(features);
  a.dh = dh; a.dh_ld = dh_ld;
  a.dgate = dgate; a.dgate_ld = dgate_ld;
  a.dup = dup; a.dup_ld = dup_ld;
  a.gate_codes = const_cast<int8_t*>(static_cast<const int8_t*>(gate_codes));
  a.gate_steps = const_cast<uint32_t*>(static_cast<const uint32_t*>(gate_steps));
  a.up_codes = const_cast<int8_t*>(static_cast<const int8_t*>(up_codes));
  a.up_steps = const_cast<uint32_t*>(static_cast<const uint32_t*>(up_steps));
  const bool vec = vec_rows(dh_ld, dtype) && vec_rows(dgate_ld, dtype) && vec_rows(dup_ld, dtype);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(panel_ctas(tokens, features));
  CKPT_DISPATCH(k_ckpt_swiglu_bwd, dtype, vec, <<<grid, kThreads, 0, s>>>(a));
  return done(cudaGetLastError(), "checkpoint swiglu backward");
}

int normpre_ckpt_sync_status(void* stream) {
  int* flags = nullptr;
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (!e) e = ckpt_flags(&flags);
  if (e) return done(e, "normpre_ckpt_sync_status");
  const int v = flags_now(flags);
  if (v) *static_cast<volatile int*>(flags) = 0;
  return v & kFlagTimeout ? fail(NORMPRE_ERR_TIMEOUT, "a bounded device wait gave up") : NORMPRE_OK;
}

}  // extern "C"
