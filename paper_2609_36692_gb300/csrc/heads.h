// [tokens][heads][head_dim] tensors of the C ABI: their checks.
#pragma once

#include <stdint.h>

#include <string>

#include "../../include/normpre.h"
#include "internal.h"

namespace normpre {

// A tensor argument as the kernels take it, strides in elements.
struct HeadsView {
  void* p;
  int64_t ts, hs;
};

// Checks one tensor argument and copies it; a stride that no address uses (a
// single row or head) is replaced by a valid one.  Returns a status and leaves
// the message to normpre_last_error(NULL).
inline int take_heads(const normpre_heads* t, int64_t tokens, int heads, int dim, int dtype, const char* name, bool output,
                      HeadsView* out) {
  auto fail = [&](int code, const char* what) {
    set_thread_error(std::string(name) + what);
    return code;
  };
  if (!t || !t->data) return fail(NORMPRE_ERR_ARG, ": null");
  const int64_t d = dim, per16 = dtype == NORMPRE_BF16 ? 8 : 4;
  int64_t ts = tokens > 1 ? t->token_stride : 0, hs = heads > 1 ? t->head_stride : 0;
  if (tokens > 1 && (ts < d || ts > (int64_t(1) << 30)))
    return fail(NORMPRE_ERR_SHAPE, ": token stride must be in [head_dim, 2^30]");
  if (heads > 1 && (hs < d || hs > (int64_t(1) << 36)))
    return fail(NORMPRE_ERR_SHAPE, ": head stride must be in [head_dim, 2^36]");
  if ((reinterpret_cast<uintptr_t>(t->data) & 15u) || ts % per16 || hs % per16)
    return fail(NORMPRE_ERR_ALIGN, ": data and strides must be multiples of 16 bytes");
  if (output && tokens > 1 && heads > 1) {
    const bool by_token = ts >= hs;   // rows outermost, or heads
    const int64_t inner = by_token ? (heads - 1) * hs + d : (tokens - 1) * ts + d;
    if ((by_token ? ts : hs) < inner) return fail(NORMPRE_ERR_SHAPE, ": overlapping strides");
  }
  if (!ts) ts = round_up(d, 8);
  if (!hs) hs = round_up(d, 8);
  *out = HeadsView{t->data, ts, hs};
  return NORMPRE_OK;
}

}  // namespace normpre
