"""Host-side checks of the query and key norms and of gradient clipping: arguments are refused before any CUDA call."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest

import test_layers_cpu as base
from test_layers_cpu import C, refused  # noqa: F401

A = 1 << 20    # an aligned address that nothing reads: every call below is refused


def rotary(C, **kw):
    cfg = C.normpre_qkrot_config(4, 2, 64, 32, 0, 1, C.NORMPRE_BF16, 1e-6)
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("field, value, status", [
    ("n_heads", 0, "SHAPE"), ("n_kv_heads", 0, "SHAPE"), ("n_heads", 65536, "SHAPE"), ("head_dim", 0, "SHAPE"),
    ("head_dim", 12, "SHAPE"), ("head_dim", 136, "SHAPE"), ("rotary_dim", -2, "SHAPE"), ("rotary_dim", 66, "SHAPE"),
    ("rotary_dim", 31, "SHAPE"), ("interleaved", 2, "ARG"), ("norm", -1, "ARG"), ("dtype", 2, "DTYPE"), ("eps", 0.0, "ARG"),
    ("eps", -1.0, "ARG"), ("eps", math.nan, "ARG"), ("eps", math.inf, "ARG")])
def test_rotary_plan_arguments(C, field, value, status):
    cfg = rotary(C, **{field: value})
    refused(C, getattr(C, "NORMPRE_ERR_" + status), C.normpre_qkrot_init, cfg, [1.0] * max(0, cfg.rotary_dim // 2))


def test_rotary_frequencies(C):
    for bad in (math.nan, math.inf, 1e7):
        refused(C, C.NORMPRE_ERR_ARG, C.normpre_qkrot_init, rotary(C), [1.0] * 15 + [bad])
    with pytest.raises(ValueError, match="frequencies"):
        C.normpre_qkrot_init(rotary(C), [1.0] * 15)
    h = ctypes.c_void_p()
    assert C.load_library().normpre_qkrot_init(ctypes.byref(rotary(C)), None, ctypes.byref(h)) == C.NORMPRE_ERR_ARG
    assert not h.value


def test_rotary_call_arguments(C):
    plan = C.normpre_qkrot_init(rotary(C), [0.5] * 16)
    bare = C.normpre_qkrot_init(rotary(C, norm=0, eps=0.0), [0.5] * 16)
    q, k = C.normpre_heads(A, 256, 64), C.normpre_heads(A, 128, 64)
    good = dict(plan=plan, tokens=5, used=5, q=q, k=k, positions=A, position_bytes=8, q_weight=A, k_weight=A, weight_dtype=0,
                q_out=q, k_out=k)
    more = dict(dq_out=q, dk_out=k, dq=q, dk=k, dq_weight=A, dk_weight=A, workspace=A)
    bad = [("SHAPE", dict(tokens=-1)), ("SHAPE", dict(tokens=(1 << 30) + 1)), ("SHAPE", dict(used=6)), ("SHAPE", dict(used=-1)),
           ("DTYPE", dict(position_bytes=2)), ("DTYPE", dict(weight_dtype=2)), ("ARG", dict(positions=0)),
           ("ALIGN", dict(positions=A + 4)), ("ALIGN", dict(q_weight=A + 2)), ("ARG", dict(q=C.normpre_heads(0, 256, 64))),
           ("ALIGN", dict(q=C.normpre_heads(A + 8, 256, 64))), ("ALIGN", dict(k=C.normpre_heads(A, 132, 64))),
           ("SHAPE", dict(k=C.normpre_heads(A, 32, 64))), ("ARG", dict(plan=bare))]
    for status, change in bad + [("SHAPE", dict(q_out=C.normpre_heads(A, 64, 64)))]:
        refused(C, getattr(C, "NORMPRE_ERR_" + status), C.normpre_qkrot_forward, *{**good, **change}.values())
    base = {n: v for n, v in good.items() if n not in ("q_out", "k_out")}
    for status, change in bad + [("ARG", dict(workspace=0)), ("ALIGN", dict(workspace=A + 8)), ("ALIGN", dict(dq_weight=A + 2)),
                                 ("ARG", dict(q_weight=0)), ("SHAPE", dict(dk=C.normpre_heads(A, 64, 64)))]:
        refused(C, getattr(C, "NORMPRE_ERR_" + status), C.normpre_qkrot_backward, *{**base, **more, **change}.values())
    assert C.normpre_qkrot_bytes(plan) > 0
    lib = C.load_library()
    assert lib.normpre_qkrot_init(None, None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_qkrot_bytes(None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_qkrot_forward(None, 1, 1, *[None] * 3, 8, None, None, 0, None, None, None) == C.NORMPRE_ERR_ARG
    # nothing to do is not an error
    assert C.normpre_qkrot_forward(*{**good, "tokens": 0, "used": 0}.values()) == C.NORMPRE_OK
    for p in (plan, bare, 0):
        C.normpre_qkrot_free(p)


def test_clip_arguments(C):
    norm = lambda g, t, s, n=A, w=A: C.normpre_grad_norm(g, t, s, n, w)  # noqa: E731
    for status, args in (("DTYPE", ([A], [2], [4])), ("SHAPE", ([A], [0], [-1])), ("SHAPE", ([A], [0], [(1 << 40) + 1])),
                         ("SHAPE", ([A] * 3, [0] * 3, [1 << 39] * 3)), ("ARG", ([0], [0], [4])), ("ALIGN", ([A + 2], [0], [4])),
                         ("ALIGN", ([A + 1], [1], [4])), ("ARG", ([A], [0], [4], 0)), ("ARG", ([A], [0], [4], A, 0)),
                         ("ALIGN", ([A], [0], [4], A + 2)), ("ALIGN", ([A], [0], [4], A, A + 8))):
        refused(C, getattr(C, "NORMPRE_ERR_" + status), norm, *args)
    clip = lambda out, t=(0,), limit=1.0, eps=0.0: C.normpre_grad_clip([A], [0], [64], out, t, limit, eps, A, A)  # noqa: E731
    for status, args in (("ARG", ([0],)), ("DTYPE", ([A], [3])), ("ALIGN", ([A + 2],)), ("ARG", ([A + 4],)), ("ARG", ([A - 4],)),
                         ("ARG", ([A], [1])), ("ARG", ([A], [0], -1.0)), ("ARG", ([A], [0], math.nan)),
                         ("ARG", ([A], [0], 1.0, -1e-9)), ("ARG", ([A], [0], 1.0, math.inf))):
        refused(C, getattr(C, "NORMPRE_ERR_" + status), clip, *args)
    assert C.normpre_grad_bytes(0) > 0 and C.normpre_grad_bytes(5000) % 16 == 0
    refused(C, C.NORMPRE_ERR_ARG, C.normpre_grad_bytes, -1)
    lib = C.load_library()
    assert lib.normpre_grad_norm(1, None, None, None, A, A, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_grad_bytes(1, None) == C.NORMPRE_ERR_ARG


@pytest.mark.parametrize("struct", ["normpre_qkrot_config"])
def test_structs(C, struct):
    base.test_structs_mirror_the_header(C, struct)


@pytest.mark.parametrize("window, sinks", [(-1, 0), (0, -1), (100, -5)])
def test_window_arguments(C, window, sinks):
    cfg = C.normpre_attn_config(4, 2, 64, 8, 1024, C.NORMPRE_BF16, 0.0)
    refused(C, C.NORMPRE_ERR_ARG, C.normpre_attn_init_window, cfg, window, sinks)
    cfg.head_dim = 12
    refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_attn_init_window, cfg, 10, 1)
    assert C.load_library().normpre_attn_init_window(None, 0, 0, None) == C.NORMPRE_ERR_ARG


SPANS = r"""
#include <algorithm>
#include <cstdio>
#include "attn.h"
using namespace normpre;
// whether some row of the query block sees some key of the key block
static bool meets(int i, int j, int len, int w, int s) {
  for (int q = 128 * i; q < std::min(len, 128 * i + 128); ++q)
    for (int k = 128 * j; k < std::min(len, 128 * j + 128); ++k)
      if (k <= q && (q - k < w || k < s)) return true;
  return false;
}
int main() {
  int bad = 0;
  for (int len : {1, 128, 129, 600, 1025})
    for (int w : {1, 2, 127, 128, 129, 256, 300, 1 << 25})
      for (int s : {0, 1, 128, 129, 300, 2000})
        for (int b = 0, n = (len + 127) / 128; b < n; ++b) {
          const KeySpan k = key_span(b, w, s);
          int down = 0, up = 0, last = b;
          for (int j = b; j >= 0; j = k.down(j), ++down) bad += !meets(b, j, 1 << 20, w, s);
          for (int j = k.first(); j <= b; j = k.up(j), ++up) bad += !meets(b, j, 1 << 20, w, s);
          int all = 0;
          for (int j = 0; j <= b; ++j) all += meets(b, j, 1 << 20, w, s);
          bad += all != down || all != up || all != k.count(b);
          for (int i = b; i < n; ++i)
            if (meets(i, b, 1 << 20, w, s)) last = i;
          bad += last_query(b, len, w, s) != last;
          // the parts of its queries follow one another, from its own block to the last
          AttnBlock e = {0, len, b, 0};
          const KeyPart whole = key_part(e, w, s, 3, 0);
          bad += whole.slot != -1 || !whole.fits || whole.first != b || whole.end != last + 1;
          for (int chunk : {1, 2, 3, 8}) {
            const int parts = key_parts(last - b + 1, chunk);
            for (int i = 0, at = b; i < parts; ++i) {
              e.part = i << 12 | (i + 6);
              const KeyPart k = key_part(e, w, s, chunk, 100);
              bad += !k.fits || k.slot != i + 5 || k.first != at || k.end <= k.first || k.end - k.first > chunk;
              at = k.end;
              bad += i + 1 == parts && at != last + 1;
            }
            e.part = parts << 12 | 1;                       // what is not of the call is known as such
            bad += key_part(e, w, s, chunk, 100).fits;
            e.part = 0 << 12 | 101;
            bad += key_part(e, w, s, chunk, 100).fits;
          }
          e.part = 1;
          bad += key_part(e, w, s, 0, 100).fits;
          e.part = -1;
          bad += key_part(e, w, s, 2, 100).fits;
        }
  std::printf("%d\n", bad);
}
"""


@pytest.mark.skipif(not shutil.which("g++") or not os.path.exists("/usr/local/cuda/include/cuda_runtime.h"),
                    reason="needs g++ and the CUDA headers")
def test_spans(tmp_path):
    """Which blocks of keys and queries meet, against all their pairs of rows."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SPANS)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I/usr/local/cuda/include",
                    "-I" + os.path.join(base.ROOT, "paper_2609_36692_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.strip() == "0"
