"""Host-side checks of the attention and checkpoint entry points: arguments are
refused before any CUDA call, and the binding mirrors the header's structs."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def C():
    from paper_2609_36692_gb300 import build
    build.build()
    from paper_2609_36692_gb300 import normpre
    return normpre


def refused(C, status, f, *args):
    with pytest.raises(C.NormPreError) as e:
        f(*args)
    assert e.value.status == status
    assert C.normpre_last_error()


@pytest.mark.parametrize("field, value, status", [
    ("n_heads", 0, "SHAPE"), ("n_heads", 5, "SHAPE"), ("n_kv_heads", 0, "SHAPE"), ("n_kv_heads", 3, "SHAPE"),
    ("head_dim", 0, "SHAPE"), ("head_dim", 12, "SHAPE"), ("head_dim", 136, "SHAPE"), ("max_seqs", 0, "SHAPE"),
    ("max_tokens", 0, "SHAPE"), ("max_tokens", 1 << 25, "SHAPE"), ("dtype", 2, "DTYPE"),
    ("scale", -1.0, "ARG"), ("scale", float("nan"), "ARG"), ("scale", float("inf"), "ARG")])
def test_attention_plan_arguments(C, field, value, status):
    cfg = C.normpre_attn_config(4, 2, 64, 8, 1024, C.NORMPRE_BF16, 0.0)
    setattr(cfg, field, value)
    refused(C, getattr(C, "NORMPRE_ERR_" + status), C.normpre_attn_init, cfg)


def test_null_arguments(C):
    lib = C.load_library()
    assert lib.normpre_attn_init(None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_attn_set_lengths(None, 0, None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_attn_forward(None, 1, None, None, None, None, None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_attn_backward(None, 1, *[None] * 10) == C.NORMPRE_ERR_ARG
    assert lib.normpre_attn_sync_status(None, None) == C.NORMPRE_ERR_ARG
    lib.normpre_attn_free(None)
    assert lib.normpre_ckpt_bytes(1, 1, None, None) == C.NORMPRE_ERR_ARG
    assert lib.normpre_ckpt_pack(1, 1, None, 0, 1, None, None, None) == C.NORMPRE_ERR_ARG


def test_checkpoint_sizes(C):
    assert C.normpre_ckpt_bytes(0, 5) == (0, 0)
    assert C.normpre_ckpt_bytes(3, 1) == (96, 12)
    assert C.normpre_ckpt_bytes(3, 128) == (384, 12)
    assert C.normpre_ckpt_bytes(3, 129) == (480, 24)
    for t, f in ((-1, 4), (1 << 31, 4), (4, 0), (4, (1 << 20) + 1), ((1 << 31) - 1, 1 << 20)):
        refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_ckpt_bytes, t, f)


def test_checkpoint_arguments(C):
    A = 1 << 20    # an aligned address that nothing reads: every call below is refused
    refused(C, C.NORMPRE_ERR_DTYPE, C.normpre_ckpt_pack, 4, 64, A, 2, 64, A, A)
    refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_ckpt_pack, 4, 64, A, 0, 63, A, A)
    refused(C, C.NORMPRE_ERR_ALIGN, C.normpre_ckpt_pack, 4, 64, A + 4, 0, 64, A, A)
    refused(C, C.NORMPRE_ERR_ALIGN, C.normpre_ckpt_pack, 4, 64, A, 0, 64, A + 8, A)
    refused(C, C.NORMPRE_ERR_ALIGN, C.normpre_ckpt_restore, 4, 64, A, A + 1, A, 0, 64)
    refused(C, C.NORMPRE_ERR_ARG, C.normpre_ckpt_restore, 4, 64, A, 0, A, 0, 64)
    refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_ckpt_wgrad, 4, 0, 64, A, 1, 64, A, A, A, 0, 64)
    refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_ckpt_wgrad, 4, 64, 64, A, 1, 63, A, A, A, 0, 64)
    refused(C, C.NORMPRE_ERR_DTYPE, C.normpre_ckpt_wgrad, 4, 64, 64, A, 5, 64, A, A, A, 0, 64)
    refused(C, C.NORMPRE_ERR_ARG, C.normpre_ckpt_wgrad, 4, 64, 64, A, 1, 64, A, A, A, 0, 64, 2)
    refused(C, C.NORMPRE_ERR_ARG, C.normpre_ckpt_swiglu, 4, 64, 0, A, 64, A, 64, A, 64, A, A, A, 0)
    refused(C, C.NORMPRE_ERR_SHAPE, C.normpre_ckpt_swiglu, 4, 64, 0, A, 64, A, 60, A, 64, A, A, A, A)
    refused(C, C.NORMPRE_ERR_DTYPE, C.normpre_ckpt_swiglu_backward, 4, 64, 3, A, A, A, A, A, 64, A, 64, A, 64)
    # nothing to do is not an error
    assert C.normpre_ckpt_pack(0, 64, 0, 0, 64, 0, 0) == C.NORMPRE_OK


@pytest.mark.parametrize("struct", ["normpre_attn_config", "normpre_heads"])
def test_structs_mirror_the_header(C, struct):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "normpre.h")).read(), flags=re.S)
    body = re.search(r"typedef\s+struct\s+%s\s*\{(.*?)\}\s*%s\s*;" % (struct, struct), src, flags=re.S).group(1)
    c_types = {"int": ctypes.c_int, "float": ctypes.c_float, "int64_t": ctypes.c_int64, "void*": ctypes.c_void_p}
    want = [(name, c_types[ty]) for ty, name in re.findall(r"(void\*|\w+)\s+(\w+)\s*;", body)]
    assert getattr(C, struct)._fields_ == want
