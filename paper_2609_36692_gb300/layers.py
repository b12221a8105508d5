"""Training operators around the optimizer step, on torch tensors: packed
causal attention and 8-bit activation checkpoints.

Like ``optim``, this only checks tensors and hands their pointers and the
current CUDA stream to the C ABI (``normpre_attn_*``, ``normpre_ckpt_*`` in
``include/normpre.h``, which has the definitions); all arithmetic runs in the
library's kernels.  ``PackedAttention.__call__``, ``linear`` and ``swiglu`` are
the differentiable forms.
"""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

import torch

from . import normpre as C
from .optim import _dtype_code


def _stream(x: torch.Tensor, stream=None) -> int:
    return (stream if stream is not None else torch.cuda.current_stream(x.device)).cuda_stream


def _cuda(x: torch.Tensor, name: str) -> torch.Tensor:
    if not x.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    return x


def _used_on(stream, *tensors) -> None:
    # tensors allocated here belong to the current stream's allocator pool;
    # tell it about another stream that works on them
    if stream is not None:
        for t in tensors:
            t.record_stream(stream)


# ---------------------------------------------------------------------------
# packed causal attention
# ---------------------------------------------------------------------------
class PackedAttention:
    """Causal attention over packs of up to ``max_seqs`` sequences in up to
    ``max_tokens`` rows, ``n_heads`` query heads in groups that share
    ``n_kv_heads`` key / value heads.

    ``set_lengths`` takes a batch's sequence lengths (once per batch); every
    layer's ``forward`` / ``backward``, or the differentiable call
    ``plan(q, k, v)``, then uses them.  q is [tokens, n_heads, head_dim], k and
    v [tokens, n_kv_heads, head_dim]: any views whose last dimension is
    contiguous and whose strides are multiples of 16 bytes.  Rows past the last
    sequence give zero outputs and gradients.
    """

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int, max_seqs: int,
                 dtype: torch.dtype = torch.bfloat16, scale: float = 0.0, device=None):
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.dtype, self.n_heads, self.n_kv_heads, self.head_dim = dtype, n_heads, n_kv_heads, head_dim
        code = {torch.float32: C.NORMPRE_F32, torch.bfloat16: C.NORMPRE_BF16}.get(dtype)
        if code is None:
            raise TypeError("unsupported dtype %s (float32 or bfloat16)" % dtype)
        self.plan = None
        cfg = C.normpre_attn_config(n_heads, n_kv_heads, head_dim, max_seqs, max_tokens, code, scale)
        with torch.cuda.device(self.device):
            self.plan = C.normpre_attn_init(cfg)

    def set_lengths(self, lengths: Sequence[int], stream=None) -> None:
        with torch.cuda.device(self.device):
            s = stream if stream is not None else torch.cuda.current_stream()
            C.normpre_attn_set_lengths(self.plan, lengths, s.cuda_stream)

    def _heads(self, x: torch.Tensor, heads: int, name: str, tokens: Optional[int] = None) -> C.normpre_heads:
        if x.device != self.device:
            raise ValueError("%s must be on %s" % (name, self.device))
        if x.dtype != self.dtype:
            raise TypeError("%s must be %s" % (name, self.dtype))
        if x.dim() != 3 or x.shape[1] != heads or x.shape[2] != self.head_dim or \
                (tokens is not None and x.shape[0] != tokens):
            raise ValueError("%s must be [%s, %d, %d] (got %s)" % (name, tokens if tokens is not None else "tokens",
                                                                   heads, self.head_dim, tuple(x.shape)))
        if x.shape[0] and x.stride(2) != 1:
            raise ValueError("%s: the last dimension must be contiguous" % name)
        return C.normpre_heads(x.data_ptr(), x.stride(0), x.stride(1))

    def _lse(self, lse: torch.Tensor, tokens: int) -> int:
        if lse.device != self.device or lse.dtype != torch.float32 or not lse.is_contiguous() or \
                tuple(lse.shape) != (self.n_heads, tokens):
            raise ValueError("lse must be a contiguous float32 [%d, %d] tensor on %s" % (self.n_heads, tokens, self.device))
        return lse.data_ptr()

    def _new(self, given, tokens: int, heads: int, stream):
        if given is None:
            given = torch.empty(tokens, heads, self.head_dim, dtype=self.dtype, device=self.device)
            _used_on(stream, given)
        return given

    def forward(self, q, k, v, out=None, lse=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out, lse): [tokens, n_heads, head_dim] and the fp32 log-sums
        [n_heads, tokens] that ``backward`` reads."""
        t = q.shape[0]
        args = [self._heads(q, self.n_heads, "q"), self._heads(k, self.n_kv_heads, "k", t),
                self._heads(v, self.n_kv_heads, "v", t)]
        out = self._new(out, t, self.n_heads, stream)
        if lse is None:
            lse = torch.empty(self.n_heads, t, dtype=torch.float32, device=self.device)
            _used_on(stream, lse)
        C.normpre_attn_forward(self.plan, t, *args, self._heads(out, self.n_heads, "out", t), self._lse(lse, t),
                               _stream(q, stream))
        return out, lse

    def backward(self, q, k, v, out, lse, dout, dq=None, dk=None, dv=None, stream=None):
        """(dq, dk, dv) for the forward pass that gave ``out`` and ``lse``."""
        t = q.shape[0]
        h, hk = self.n_heads, self.n_kv_heads
        args = [self._heads(q, h, "q"), self._heads(k, hk, "k", t), self._heads(v, hk, "v", t),
                self._heads(out, h, "out", t)]
        do = self._heads(dout, h, "dout", t)
        dq, dk, dv = self._new(dq, t, h, stream), self._new(dk, t, hk, stream), self._new(dv, t, hk, stream)
        C.normpre_attn_backward(self.plan, t, *args, self._lse(lse, t), do, self._heads(dq, h, "dq", t),
                                self._heads(dk, hk, "dk", t), self._heads(dv, hk, "dv", t), _stream(q, stream))
        return dq, dk, dv

    def __call__(self, q, k, v) -> torch.Tensor:
        """Differentiable attention.  The lengths must not change between a
        call and its backward pass."""
        return _Attention.apply(self, q, k, v)

    def status(self, stream=None, raise_on_error: bool = True) -> int:
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        return C.normpre_attn_sync_status(self.plan, s.cuda_stream, raise_on_error)

    def close(self) -> None:
        if self.plan:
            C.normpre_attn_free(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _aligned(x: torch.Tensor) -> torch.Tensor:
    """x itself where the kernels take its layout, else a contiguous copy."""
    per16 = 16 // x.element_size()
    if x.numel() == 0 or (x.stride(2) == 1 and x.data_ptr() % 16 == 0 and
                          all(x.shape[i] == 1 or (x.stride(i) % per16 == 0 and x.stride(i) >= x.shape[2])
                              for i in (0, 1))):
        return x
    return x.contiguous()


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, q, k, v):
        out, lse = plan.forward(q, k, v)
        ctx.plan = plan
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        # autograd may hand over an expanded gradient
        return (None, *ctx.plan.backward(q, k, v, out, lse, _aligned(dout)))


# ---------------------------------------------------------------------------
# 8-bit activation checkpoints
# ---------------------------------------------------------------------------
class Checkpoint:
    """A [tokens, features] matrix kept in 8 bits (``normpre_ckpt_pack``)."""

    def __init__(self, codes: torch.Tensor, steps: torch.Tensor, tokens: int, features: int, dtype: torch.dtype):
        self.codes, self.steps, self.tokens, self.features, self.dtype = codes, steps, tokens, features, dtype

    @classmethod
    def empty(cls, tokens: int, features: int, dtype: torch.dtype, device) -> "Checkpoint":
        nc, ns = C.normpre_ckpt_bytes(tokens, features)
        return cls(torch.empty(nc, dtype=torch.int8, device=device), torch.empty(ns, dtype=torch.uint8, device=device),
                   tokens, features, dtype)

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.steps.numel()

    def restore(self, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The values it stands for, in the dtype of what was packed by default."""
        if out is None:
            out = torch.empty(self.tokens, self.features, dtype=dtype or self.dtype, device=self.codes.device)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError("out must be %s" % dtype)
        ld = _matrix(out, "out", (self.tokens, self.features))
        with torch.cuda.device(out.device):
            C.normpre_ckpt_restore(self.tokens, self.features, self.codes.data_ptr(), self.steps.data_ptr(),
                                   out.data_ptr(), _dtype_code(out), ld, _stream(out))
        return out


def _matrix(x: torch.Tensor, name: str, shape=None, device=None) -> int:
    """Checks a 2-D tensor and returns its row stride."""
    _cuda(x, name)
    if x.dim() != 2 or (shape is not None and tuple(x.shape) != tuple(shape)):
        raise ValueError("%s must be %s (got %s)" % (name, list(shape) if shape is not None else "a matrix", tuple(x.shape)))
    if device is not None and x.device != device:
        raise ValueError("%s must be on %s" % (name, device))
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError("%s: rows must be contiguous" % name)
    if x.shape[0] > 1 and x.stride(0) < x.shape[1]:
        raise ValueError("%s: rows must not overlap" % name)
    _dtype_code(x)
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def ckpt_pack(x: torch.Tensor) -> Checkpoint:
    """The 8-bit checkpoint of a [tokens, features] matrix (fp32 or bf16)."""
    ld = _matrix(x, "x")
    ck = Checkpoint.empty(x.shape[0], x.shape[1], x.dtype, x.device)
    with torch.cuda.device(x.device):
        C.normpre_ckpt_pack(ck.tokens, ck.features, x.data_ptr(), _dtype_code(x), ld, ck.codes.data_ptr(),
                            ck.steps.data_ptr(), _stream(x))
    return ck


def ckpt_wgrad(dy: torch.Tensor, ck: Checkpoint, dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """dW = dY^T xhat, [out_features, features]: the weight gradient of
    y = x W^T from x's checkpoint; added to ``out`` with ``accumulate``."""
    ld = _matrix(dy, "dy", (ck.tokens, dy.shape[1] if dy.dim() == 2 else -1), ck.codes.device)
    shape = (dy.shape[1], ck.features)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty(shape, dtype=dtype or dy.dtype, device=dy.device)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError("out must be %s" % dtype)
    out_ld = _matrix(out, "out", shape, dy.device)
    with torch.cuda.device(dy.device):
        C.normpre_ckpt_wgrad(ck.tokens, shape[0], shape[1], dy.data_ptr(), _dtype_code(dy), ld, ck.codes.data_ptr(),
                             ck.steps.data_ptr(), out.data_ptr(), _dtype_code(out), out_ld, accumulate, _stream(dy))
    return out


def ckpt_swiglu(gate: torch.Tensor, up: torch.Tensor):
    """(h, gate's checkpoint, up's checkpoint) with h = silu(gate) * up."""
    gl = _matrix(gate, "gate")
    ul = _matrix(up, "up", gate.shape, gate.device)
    if up.dtype != gate.dtype:
        raise TypeError("gate and up must have one dtype")
    t, f = gate.shape
    h = torch.empty(t, f, dtype=gate.dtype, device=gate.device)
    cg = Checkpoint.empty(t, f, gate.dtype, gate.device)
    cu = Checkpoint.empty(t, f, gate.dtype, gate.device)
    with torch.cuda.device(gate.device):
        C.normpre_ckpt_swiglu(t, f, _dtype_code(gate), gate.data_ptr(), gl, up.data_ptr(), ul, h.data_ptr(), f,
                              cg.codes.data_ptr(), cg.steps.data_ptr(), cu.codes.data_ptr(), cu.steps.data_ptr(),
                              _stream(gate))
    return h, cg, cu


def ckpt_swiglu_backward(gate: Checkpoint, up: Checkpoint, dh: torch.Tensor):
    """(dgate, dup) from the checkpoints that ``ckpt_swiglu`` gave."""
    t, f = gate.tokens, gate.features
    if (up.tokens, up.features) != (t, f):
        raise ValueError("the checkpoints' shapes differ")
    ld = _matrix(dh, "dh", (t, f), gate.codes.device)
    dgate, dup = torch.empty_like(dh, memory_format=torch.contiguous_format), \
        torch.empty_like(dh, memory_format=torch.contiguous_format)
    with torch.cuda.device(dh.device):
        C.normpre_ckpt_swiglu_backward(t, f, _dtype_code(dh), gate.codes.data_ptr(), gate.steps.data_ptr(),
                                       up.codes.data_ptr(), up.steps.data_ptr(), dh.data_ptr(), ld, dgate.data_ptr(),
                                       f, dup.data_ptr(), f, _stream(dh))
    return dgate, dup


def ckpt_status(stream=None, raise_on_error: bool = True) -> int:
    """Synchronizes and reports the checkpoint kernels' device flag."""
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.normpre_ckpt_sync_status(s.cuda_stream, raise_on_error)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """A matrix the kernels take: x, or a contiguous copy."""
    ok = x.data_ptr() % 16 == 0 and (x.shape[1] <= 1 or x.stride(1) == 1) and \
        (x.shape[0] <= 1 or x.stride(0) >= x.shape[1])
    return x if ok else x.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        ctx.ck = ckpt_pack(_rows(x))
        ctx.save_for_backward(weight)
        return x @ weight.to(x.dtype).t()

    @staticmethod
    def backward(ctx, dy):
        weight, = ctx.saved_tensors
        dy = _rows(dy)
        dx = dy @ weight.to(dy.dtype) if ctx.needs_input_grad[0] else None
        dw = ckpt_wgrad(dy, ctx.ck, dtype=weight.dtype) if ctx.needs_input_grad[1] else None
        return dx, dw


def linear(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """Differentiable y = x W^T that keeps x in 8 bits for its backward pass;
    the weight gradient comes in the weight's dtype."""
    return _Linear.apply(x, weight)


class _SwiGLU(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, up):
        h, ctx.gate, ctx.up = ckpt_swiglu(_rows(gate), _rows(up))
        return h

    @staticmethod
    def backward(ctx, dh):
        return ckpt_swiglu_backward(ctx.gate, ctx.up, _rows(dh))


def swiglu(gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
    """Differentiable silu(gate) * up that keeps gate and up in 8 bits."""
    return _SwiGLU.apply(gate, up)
