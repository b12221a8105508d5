"""Training operators around the optimizer step, on torch tensors: packed
causal attention and 8-bit activation checkpoints.

Like ``optim``, this only checks tensors and hands their pointers and the
current CUDA stream to the C ABI (``normpre_attn_*``, ``normpre_ckpt_*`` in
``include/normpre.h``, which has the definitions); all arithmetic runs in the
library's kernels.  ``PackedAttention.__call__``, ``linear`` and ``swiglu`` are
the differentiable forms; they have first derivatives only, and asking for
another one raises.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import normpre as C

_CODES = {torch.float32: C.NORMPRE_F32, torch.bfloat16: C.NORMPRE_BF16}
# The handle of a device's current stream, without the Stream object around it
# (a tenth of a microsecond instead of two).
_current_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _dtype_code(x: torch.Tensor) -> int:
    code = _CODES.get(x.dtype)
    if code is None:
        raise TypeError("unsupported dtype %s (float32 or bfloat16)" % x.dtype)
    return code


def _on(device: torch.device, f, *args) -> None:
    """f(*args, stream) with `device` current, on its current stream."""
    index = device.index
    if _current_device() == index:
        f(*args, _current_stream(index))
    else:
        with torch.cuda.device(index):
            f(*args, _current_stream(index))


def _used_on(stream, *tensors) -> None:
    # the memory of a tensor that is freed while another stream than its own
    # still works on it must wait for that stream before it is given out again
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _empty(shape, dtype, device: torch.device, stream) -> torch.Tensor:
    """An output that work on `stream` (None: the current one) writes.  It comes
    from that stream's own pool: memory of the current stream's may still be
    read or written by what was queued there before."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        x = torch.empty(shape, dtype=dtype, device=device)
    x.record_stream(torch.cuda.current_stream(device))
    return x


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

    With `stream`, a call's work runs there instead of on the current stream;
    the caller orders it after what wrote its inputs and lengths, and before
    what reads its outputs.
    """

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int, max_seqs: int,
                 dtype: torch.dtype = torch.bfloat16, scale: float = 0.0, device=None):
        index = None if device is None else torch.device(device).index
        self.device = torch.device("cuda", torch.cuda.current_device() if index is None else index)
        self.dtype, self.n_heads, self.n_kv_heads, self.head_dim = dtype, n_heads, n_kv_heads, head_dim
        code = _CODES.get(dtype)
        if code is None:
            raise TypeError("unsupported dtype %s (float32 or bfloat16)" % dtype)
        self.plan, self.lengths = None, ()
        cfg = C.normpre_attn_config(n_heads, n_kv_heads, head_dim, max_seqs, max_tokens, code, scale)
        with torch.cuda.device(self.device):
            self.plan = C.normpre_attn_init(cfg)

    def set_lengths(self, lengths: Sequence[int], stream=None) -> None:
        lengths = tuple(int(n) for n in lengths)
        with torch.cuda.device(self.device):
            s = stream if stream is not None else torch.cuda.current_stream()
            C.normpre_attn_set_lengths(self.plan, lengths, s.cuda_stream)
        self.lengths = lengths

    def _check(self, x: torch.Tensor, name: str, tokens: int, heads: int):
        if x.device != self.device:
            raise ValueError("%s must be on %s" % (name, self.device))
        if x.dtype != self.dtype:
            raise TypeError("%s must be %s" % (name, self.dtype))
        if x.shape != (tokens, heads, self.head_dim):
            raise ValueError("%s must be [%d, %d, %d] (got %s)" % (name, tokens, heads, self.head_dim, tuple(x.shape)))
        st, sh, sd = x.stride()
        if sd != 1 and tokens:
            raise ValueError("%s: the last dimension must be contiguous" % name)
        return x.data_ptr(), st, sh

    def _lse(self, lse: torch.Tensor, tokens: int) -> int:
        if lse.device != self.device or lse.dtype != torch.float32 or not lse.is_contiguous() or \
                lse.shape != (self.n_heads, tokens):
            raise ValueError("lse must be a contiguous float32 [%d, %d] tensor on %s" % (self.n_heads, tokens, self.device))
        return lse.data_ptr()

    def _new(self, tokens: int, heads: int, stream):
        return _empty((tokens, heads, self.head_dim), self.dtype, self.device, stream)

    def forward(self, q, k, v, out=None, lse=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out, lse): [tokens, n_heads, head_dim] and the fp32 log-sums
        [n_heads, tokens] that ``backward`` reads."""
        t, h, hk = q.shape[0], self.n_heads, self.n_kv_heads
        check = self._check
        args = (*check(q, "q", t, h), *check(k, "k", t, hk), *check(v, "v", t, hk))
        _used_on(stream, q, k, v, out, lse)
        if out is None:
            out = self._new(t, h, stream)
        if lse is None:
            lse = _empty((h, t), torch.float32, self.device, stream)
        heads = (ctypes.c_int64 * 12)(*args, *check(out, "out", t, h))
        at = ctypes.addressof(heads)
        C.normpre_attn_forward(self.plan, t, at, at + 24, at + 48, at + 72, self._lse(lse, t),
                               _current_stream(self.device.index) if stream is None else stream.cuda_stream)
        return out, lse

    def backward(self, q, k, v, out, lse, dout, dq=None, dk=None, dv=None, stream=None):
        """(dq, dk, dv) for the forward pass that gave ``out`` and ``lse``."""
        t, h, hk = q.shape[0], self.n_heads, self.n_kv_heads
        check = self._check
        args = (*check(q, "q", t, h), *check(k, "k", t, hk), *check(v, "v", t, hk), *check(out, "out", t, h),
                *check(dout, "dout", t, h))
        _used_on(stream, q, k, v, out, lse, dout, dq, dk, dv)
        if dq is None:
            dq = self._new(t, h, stream)
        if dk is None:
            dk = self._new(t, hk, stream)
        if dv is None:
            dv = self._new(t, hk, stream)
        heads = (ctypes.c_int64 * 24)(*args, *check(dq, "dq", t, h), *check(dk, "dk", t, hk), *check(dv, "dv", t, hk))
        at = ctypes.addressof(heads)
        C.normpre_attn_backward(self.plan, t, at, at + 24, at + 48, at + 72, self._lse(lse, t), at + 96, at + 120,
                                at + 144, at + 168,
                                _current_stream(self.device.index) if stream is None else stream.cuda_stream)
        return dq, dk, dv

    def __call__(self, q, k, v) -> torch.Tensor:
        """Differentiable attention.  A backward pass runs with the plan's
        lengths: they must be its call's (else it raises)."""
        return _Attention.apply(self, q, k, v)

    def status(self, stream=None, raise_on_error: bool = True) -> int:
        """Synchronizes, and reports and clears what the plan's kernels flagged.
        A flag that is not cleared makes the plan's next call raise."""
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
        ctx.plan, ctx.lengths = plan, plan.lengths
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        if ctx.lengths != ctx.plan.lengths:
            raise RuntimeError("the plan's lengths changed between an attention call and its backward pass; give "
                               "set_lengths the call's lengths again, or use a plan for each batch in flight")
        # autograd may hand over an expanded gradient
        return (None, *ctx.plan.backward(q, k, v, out, lse, _aligned(dout)))


# ---------------------------------------------------------------------------
# 8-bit activation checkpoints
# ---------------------------------------------------------------------------
class Checkpoint:
    """A [tokens, features] matrix kept in 8 bits (``normpre_ckpt_pack``):
    ``codes`` and ``steps`` in one allocation."""

    __slots__ = ("data", "tokens", "features", "dtype", "device", "nbytes", "codes_ptr", "steps_ptr")

    def __init__(self, tokens: int, features: int, dtype: torch.dtype, device: torch.device,
                 data: Optional[torch.Tensor] = None):
        # the sizes of normpre_ckpt_bytes; the codes' is a multiple of 32, so the steps are aligned too
        codes = tokens * ((features + 31) // 32 * 32)
        self.nbytes = codes + 4 * tokens * ((features + 127) // 128)
        self.data = torch.empty(self.nbytes, dtype=torch.uint8, device=device) if data is None else data
        self.tokens, self.features, self.dtype, self.device = tokens, features, dtype, device
        self.codes_ptr = self.data.data_ptr()
        self.steps_ptr = self.codes_ptr + codes

    @property
    def codes(self) -> torch.Tensor:
        return self.data[:self.steps_ptr - self.codes_ptr].view(torch.int8)

    @property
    def steps(self) -> torch.Tensor:
        return self.data[self.steps_ptr - self.codes_ptr:]

    def restore(self, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The values it stands for, in the dtype of what was packed by default."""
        if out is None:
            out = torch.empty((self.tokens, self.features), dtype=dtype or self.dtype, device=self.device)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError("out must be %s" % dtype)
        ld = _matrix(out, "out", (self.tokens, self.features), self.device)
        _on(self.device, C.normpre_ckpt_restore, self.tokens, self.features, self.codes_ptr, self.steps_ptr,
            out.data_ptr(), _dtype_code(out), ld)
        return out


def _matrix(x: torch.Tensor, name: str, shape=None, device=None) -> int:
    """Checks a 2-D tensor and returns its row stride."""
    if not x.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if x.dim() != 2 or (shape is not None and x.shape != shape):
        raise ValueError("%s must be %s (got %s)" % (name, list(shape) if shape is not None else "a matrix", tuple(x.shape)))
    if device is not None and x.device != device:
        raise ValueError("%s must be on %s" % (name, device))
    rows, cols = x.shape
    ld, step = x.stride()
    if cols > 1 and step != 1:
        raise ValueError("%s: rows must be contiguous" % name)
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError("%s: rows must not overlap" % name)
    return ld


def ckpt_pack(x: torch.Tensor) -> Checkpoint:
    """The 8-bit checkpoint of a [tokens, features] matrix (fp32 or bf16)."""
    ld, code = _matrix(x, "x"), _dtype_code(x)
    t, f = x.shape
    ck = Checkpoint(t, f, x.dtype, x.device)
    _on(ck.device, C.normpre_ckpt_pack, t, f, x.data_ptr(), code, ld, ck.codes_ptr, ck.steps_ptr)
    return ck


def ckpt_wgrad(dy: torch.Tensor, ck: Checkpoint, dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """dW = dY^T xhat, [out_features, features]: the weight gradient of
    y = x W^T from x's checkpoint; added to ``out`` with ``accumulate``.  bf16 dY
    whose rows start on 16-byte boundaries runs on the tensor cores; fp32 dY and
    other row strides (an odd out_features) on fp32 units, 30 to 60 times
    slower."""
    ld = _matrix(dy, "dy", (ck.tokens, dy.shape[1] if dy.dim() == 2 else -1), ck.device)
    shape = (dy.shape[1], ck.features)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty(shape, dtype=dtype or dy.dtype, device=ck.device)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError("out must be %s" % dtype)
    out_ld = _matrix(out, "out", shape, ck.device)
    _on(ck.device, C.normpre_ckpt_wgrad, ck.tokens, shape[0], shape[1], dy.data_ptr(), _dtype_code(dy), ld,
        ck.codes_ptr, ck.steps_ptr, out.data_ptr(), _dtype_code(out), out_ld, accumulate)
    return out


def ckpt_swiglu(gate: torch.Tensor, up: torch.Tensor):
    """(h, gate's checkpoint, up's checkpoint) with h = silu(gate) * up."""
    gl = _matrix(gate, "gate")
    ul = _matrix(up, "up", gate.shape, gate.device)
    if up.dtype != gate.dtype:
        raise TypeError("gate and up must have one dtype")
    code, device = _dtype_code(gate), gate.device
    t, f = gate.shape
    h = torch.empty((t, f), dtype=gate.dtype, device=device)
    cg, cu = Checkpoint(t, f, gate.dtype, device), Checkpoint(t, f, gate.dtype, device)
    _on(device, C.normpre_ckpt_swiglu, t, f, code, gate.data_ptr(), gl, up.data_ptr(), ul, h.data_ptr(), f,
        cg.codes_ptr, cg.steps_ptr, cu.codes_ptr, cu.steps_ptr)
    return h, cg, cu


def ckpt_swiglu_backward(gate: Checkpoint, up: Checkpoint, dh: torch.Tensor):
    """(dgate, dup) from the checkpoints that ``ckpt_swiglu`` gave."""
    t, f = gate.tokens, gate.features
    if (up.tokens, up.features) != (t, f) or up.device != gate.device:
        raise ValueError("the checkpoints' shapes or devices differ")
    ld, code = _matrix(dh, "dh", (t, f), gate.device), _dtype_code(dh)
    dgate = torch.empty((t, f), dtype=dh.dtype, device=gate.device)
    dup = torch.empty((t, f), dtype=dh.dtype, device=gate.device)
    _on(gate.device, C.normpre_ckpt_swiglu_backward, t, f, code, gate.codes_ptr, gate.steps_ptr, up.codes_ptr,
        up.steps_ptr, dh.data_ptr(), ld, dgate.data_ptr(), f, dup.data_ptr(), f)
    return dgate, dup


def ckpt_status(stream=None, raise_on_error: bool = True) -> int:
    """Synchronizes, and reports and clears the checkpoint kernels' flag.  A flag
    that is not cleared makes the next weight gradient raise."""
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
        ctx.ck = ckpt_pack(_rows(x.reshape(-1, x.shape[-1])))
        ctx.save_for_backward(weight)
        return x @ weight.to(x.dtype).t()

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        weight, = ctx.saved_tensors
        dx = dy @ weight.to(dy.dtype) if ctx.needs_input_grad[0] else None
        dw = ckpt_wgrad(_rows(dy.reshape(-1, dy.shape[-1])), ctx.ck, dtype=weight.dtype) if ctx.needs_input_grad[1] else None
        return dx, dw


def linear(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """Differentiable y = x W^T, x [..., features], that keeps x in 8 bits for
    its backward pass; the weight gradient comes in the weight's dtype.  Nothing
    is kept where there will be none.  The weight gradient is this library's
    kernel; y and x's gradient are torch's matrix products."""
    if not (torch.is_grad_enabled() and weight.requires_grad):
        return x @ weight.to(x.dtype).t()
    return _Linear.apply(x, weight)


class _SwiGLU(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, up):
        h, ctx.gate, ctx.up = ckpt_swiglu(_rows(gate), _rows(up))
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        return ckpt_swiglu_backward(ctx.gate, ctx.up, _rows(dh))


def swiglu(gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
    """Differentiable silu(gate) * up that keeps gate and up in 8 bits."""
    return _SwiGLU.apply(gate, up)
