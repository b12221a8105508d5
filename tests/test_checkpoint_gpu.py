"""8-bit activation checkpoints on the GPU against their definition.

Pack and restore are exact: the expected codes, steps and values are computed
in 64 bits and must match to the bit.  The weight gradient sums products of
numbers that are exact in bf16: fp32 sums of n terms with random signs stay
within a few times sqrt(n) 2^-24 of the result, below 1e-5 relative Frobenius
error for the sizes here; a bf16 result adds one rounding, at most 2^-8 (8 significant bits).  The gated
activation's arithmetic costs a few fp32 roundings (1e-6) and the same last
rounding.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (64, 128), (65, 127), (37, 1001), (130, 257), (200, 768), (2, 5504)]


def dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def definition(x):
    """Codes (int), biased steps (uint8; 255 non-finite) and values in 64 bits."""
    x = np.asarray(x, np.float64)
    t, f = x.shape
    nb = -(-f // 32)
    y = np.zeros((t, nb * 32))
    y[:, :f] = x
    y = y.reshape(t, nb, 32)
    bad = ~np.isfinite(y).all(-1)
    top = np.abs(np.where(np.isfinite(y), y, 0)).max(-1)
    e = np.full((t, nb), -126, dtype=int)
    for cand in range(-126, 130):                      # the least e that holds
        e = np.where(top > 127.0 * 2.0 ** e, cand + 1, e)
    codes = np.where(bad[..., None], 0, np.rint(np.where(bad[..., None], 0, y) / 2.0 ** e[..., None]))
    values = np.where(bad[..., None], np.nan, codes * 2.0 ** e[..., None])
    return codes.reshape(t, -1).astype(int), np.where(bad, 255, e + 127), values.reshape(t, -1)[:, :f]


def sample(seed, t, f, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, f, generator=g, device="cuda") * torch.exp(2 * torch.randn(f, generator=g, device="cuda"))
    return x.to(dt(dtype))


def rel(x, ref):
    import torch
    ref = torch.as_tensor(ref, device=x.device, dtype=torch.float64)
    n = torch.linalg.norm(ref)
    e = torch.linalg.norm(x.double() - ref)
    return float(e / n) if float(n) > 0 else float(e)


def unpacked(ck):
    """Codes and step bytes of a checkpoint as [tokens, blocks * 32] / [tokens, blocks]."""
    t, f = ck.tokens, ck.features
    nb = -(-f // 32)
    codes = ck.codes.view(t, nb * 32).cpu().numpy().astype(int)
    steps = ck.steps.view(-(-f // 128), t, 4).permute(1, 0, 2).reshape(t, -1).cpu().numpy().astype(int)
    assert (steps[:, nb:] == 1).all()
    return codes, steps[:, :nb]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_pack_and_restore(shape, dtype):
    import torch
    from paper_2609_36692_gb300 import layers as L
    x = sample(sum(shape), *shape, dtype)
    ck = L.ckpt_pack(x)
    codes, steps, values = definition(x.float().cpu().numpy())
    got_codes, got_steps = unpacked(ck)
    assert np.array_equal(got_codes, codes) and np.array_equal(got_steps, steps)
    for out in ("f32", "bf16"):
        assert np.array_equal(ck.restore(dt(out)).float().cpu().numpy(), values.astype(np.float32))
    assert ck.restore().dtype == x.dtype and torch.equal(ck.restore(), L.ckpt_pack(x).restore())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_at_the_edges(dtype):
    """Ties, maxima on both sides of 127 steps, zeros, subnormals, the largest
    numbers, and non-finite values, which mark their own block only."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    rows = []
    for top in (127.0, 127.5, 128.0, 63.5, 64.0, 126.9, 3.3e38, 2.0 ** -126, 2.0 ** -133, 2.0 ** -140, 0.0, 1e-30):
        r = np.zeros(96)
        r[:32] = top * np.linspace(-1, 1, 32)
        r[32:64] = np.arange(32) + 0.5
        r[32] = 127.0                           # step 1: halves are ties
        r[64] = -top
        rows.append(r)
    x = torch.tensor(np.array(rows), dtype=torch.float64).to(torch.float32).to(dt(dtype)).cuda()
    for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
        x[i, 40 + i] = bad
    ck = L.ckpt_pack(x)
    codes, steps, values = definition(x.double().cpu().numpy())
    got_codes, got_steps = unpacked(ck)
    assert np.array_equal(got_codes, codes) and np.array_equal(got_steps, steps)
    assert np.array_equal(ck.restore(torch.float32).cpu().numpy(), values.astype(np.float32), equal_nan=True)
    assert bool(torch.isnan(ck.restore(torch.float32)[:3, 32:64]).all())
    assert bool(torch.isfinite(ck.restore(torch.float32)[:3, :32]).all())


def test_packed_error_is_half_a_step():
    import torch
    from paper_2609_36692_gb300 import layers as L
    x = sample(1, 300, 768, "f32")
    d = (L.ckpt_pack(x).restore() - x).abs().view(300, 24, 32).amax(-1)
    assert bool((d <= x.abs().view(300, 24, 32).amax(-1) / 127).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows(dtype):
    import torch
    from paper_2609_36692_gb300 import layers as L
    x = sample(2, 77, 203, dtype)
    for pad in (5, 53):                              # off and on 16-byte row boundaries
        wide = torch.zeros(77, 203 + pad, dtype=x.dtype, device="cuda")
        wide[:, :203] = x
        a, b = L.ckpt_pack(x), L.ckpt_pack(wide[:, :203])
        assert torch.equal(a.codes, b.codes) and torch.equal(a.steps, b.steps)
        wide.fill_(7)
        assert torch.equal(b.restore(out=wide[:, :203]), a.restore())
        assert bool((wide[:, 203:] == 7).all())


WGRAD = [(1, 64, 64), (2, 8, 33), (63, 72, 130), (64, 128, 128), (65, 136, 100), (200, 129, 257), (500, 768, 768),
         (1000, 256, 2048), (129, 1, 1), (700, 520, 1000), (4096, 264, 392)]


@pytest.mark.parametrize("dy_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dw_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", WGRAD, ids=str)
def test_weight_gradient(shape, dy_dtype, dw_dtype):
    import torch
    from paper_2609_36692_gb300 import layers as L
    t, n, f = shape
    x = sample(t + n, t, f, "bf16")
    dy = sample(f, t, n, dy_dtype)
    ck = L.ckpt_pack(x)
    ref = dy.double().T @ ck.restore(torch.float32).double()
    tol = 1e-5 + (2.0 ** -8 if dw_dtype == "bf16" else 0)
    dw = L.ckpt_wgrad(dy, ck, dtype=dt(dw_dtype))
    assert L.ckpt_status() == 0
    assert rel(dw, ref) <= tol
    assert torch.equal(dw, L.ckpt_wgrad(dy, ck, dtype=dt(dw_dtype)))       # the same bits again
    # accumulation, into rows of a wider buffer
    wide = torch.full((n, f + 13), 3.0, dtype=dt(dw_dtype), device="cuda")
    start = sample(9, n, f, dw_dtype)
    wide[:, :f] = start
    L.ckpt_wgrad(dy, ck, out=wide[:, :f], accumulate=True)
    assert rel(wide[:, :f], ref + start.double()) <= tol
    assert bool((wide[:, f:] == 3.0).all())


@pytest.mark.parametrize("dy_dtype", ["f32", "bf16"])
def test_weight_gradient_of_strided_rows(dy_dtype):
    import torch
    from paper_2609_36692_gb300 import layers as L
    ck = L.ckpt_pack(sample(3, 300, 200, "bf16"))
    dy = sample(4, 300, 264, dy_dtype)
    ref = dy.double().T @ ck.restore(torch.float32).double()
    for pad in (3, 8, 64):
        wide = torch.full((300, 264 + pad), float("nan"), dtype=dy.dtype, device="cuda")
        wide[:, :264] = dy
        assert rel(L.ckpt_wgrad(wide[:, :264], ck, dtype=torch.float32), ref) <= 1e-5


def test_weight_gradient_without_tokens():
    import torch
    from paper_2609_36692_gb300 import layers as L
    ck = L.ckpt_pack(torch.empty(0, 40, device="cuda"))
    dy = torch.empty(0, 24, device="cuda", dtype=torch.bfloat16)
    out = torch.full((24, 40), 5.0, device="cuda")
    L.ckpt_wgrad(dy, ck, out=out, accumulate=True)
    assert bool((out == 5.0).all())
    L.ckpt_wgrad(dy, ck, out=out)
    assert not bool(out.any())
    assert ck.restore().shape == (0, 40)


@pytest.mark.parametrize("dy_dtype", ["f32", "bf16"])
def test_weight_gradient_non_finite(dy_dtype):
    """A non-finite block of the checkpoint, or a non-finite dY, reaches the
    features (rows) it belongs to and no others."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    x, dy = sample(5, 150, 256, "bf16"), sample(6, 150, 200, dy_dtype)
    x[40, 70] = float("inf")
    dw = L.ckpt_wgrad(dy, L.ckpt_pack(x), dtype=torch.float32)
    assert bool(torch.isnan(dw[:, 64:96]).all())
    assert bool(torch.isfinite(dw[:, :64]).all()) and bool(torch.isfinite(dw[:, 96:]).all())
    x[40, 70] = 1.0
    dy[7, 9] = float("nan")
    dw = L.ckpt_wgrad(dy, L.ckpt_pack(x), dtype=torch.float32)
    assert bool(torch.isnan(dw[9]).all())
    dw[9] = 0
    assert bool(torch.isfinite(dw).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_swiglu(shape, dtype):
    import torch
    from paper_2609_36692_gb300 import layers as L
    gate, up, dh = (sample(i, *shape, dtype) for i in (1, 2, 3))
    gate = (gate.float().clamp(-90, 90)).to(dt(dtype))
    h, cg, cu = L.ckpt_swiglu(gate, up)
    for ck, x in ((cg, gate), (cu, up)):
        want = L.ckpt_pack(x)
        assert torch.equal(ck.codes, want.codes) and torch.equal(ck.steps, want.steps)
    tol = 2e-6 if dtype == "f32" else 2.0 ** -8 + 2e-6
    g, u = gate.double(), up.double()
    assert rel(h, g * torch.sigmoid(g) * u) <= tol
    g, u, d = cg.restore(torch.float32).double(), cu.restore(torch.float32).double(), dh.double()
    s = torch.sigmoid(g)
    dgate, dup = L.ckpt_swiglu_backward(cg, cu, dh)
    assert rel(dgate, d * u * s * (1 + g * (1 - s))) <= tol
    assert rel(dup, d * g * s) <= tol


def test_swiglu_gradient_against_differences():
    """Inputs that a checkpoint keeps exactly (whole numbers over 16): the
    backward pass is then the forward's derivative.  fp64 differences of the
    formula, step 1e-6."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    g = torch.Generator(device="cuda").manual_seed(4)
    gate, up = (torch.randint(-60, 61, (20, 96), generator=g, device="cuda").float() / 16 for _ in range(2))
    dh = torch.randn(20, 96, generator=g, device="cuda")
    h, cg, cu = L.ckpt_swiglu(gate, up)
    assert torch.equal(cg.restore(), gate) and torch.equal(cu.restore(), up)
    dgate, dup = L.ckpt_swiglu_backward(cg, cu, dh)
    f = lambda a, b: a * torch.sigmoid(a) * b  # noqa: E731
    a, b, e = gate.double(), up.double(), 1e-6
    assert rel(h, f(a, b)) <= 2e-6
    assert rel(dgate, dh.double() * (f(a + e, b) - f(a - e, b)) / (2 * e)) <= 1e-5
    assert rel(dup, dh.double() * (f(a, b + e) - f(a, b - e)) / (2 * e)) <= 1e-5


def test_differentiable_forms():
    import torch
    from paper_2609_36692_gb300 import layers as L
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(100, 96, generator=g, device="cuda").to(torch.bfloat16).requires_grad_()
    w1, w2 = (torch.randn(160, 96, generator=g, device="cuda").mul_(0.1).requires_grad_() for _ in range(2))
    w3 = torch.randn(96, 160, generator=g, device="cuda").mul_(0.1).requires_grad_()
    y = L.linear(L.swiglu(L.linear(x, w1), L.linear(x, w2)), w3)
    y.backward(torch.ones_like(y))
    grads = [p.grad.double() for p in (x, w1, w2, w3)]
    xs, ws = x.detach().double().requires_grad_(), [w.detach().double().requires_grad_() for w in (w1, w2, w3)]
    a, b = xs @ ws[0].T, xs @ ws[1].T
    z = (a * torch.sigmoid(a) * b) @ ws[2].T
    z.backward(torch.ones_like(z))
    # bf16 activations and weights (2^-8 each, four in a chain) and 8-bit
    # checkpoints (a step of max / 64 at most over a uniform error: 1% rms)
    for got, p in zip(grads, (xs, *ws)):
        assert rel(got, p.grad) <= 3e-2
    assert w1.grad.dtype == torch.float32 and x.grad.dtype == torch.bfloat16


def test_other_streams():
    import torch
    from paper_2609_36692_gb300 import layers as L
    x, dy = sample(7, 500, 256, "bf16"), sample(8, 500, 128, "bf16")
    want = L.ckpt_wgrad(dy, L.ckpt_pack(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = L.ckpt_wgrad(dy, L.ckpt_pack(x))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals():
    import torch
    from paper_2609_36692_gb300 import layers as L
    from paper_2609_36692_gb300 import normpre as C
    x = sample(1, 8, 64, "f32")
    with pytest.raises(ValueError, match="CUDA"):
        L.ckpt_pack(x.cpu())
    with pytest.raises(TypeError, match="dtype"):
        L.ckpt_pack(x.half())
    with pytest.raises(ValueError, match="matrix"):
        L.ckpt_pack(x[0])
    with pytest.raises(ValueError, match="contiguous"):
        L.ckpt_pack(x.T)
    with pytest.raises(ValueError, match="overlap"):
        L.ckpt_pack(x[:1].expand(8, 64))
    ck = L.ckpt_pack(x)
    with pytest.raises(ValueError, match="dy must be"):
        L.ckpt_wgrad(x[:7], ck)
    with pytest.raises(ValueError, match="accumulate"):
        L.ckpt_wgrad(x, ck, accumulate=True)
    with pytest.raises(ValueError, match="out must be"):
        L.ckpt_wgrad(x, ck, out=torch.empty(3, 3, device="cuda"))
    with pytest.raises(TypeError, match="one dtype"):
        L.ckpt_swiglu(x, x.bfloat16())
    with pytest.raises(C.NormPreError) as e:
        L.ckpt_pack(torch.empty(100, device="cuda")[1:65].view(1, 64))
    assert e.value.status == C.NORMPRE_ERR_ALIGN
