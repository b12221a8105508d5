"""Packed causal attention on the GPU against the definition in 64 bits.

Tolerances (relative Frobenius error).  fp32: products and sums of a few
hundred fp32 terms, 2^-24 each with random signs, through an exponential whose
argument stays below 64: 64 * 2^-24 = 4e-6, doubled for the backward's second
product, 1e-5.  bf16: one rounding (8 significant bits) costs at most 2^-8 and
in the root mean square less than 2^-9; the forward pass
rounds the probabilities and the output (2 * 2^-9 = 3.9e-3), the backward pass
the probabilities, ds, the forward's output inside delta, and its own output,
with ds carrying two of them (5 * 2^-9 = 9.8e-3).
"""
import math

import pytest

pytestmark = pytest.mark.gpu

TOL = {("f32", "fwd"): 1e-5, ("f32", "bwd"): 1e-5, ("bf16", "fwd"): 3.95e-3, ("bf16", "bwd"): 9.8e-3}
LAYOUTS = [(2, 2, 64), (4, 2, 128), (6, 2, 96), (3, 1, 64), (5, 5, 80), (1, 1, 8), (4, 1, 128)]
LENGTHS = [[1], [2, 0, 1], [127, 128, 129, 1], [64, 0, 65, 63], [300, 513], [1000], [0, 0], [256, 384]]


def dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def make(seed, tokens, h, hk, d, dtype, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(tokens, h + 2 * hk, d, generator=g, device="cuda")
    x[:, :h] *= scale
    x = x.to(dt(dtype))
    do = torch.randn(tokens, h, d, generator=g, device="cuda").to(dt(dtype))
    return x[:, :h], x[:, h:h + hk], x[:, h + hk:], do


def reference(q, k, v, do, lengths, scale=None):
    """Out, log-sum and gradients in 64 bits; rows outside the sequences zero;
    and for each of them the root sum square of its terms, None for the first
    two.  A row that sees one key has ds = 0 by cancellation, so that dq's and
    dk's errors are measured against their terms where those are larger."""
    import torch
    t, h, d = q.shape
    hk = k.shape[1]
    g = h // hk
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    z = lambda n: torch.zeros(t, n, d, dtype=torch.float64, device=q.device)  # noqa: E731
    out, dq, dk, dv = z(h), z(h), z(hk), z(hk)
    lse = torch.full((h, t), -math.inf, dtype=torch.float64, device=q.device)
    terms = [0.0, 0.0, 0.0]
    at = 0
    for n in lengths:
        r = slice(at, at + n)
        at += n
        if n == 0:
            continue
        mask = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
        for i in range(h):
            qq, kk, vv, dd = (x[r, j].double() for x, j in ((q, i), (k, i // g), (v, i // g), (do, i)))
            s = (scale * qq @ kk.T).masked_fill(mask, -math.inf)
            lse[i, r] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[i, r, None])
            o = p @ vv
            dp, delta = dd @ vv.T, (dd * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            size = (p * (dp.abs() + delta.abs())) ** 2
            terms[0] += float((scale ** 2 * size @ (kk ** 2)).sum())
            terms[1] += float((scale ** 2 * size.T @ (qq ** 2)).sum())
            out[r, i], dq[r, i] = o, scale * ds @ kk
            dk[r, i // g] += scale * ds.T @ qq
            dv[r, i // g] += p.T @ dd
    return out, lse, dq, dk, dv, [x ** 0.5 for x in terms]


def err(x, ref, terms=0.0):
    import torch
    n = max(float(torch.linalg.norm(ref)), terms)
    e = float(torch.linalg.norm(x.double() - ref))
    return e / n if n > 0 else e


def plan_for(h, hk, d, tokens, lengths, dtype, **kw):
    from paper_2609_36692_gb300.layers import PackedAttention
    p = PackedAttention(h, hk, d, max_tokens=max(1, tokens), max_seqs=max(1, len(lengths)), dtype=dt(dtype), **kw)
    p.set_lengths(lengths)
    return p


def check_forward(plan, q, k, v, do, lengths, dtype, scale=None):
    import torch
    ref = reference(q, k, v, do, lengths, scale)
    out, lse = plan.forward(q, k, v)
    assert plan.status() == 0
    n = sum(lengths)
    assert err(out, ref[0]) <= TOL[dtype, "fwd"]
    assert torch.equal(lse[:, n:], torch.full_like(lse[:, n:], -math.inf))
    if n:
        # absolute: the argument of the exponential carries the error
        assert float((lse[:, :n].double() - ref[1][:, :n]).abs().max()) <= 2e-5 * max(1.0, float(ref[1][:, :n].abs().max()))
    assert not bool(out[n:].any())
    return out, lse, ref


def check_backward(plan, q, k, v, do, out, lse, ref, lengths, dtype):
    grads = plan.backward(q, k, v, out, lse, do)
    assert plan.status() == 0
    n = sum(lengths)
    for name, x, r, m in zip(("dq", "dk", "dv"), grads, ref[2:5], ref[5]):
        assert err(x, r, m) <= TOL[dtype, "bwd"], name
        assert not bool(x[n:].any()), name
    return grads


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_forward_and_backward(layout, lengths, dtype):
    h, hk, d = layout
    tokens = sum(lengths) + 3
    q, k, v, do = make(len(lengths) + d, tokens, h, hk, d, dtype)
    plan = plan_for(h, hk, d, tokens, lengths, dtype)
    out, lse, ref = check_forward(plan, q, k, v, do, lengths, dtype)
    check_backward(plan, q, k, v, do, out, lse, ref, lengths, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences_and_no_tail(dtype):
    lengths = [1 + (37 * i) % 200 for i in range(70)]
    h, hk, d = 2, 1, 64
    q, k, v, do = make(5, sum(lengths), h, hk, d, dtype)
    plan = plan_for(h, hk, d, sum(lengths), lengths, dtype)
    out, lse, ref = check_forward(plan, q, k, v, do, lengths, dtype)
    check_backward(plan, q, k, v, do, out, lse, ref, lengths, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sharp_scores(dtype):
    """Scores of up to a hundred, and maxima that grow along the keys, so that
    the running maximum moves at every block."""
    import torch
    h, hk, d, lengths = 2, 2, 64, [700]
    q, k, v, do = (x.contiguous() for x in make(6, 700, h, hk, d, dtype, scale=3.0))
    # later keys are larger; the first coordinate orders the scores both ways
    k *= torch.linspace(0.2, 2.0, 700, device="cuda").to(k.dtype)[:, None, None]
    q[:, 0, 0], k[:, :, 0] = 4.0, torch.linspace(0, 60, 700, device="cuda").to(k.dtype)[:, None]
    q[:, 1, 0] = -4.0
    plan = plan_for(h, hk, d, 700, lengths, dtype)
    out, lse, ref = check_forward(plan, q, k, v, do, lengths, dtype)
    # errors of the log-sum grow with the scores: 2^-24 * 100 in the exponent
    grads = plan.backward(q, k, v, out, lse, do)
    for x, r in zip(grads, ref[2:5]):
        assert err(x, r) <= (4e-5 if dtype == "f32" else 2e-2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scale_argument(dtype):
    h, hk, d, lengths = 2, 1, 128, [200]
    q, k, v, do = make(7, 200, h, hk, d, dtype)
    plan = plan_for(h, hk, d, 200, lengths, dtype, scale=0.25)
    out, lse, ref = check_forward(plan, q, k, v, do, lengths, dtype, scale=0.25)
    check_backward(plan, q, k, v, do, out, lse, ref, lengths, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.3e38])
def test_other_rows_do_not_reach_a_sequence(dtype, bad):
    """What rows past the sequences and rows of other sequences hold stays
    there: the same bits as with ordinary values."""
    import torch
    h, hk, d, lengths = 4, 2, 128, [130, 77, 200]
    tokens = sum(lengths) + 140
    q, k, v, do = (x.contiguous() for x in make(8, tokens, h, hk, d, dtype))
    plan = plan_for(h, hk, d, tokens, lengths, dtype)
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    q2, k2, v2, do2 = (x.clone() for x in (q, k, v, do))
    for x in (q2, k2, v2, do2):
        x[130:207] = bad          # the middle sequence
        x[sum(lengths):] = bad    # the tail
    out2, lse2 = plan.forward(q2, k2, v2)
    out2[sum(lengths):] = bad     # nothing reads what the tail holds
    lse2[:, sum(lengths):] = bad
    grads2 = plan.backward(q2, k2, v2, out2, lse2, do2)
    assert plan.status() == 0
    keep = torch.cat([torch.arange(0, 130), torch.arange(207, 407)]).cuda()
    assert torch.equal(out2[keep], out[keep]) and torch.equal(lse2[:, keep], lse[:, keep])
    for a, b in zip(grads2, grads):
        assert torch.equal(a[keep], b[keep])
        assert not bool(a[407:].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_reaches_the_rows_that_see_it(dtype):
    import torch
    h, hk, d = 1, 1, 64
    q, k, v, _ = (x.contiguous() for x in make(9, 300, h, hk, d, dtype))
    k[260, 0, 3] = float("nan")
    out, lse = plan_for(h, hk, d, 300, [300], dtype).forward(q, k, v)
    assert bool(torch.isnan(out[260:]).all()) and bool(torch.isnan(lse[:, 260:]).all())
    assert bool(torch.isfinite(out[:256]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts_of_memory(dtype):
    """Slices of a fused projection, head-major tensors and given outputs with
    strides of their own give the bits of contiguous ones."""
    import torch
    h, hk, d, lengths = 4, 2, 64, [150, 33]
    q, k, v, do = make(10, 183, h, hk, d, dtype)
    plan = plan_for(h, hk, d, 183, lengths, dtype)
    c = [x.contiguous() for x in (q, k, v, do)]
    out, lse = plan.forward(*c[:3])
    grads = plan.backward(*c[:3], out, lse, c[3])
    hm = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, do)]
    fused = torch.full((183, h + 2 * hk, d), 7.0, dtype=dt(dtype), device="cuda")
    views = (fused[:, :h], fused[:, h:h + hk], fused[:, h + hk:])
    wide = torch.full((183, h, 2 * d), 7.0, dtype=dt(dtype), device="cuda")
    for ins in ([q, k, v, do], hm):
        o2, l2 = plan.forward(*ins[:3], out=wide[:, :, :d])
        assert torch.equal(o2, out) and torch.equal(l2, lse)
        assert bool((wide[:, :, d:] == 7.0).all())
        g2 = plan.backward(*ins[:3], o2, l2, ins[3], *views)
        for a, b in zip(g2, grads):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(dtype):
    import torch
    h, hk, d, n = 1, 1, 64, 1200
    stride = 1 << 21                       # 1200 rows span 2.5e9 elements
    q, k, v, do = (x.contiguous() for x in make(11, n, h, hk, d, dtype))
    plan = plan_for(h, hk, d, n, [n], dtype)
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    big = torch.empty(n * stride, dtype=dt(dtype), device="cuda").view(n, stride)

    def far(x, at):
        y = big[:, at:at + d].unsqueeze(1)
        y.copy_(x)
        return y
    ins = [far(x, 64 * i) for i, x in enumerate((q, k, v, do))]
    o2, l2 = plan.forward(*ins[:3], out=big[:, 512:512 + d].unsqueeze(1))
    g2 = plan.backward(*ins[:3], o2, l2, ins[3], *(big[:, a:a + d].unsqueeze(1) for a in (1024, 2048, 4096)))
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    for a, b in zip(g2, grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_again_new_lengths_and_other_streams(dtype):
    import torch
    h, hk, d = 4, 2, 128
    q, k, v, do = make(12, 512, h, hk, d, dtype)
    plan = plan_for(h, hk, d, 512, [300, 212], dtype)
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    plan.set_lengths([512])
    plan.forward(q, k, v)
    plan.set_lengths([])
    z, zl = plan.forward(q, k, v)
    assert not bool(z.any()) and bool((zl == -math.inf).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.set_lengths([300, 212])
        o2, l2 = plan.forward(q, k, v)
        g2 = plan.backward(q, k, v, o2, l2, do)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    for a, b in zip(grads, g2):
        assert torch.equal(a, b)


def test_capture_in_a_graph():
    import torch
    h, hk, d = 4, 2, 128
    q, k, v, do = make(13, 400, h, hk, d, "bf16")
    plan = plan_for(h, hk, d, 400, [123, 277], "bf16")
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o2, l2 = plan.forward(q, k, v)
        g2 = plan.backward(q, k, v, o2, l2, do)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    for a, b in zip(g2, grads):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    """Central differences of sum(out * w) along random directions.  fp32
    forward, step 2^-6: the difference carries 2^-24 * |loss terms| / step and a
    third-order term of step^2; both are below 2e-3 of the slope here."""
    import torch
    h, hk, d, lengths = 2, 1, 64, [40, 23]
    q, k, v, w = (x.contiguous() for x in make(14, 63, h, hk, d, "f32"))
    plan = plan_for(h, hk, d, 63, lengths, "f32")
    loss = lambda *x: float((plan.forward(*x)[0].double() * w.double()).sum())  # noqa: E731
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, w)
    g = torch.Generator(device="cuda").manual_seed(3)
    for i, grad in enumerate(grads):
        # along the gradient plus noise, so that the slope is not small
        u = grad / grad.norm() + 0.02 * torch.randn(grad.shape, generator=g, device="cuda")
        step = 2.0 ** -6
        x = [q, k, v]
        hi = [y + step * u if j == i else y for j, y in enumerate(x)]
        lo = [y - step * u if j == i else y for j, y in enumerate(x)]
        slope = (loss(*hi) - loss(*lo)) / (2 * step)
        assert abs(slope - float((grad.double() * u.double()).sum())) <= 2e-3 * abs(slope)


def test_autograd():
    import torch
    h, hk, d, lengths = 4, 2, 64, [100, 28]
    q, k, v, do = (x.contiguous() for x in make(15, 128, h, hk, d, "bf16"))
    plan = plan_for(h, hk, d, 128, lengths, "bf16")
    ref = reference(q, k, v, do, lengths)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    (plan(*leaves) * do).sum().backward()
    for x, r in zip(leaves, ref[2:5]):
        assert err(x.grad, r) <= TOL["bf16", "bwd"]
    # an expanded gradient (the sum's) is laid out before the kernels read it
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    plan(*leaves).sum().backward()
    ref = reference(q, k, v, torch.ones_like(do), lengths)
    assert err(leaves[2].grad, ref[4]) <= TOL["bf16", "bwd"]


def test_refusals():
    import torch
    from paper_2609_36692_gb300 import normpre as C
    q, k, v, do = make(16, 64, 4, 2, 64, "bf16")
    plan = plan_for(4, 2, 64, 64, [64], "bf16")
    with pytest.raises(TypeError, match="bfloat16"):
        plan.forward(q.float(), k, v)
    with pytest.raises(ValueError, match="k must be"):
        plan.forward(q, q, v)
    with pytest.raises(ValueError, match="cuda"):
        plan.forward(q.cpu(), k, v)
    with pytest.raises(ValueError, match="lse"):
        plan.forward(q, k, v, lse=torch.empty(64, 4, device="cuda"))
    with pytest.raises(C.NormPreError) as e:      # rows off 16-byte boundaries
        plan.forward(torch.empty(64, 4, 65, dtype=torch.bfloat16, device="cuda")[:, :, 1:], k, v)
    assert e.value.status == C.NORMPRE_ERR_ALIGN
    with pytest.raises(C.NormPreError) as e:      # broadcast rows
        plan.forward(q, k[:1].expand(64, 2, 64), v)
    assert e.value.status == C.NORMPRE_ERR_SHAPE
    with pytest.raises(C.NormPreError) as e:      # an output that overlaps itself
        plan.forward(q, k, v, out=torch.empty(64 * 64 + 4 * 64, dtype=torch.bfloat16, device="cuda").as_strided(
            (64, 4, 64), (64, 64, 1)))
    assert e.value.status == C.NORMPRE_ERR_SHAPE
    with pytest.raises(C.NormPreError) as e:      # fewer rows than the lengths
        plan.forward(q[:60], k[:60], v[:60])
    assert e.value.status == C.NORMPRE_ERR_SHAPE
    for lengths, status in (([65], C.NORMPRE_ERR_SHAPE), ([1, 1], C.NORMPRE_ERR_SHAPE), ([-1], C.NORMPRE_ERR_ARG)):
        with pytest.raises(C.NormPreError) as e:
            plan.set_lengths(lengths)
        assert e.value.status == status
    out, _ = plan.forward(q, k, v)                # a refused call leaves the plan as it was
    assert bool(torch.isfinite(out.float()).all()) and bool(out.any())
