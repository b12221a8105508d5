"""Norms of queries and keys with the rotation of their positions, against the
definition in 64 bits.

Tolerances, in units u = 2^-24 of what a value is summed from.  A mean of up to
128 squares: a lane's 16 products one after the other, up to 4 sums of lanes, the
division: at most 21 u, so that r is off by 11 u, with the inverse root's own 2,
13.  xh: 14, y: 15; cos and sin: their function's 2, its argument's 1 and the
argument cut off at 2^-34 of a turn, together 4; the two products and their sum,
2: a result is within 21 u of |y_a| + |y_b|.  Backward: g within 6 u of its two
terms, u = g w 7, their product with xh 21, its mean 21 more, times xh 15: the
result, with r's 13, within 75 u of r (|u| + |xh| mean|u xh|).  A weight's
gradient: terms of 20 u, and a sum over rows of at most as many additions one
after the other as a warp has rows, plus 40 for what follows.  bf16 results have
one rounding more, 2^-8.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-6


def dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def half_step(t):
    import torch
    return 2.0 ** -8 if t == torch.bfloat16 else 0.0


def make(seed, tokens, h, hk, d, dtype, wdtype="f32", first=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = randn(tokens, h + 2 * hk, d)
    x *= torch.exp(2 * randn(tokens, h + 2 * hk, 1))           # rows of very different sizes
    x = x.to(dt(dtype))
    w = [(1 + 0.5 * randn(d)).to(dt(wdtype)) for _ in range(2)]
    dz = randn(tokens, h + hk, d).to(dt(dtype))
    pos = first + torch.arange(tokens, device="cuda") % 1000
    return dict(q=x[:, :h], k=x[:, h:h + hk], positions=pos, qw=w[0], kw=w[1], dq=dz[:, :h], dk=dz[:, h:])


def pairs(d, r, inter):
    """The pairs' dimensions, and those that pass."""
    a = [2 * i if inter else i for i in range(r // 2)]
    b = [2 * i + 1 if inter else i + r // 2 for i in range(r // 2)]
    return a, b


def reference(x, w, positions, dz, r, inter, base=10000.0, eps=EPS, norm=True, frequencies=None):
    """(z, |terms|, dx, |terms|, dw, |terms|) in 64 bits.  Angles by exact whole
    numbers of 2^-200 turns, so that far positions lose nothing."""
    import torch
    t, n, d = x.shape
    f64 = torch.float64
    x, dz = x.double(), dz.double()
    w = torch.ones(d, dtype=f64, device=x.device) if w is None else w.double()
    f = frequencies if frequencies is not None else [base ** (-2.0 * i / r) for i in range(r // 2)]
    # p f / 2 pi: a product of the position with a whole number of 2^-200 turns
    two_pi = 31415926535897932384626433832795028841971693993751058209749445923 * 2
    turn = [int(math.ldexp(y, 300)) * 10 ** 64 * (1 << 100) // (two_pi << 200) if y else 0 for y in f]   # 2^-200 turns
    places = [int(p) for p in positions.tolist()] if r else [0] * t
    known = {}
    for p in set(places):
        known[p] = [2 * math.pi * ((p * u) % (1 << 200)) / (1 << 200) for u in turn]
    angle = torch.tensor([known[p] for p in places], dtype=f64, device=x.device).view(t, 1, r // 2)
    c, s = torch.cos(angle), torch.sin(angle)
    a, b = pairs(d, r, inter)
    inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) if norm else torch.ones(t, n, 1, dtype=f64, device=x.device)
    xh = x * inv

    def turned(y, c, s):
        z, m = y.clone(), y.abs()
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
        both = m[..., a] + m[..., b]
        m[..., a], m[..., b] = both, both
        return z, m
    z, zm = turned(xh * w, c, s)
    g, gm = turned(dz, c, -s)
    u, um = g * w, gm * w.abs()
    if not norm:
        return z, zm, g, gm, None, None
    mean, mm = (u * xh).mean(-1, keepdim=True), (um * xh.abs()).mean(-1, keepdim=True)
    dx, dxm = inv * (u - xh * mean), inv * (um + xh.abs() * mm)
    return z, zm, dx, dxm, (g * xh).sum((0, 1)), (gm * xh.abs()).sum((0, 1))


def within(x, ref, terms, units):
    """Each value to `units` of 2^-24 of its terms, and its own rounding."""
    bound = units * U * terms + half_step(x.dtype) * (ref.abs() + units * U * terms) + 2.0 ** -133
    worst = float(((x.double() - ref).abs() / bound).max()) if x.numel() else 0.0
    assert worst <= 1.0, worst


def check(plan, s, r, inter, used=None, weights=True, **kw):
    import torch
    t = s["q"].shape[0]
    n = t if used is None else used
    qw, kw_ = (s["qw"], s["kw"]) if weights else (None, None)
    q, k = plan.forward(s["q"], s["k"], s["positions"], qw, kw_, used=used)
    dq, dk, dqw, dkw = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], qw, kw_, used=used)
    for x, w, dz, z, dx, dw in ((s["q"], qw, s["dq"], q, dq, dqw), (s["k"], kw_, s["dk"], k, dk, dkw)):
        ref = reference(x[:n], w, s["positions"][:n], dz[:n], r, inter, **kw)
        within(z[:n], ref[0], ref[1], 21)
        within(dx[:n], ref[2], ref[3], 75)
        assert not bool(z[n:].any()) and not bool(dx[n:].any())
        assert z.dtype == dx.dtype == x.dtype
        if w is None:
            assert dw is None
        else:
            # rows of a warp: at most one in 8 * 2 of an SM's eight warps' share, and no fewer than one
            within(dw, ref[4], ref[5], 60 + n * x.shape[1] // 256)
            assert dw.dtype == w.dtype
    return q, k, dq, dk, dqw, dkw


LAYOUTS = [(12, 12, 64), (16, 8, 128), (8, 1, 128), (6, 2, 96), (5, 5, 80), (1, 1, 8), (3, 1, 24)]


def plan_for(h, hk, d, dtype, r, inter, **kw):
    from paper_2609_36692_gb300.layers import QKNormRotary
    return QKNormRotary(h, hk, d, rotary_dim=r, interleaved=inter, eps=EPS, dtype=dt(dtype), **kw)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype, wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_forward_and_backward(layout, dtype, wdtype, inter):
    h, hk, d = layout
    for tokens, r in ((1, d), (3, d // 2), (37, 2 * (d // 8)), (130, 2), (300, d), (41, 0), (65, d - 2)):
        s = make(tokens + d, tokens, h, hk, d, dtype, wdtype, first=11)
        check(plan_for(h, hk, d, dtype, r, inter), s, r, inter)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [2500, 20000])
def test_many_tokens(tokens, dtype):
    s = make(tokens, tokens, 16, 8, 128, dtype, "f32")
    check(plan_for(16, 8, 128, dtype, 128, False, base=1e6), s, 128, False, base=1e6)


@pytest.mark.parametrize("inter", [False, True])
def test_options(inter):
    """No weights, one weight, no norm, given frequencies, 4-byte positions."""
    import torch
    s = make(1, 50, 4, 2, 64, "f32")
    plan = plan_for(4, 2, 64, "f32", 64, inter)
    check(plan, s, 64, inter, weights=False)
    q, k = plan.forward(s["q"], s["k"], s["positions"], s["qw"])
    assert torch.equal(q, plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])[0])
    assert torch.equal(k, plan.forward(s["q"], s["k"], s["positions"], None, None)[1])
    got = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], None, s["kw"])
    assert got[2] is None
    assert torch.equal(got[3], plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])[3])
    assert plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"], weights=False)[2:] == (None, None)
    assert torch.equal(q, plan.forward(s["q"], s["k"], s["positions"].int(), s["qw"])[0])
    check(plan_for(4, 2, 64, "f32", 64, inter, norm=False), s, 64, inter, weights=False, norm=False)
    f = [0.0, 1.0, -0.25, 3.0, 1e-9] + [0.1] * 11
    check(plan_for(4, 2, 64, "f32", 32, inter, frequencies=f), s, 32, inter, frequencies=f)


@pytest.mark.parametrize("first", [1000003, (1 << 31) - 7, (1 << 40) + 12345, -9, -(1 << 33)])
def test_far_positions(first):
    """A frequency is a whole number of 2^-64 turns: off by 2^-64 of a turn, and by
    the 2^-53 of its own 64-bit value.  At position p the angle is off by up to
    p f 2^-53 radians, which joins the bound where it counts."""
    import torch
    s = make(2, 20, 2, 1, 64, "f32", first=first)
    plan = plan_for(2, 1, 64, "f32", 64, False)
    q, k = plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
    for x, w, z in ((s["q"], s["qw"], q), (s["k"], s["kw"], k)):
        ref = reference(x, w, s["positions"], torch.zeros_like(x), 64, False)
        within(z, ref[0], ref[1], 21 + (abs(first) + 1000) * 2.0 ** -53 / U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [0.0, 1e-38, 1e-25, 1e-12, 1e15, 1e19, 1e30, 2e38])
def test_rows_of_any_size(size, dtype):
    """Rows whose squares leave fp32's range, beside ordinary ones in the warp."""
    import torch
    s = make(3, 64, 4, 2, 64, dtype)
    # one row in three, at most `size` large
    x = s["q"]
    y = x[1::3].double()
    x[1::3] = (y / y.abs().amax(-1, keepdim=True) * size).to(x.dtype)
    plan = plan_for(4, 2, 64, dtype, 64, False)
    q, _ = plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
    dq, _, dqw, _ = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
    ref = reference(s["q"], s["qw"], s["positions"], s["dq"], 64, False)
    within(q, ref[0], ref[1], 21)
    within(dq, ref[2], ref[3], 75)
    within(dqw, ref[4], ref[5], 60)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_values_beside_large_ones(dtype):
    """A row of values from 1e-20 to 1e25: each to its own size."""
    import torch
    s = make(13, 33, 4, 2, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    size = 10.0 ** (-20 + 45 * torch.rand(33, 4, 1, 128, generator=g, device="cuda"))
    size = torch.cat([size, size], 2).reshape(33, 4, 256)[..., ::2]
    s["q"].copy_((s["q"].float() * size).to(s["q"].dtype))
    plan = plan_for(4, 2, 128, dtype, 64, True)
    q, _ = plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
    dq, _, dqw, _ = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
    ref = reference(s["q"], s["qw"], s["positions"], s["dq"], 64, True)
    within(q, ref[0], ref[1], 21)
    within(dq, ref[2], ref[3], 75)
    within(dqw, ref[4], ref[5], 60)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, 1e30])
def test_what_is_not_finite_stays_in_its_row(bad, dtype):
    """Nothing of a row, large ones included, changes a bit of the others."""
    import torch
    s = make(4, 40, 4, 2, 64, dtype)
    plan = plan_for(4, 2, 64, dtype, 32, False)
    args = s["positions"], s["qw"], s["kw"]
    q, k = plan.forward(s["q"], s["k"], *args)
    dq, dk = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])[:2]
    q2 = s["q"].clone()
    q2[17, 2, 5] = bad
    rest = torch.ones(40, 4, dtype=torch.bool, device="cuda")
    rest[17, 2] = False
    got = plan.forward(q2, s["k"], *args)
    assert torch.equal(got[0][rest], q[rest]) and torch.equal(got[1], k)
    assert bool(torch.isnan(got[0][17, 2, 5])) or bad == 1e30
    got = plan.backward(q2, s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
    assert torch.equal(got[0][rest], dq[rest]) and torch.equal(got[1], dk)
    assert bool(torch.isnan(got[2][5])) or bad == 1e30


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding(dtype):
    import torch
    s = make(5, 70, 6, 2, 96, dtype)
    for x in (s["q"], s["k"], s["dq"], s["dk"]):
        x[50:] = math.nan
    s["positions"][50:] = -(1 << 60)
    plan = plan_for(6, 2, 96, dtype, 96, True)
    check(plan, s, 96, True, used=50)
    got = plan.forward(s["q"], s["k"], s["positions"], used=0)
    assert not bool(got[0].any()) and not bool(got[1].any())
    got = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"], used=0)
    assert not any(bool(x.any()) for x in got)


def test_no_tokens():
    import torch
    s = make(6, 5, 4, 2, 64, "bf16")
    z = {n: s[n][:0] for n in ("q", "k", "positions", "dq", "dk")}
    plan = plan_for(4, 2, 64, "bf16", 64, False)
    q, k = plan.forward(z["q"], z["k"], z["positions"], s["qw"], s["kw"])
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    got = plan.backward(z["q"], z["k"], z["positions"], z["dq"], z["dk"], s["qw"], s["kw"])
    assert got[0].shape == (0, 4, 64) and not bool(got[2].any()) and not bool(got[3].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("r, inter", [(64, False), (64, True), (16, False), (6, False), (2, False)])
def test_layouts_of_memory(r, inter, dtype):
    """Slices of a fused projection, head-major tensors, outputs with strides of
    their own, and outputs over their inputs give the bits of contiguous ones."""
    import torch
    h, hk, d = 4, 2, 64
    s = make(7, 150, h, hk, d, dtype)
    plan = plan_for(h, hk, d, dtype, r, inter)
    w = s["qw"], s["kw"]
    c = {n: s[n].contiguous() for n in ("q", "k", "dq", "dk")}
    want = plan.forward(c["q"], c["k"], s["positions"], *w)
    want += plan.backward(c["q"], c["k"], s["positions"], c["dq"], c["dk"], *w)
    wide = [torch.full((150, x, 2 * d), 7.0, dtype=dt(dtype), device="cuda") for x in (h, hk)]
    for f in (lambda x: x, lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)):
        i = {n: f(s[n]) for n in c}
        got = plan.forward(i["q"], i["k"], s["positions"], *w, q_out=wide[0][:, :, :d], k_out=wide[1][:, :, :d])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        got = plan.backward(i["q"], i["k"], s["positions"], i["dq"], i["dk"], *w, dq=wide[0][:, :, :d], dk=wide[1][:, :, :d])
        assert all(torch.equal(a, b) for a, b in zip(got, want[2:]))
        assert all(bool((x[:, :, d:] == 7.0).all()) for x in wide)
    # in place
    i = {n: x.clone() for n, x in c.items()}
    plan.backward(i["q"], i["k"], s["positions"], i["dq"], i["dk"], *w, dq=i["dq"], dk=i["dk"])
    assert torch.equal(i["dq"], want[2]) and torch.equal(i["dk"], want[3])
    plan.forward(i["q"], i["k"], s["positions"], *w, q_out=i["q"], k_out=i["k"])
    assert torch.equal(i["q"], want[0]) and torch.equal(i["k"], want[1])


def test_offsets_beyond_32_bits():
    import torch
    h, hk, d, n, stride = 1, 1, 64, 1200, 1 << 21
    s = make(8, n, h, hk, d, "bf16")
    plan = plan_for(h, hk, d, "bf16", d, False)
    want = plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
    want += plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
    big = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda").view(n, stride)
    at = lambda i: big[:, 64 * i:64 * i + d].unsqueeze(1)  # noqa: E731
    for i, name in enumerate(("q", "k", "dq", "dk")):
        at(i).copy_(s[name])
    got = plan.forward(at(0), at(1), s["positions"], s["qw"], s["kw"], q_out=at(4), k_out=at(5))
    got += plan.backward(at(0), at(1), s["positions"], at(2), at(3), s["qw"], s["kw"], dq=at(6), dk=at(7))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_streams_and_capture():
    import torch
    s = make(9, 3000, 16, 8, 128, "bf16", "bf16")
    plan = plan_for(16, 8, 128, "bf16", 128, False)
    w = s["qw"], s["kw"]

    def calls(stream=None):
        q, k = plan.forward(s["q"], s["k"], s["positions"], *w, stream=stream)
        return (q, k, *plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], *w, stream=stream))
    want = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [calls(), calls(side)]                  # two calls at once
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(calls())
    for g, st in zip(graphs, (side, torch.cuda.Stream())):
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    for outs in got:
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_gradient_against_differences():
    """Central differences of sum(z * v), fp32.  With a step of 2^-6 along a
    direction of length one the quotient carries 2^-24 of the loss's terms / step
    and a third-order term of step^2, both below 2e-3 of the slope here."""
    import torch
    s = make(10, 20, 2, 1, 64, "f32")
    s["q"], s["k"] = (torch.randn(20, n, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)) for n in (2, 1))
    plan = plan_for(2, 1, 64, "f32", 48, True)
    x = [s["q"], s["k"], s["qw"], s["kw"]]

    def loss(q, k, qw, kw):
        a, b = plan.forward(q, k, s["positions"], qw, kw)
        return float((a.double() * s["dq"].double()).sum() + (b.double() * s["dk"].double()).sum())
    for i, grad in enumerate(plan.backward(x[0], x[1], s["positions"], s["dq"], s["dk"], x[2], x[3])):
        u = grad / grad.norm()
        step = 2.0 ** -6
        hi, lo = ([y + sign * step * u if j == i else y for j, y in enumerate(x)] for sign in (1, -1))
        slope = (loss(*hi) - loss(*lo)) / (2 * step)
        assert abs(slope - float((grad.double() * u.double()).sum())) <= 2e-3 * abs(slope)


def test_autograd():
    """Queries and keys are slices of one projection, which gets both gradients;
    expanded gradients of the results are laid out first."""
    import torch
    s = make(11, 60, 4, 2, 64, "bf16")
    plan = plan_for(4, 2, 64, "bf16", 64, False)
    x = torch.cat([s["q"], s["k"]], 1).requires_grad_()
    w = [s[n].clone().requires_grad_() for n in ("qw", "kw")]
    q, k = plan(x[:, :4], x[:, 4:], s["positions"], *w, used=55)
    ((q * s["dq"]).sum() + (k * s["dk"]).sum()).backward()
    want = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"], used=55)
    assert torch.equal(x.grad, torch.cat(want[:2], 1))
    assert torch.equal(w[0].grad, want[2]) and torch.equal(w[1].grad, want[3])
    # only one result is used, one input wants a gradient
    x2 = s["q"].clone().requires_grad_()
    q, k = plan(x2, s["k"], s["positions"], s["qw"], s["kw"])
    q.sum().backward()
    ones = torch.ones_like(s["dq"])
    assert torch.equal(x2.grad, plan.backward(s["q"], s["k"], s["positions"], ones, torch.zeros_like(s["dk"]), s["qw"], s["kw"])[0])
    with pytest.raises(RuntimeError, match="once_differentiable|twice|differentiable"):
        x3 = s["q"].clone().requires_grad_()
        g, = torch.autograd.grad(plan(x3, s["k"], s["positions"], s["qw"], s["kw"])[0].float().square().sum(), x3, create_graph=True)
        g.sum().backward()


def test_refusals():
    import torch
    from paper_2609_36692_gb300 import normpre as C
    s = make(12, 20, 4, 2, 64, "bf16")
    plan = plan_for(4, 2, 64, "bf16", 64, False)
    q, k, p, qw, kw = (s[n] for n in ("q", "k", "positions", "qw", "kw"))
    for exc, args in ((TypeError, (q.float(), k, p, qw, kw)), (ValueError, (q, q, p, qw, kw)),
                      (ValueError, (q.cpu(), k, p, qw, kw)), (ValueError, (q, k.cpu(), p, qw, kw)),
                      (ValueError, (q, k, None, qw, kw)), (ValueError, (q, k, p.float(), qw, kw)),
                      (ValueError, (q, k, p[:19], qw, kw)), (ValueError, (q, k, p.cpu(), qw, kw)),
                      (ValueError, (q, k, p.repeat_interleave(2)[::2], qw, kw)), (ValueError, (q, k, p, qw[:32], kw)),
                      (TypeError, (q, k, p, qw, kw.bfloat16())), (TypeError, (q, k, p, qw.half(), kw.half())),
                      (ValueError, (q, k, p, qw.cpu(), kw))):
        with pytest.raises(exc):
            plan.forward(*args)
    for used, status in ((21, C.NORMPRE_ERR_SHAPE), (-1, C.NORMPRE_ERR_SHAPE)):
        with pytest.raises(C.NormPreError) as e:
            plan.forward(q, k, p, qw, kw, used=used)
        assert e.value.status == status
    with pytest.raises(C.NormPreError) as e:      # rows off 16-byte boundaries
        plan.forward(torch.empty(20, 4, 65, dtype=torch.bfloat16, device="cuda")[:, :, 1:], k, p, qw, kw)
    assert e.value.status == C.NORMPRE_ERR_ALIGN
    with pytest.raises(C.NormPreError) as e:      # an output that overlaps itself
        plan.forward(q, k, p, qw, kw, q_out=torch.empty(6000, dtype=torch.bfloat16, device="cuda").as_strided((20, 4, 64), (64, 64, 1)))
    assert e.value.status == C.NORMPRE_ERR_SHAPE
    bare = plan_for(4, 2, 64, "bf16", 64, False, norm=False)
    with pytest.raises(C.NormPreError) as e:
        bare.forward(q, k, p, qw, kw)
    assert e.value.status == C.NORMPRE_ERR_ARG
    plan.close()
    with pytest.raises(C.NormPreError) as e:
        plan.forward(q, k, p, qw, kw)
    assert e.value.status == C.NORMPRE_ERR_ARG
