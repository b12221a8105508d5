"""The layer operators at the ends of their ranges: steps near the largest fp32
number in the weight gradient, large scores in attention, large gates; and what
the differentiable forms refuse.

References are in 64 bits; each test derives its tolerance.
"""
import pytest

from test_attention_gpu import TOL, err, make, plan_for, reference
from test_checkpoint_gpu import dt, rel, sample

pytestmark = pytest.mark.gpu


# few tiles (their tokens are split) and many (pairs of CTAs)
@pytest.mark.parametrize("shape", [(200, 264, 256), (64, 128, 128), (130, 5000, 1145)], ids=str)
@pytest.mark.parametrize("dy_dtype", ["f32", "bf16"])
def test_weight_gradient_of_large_steps(shape, dy_dtype):
    """Blocks on both sides of a step of 2^105 (below, 1e34, 3.3e38): what
    restores to finite values gives finite sums, zeros in dY included.  The
    tolerance is that of ordinary values, feature block by feature block."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    t, n, f = shape
    x = sample(t, t, f, "bf16").float()
    for i, top in enumerate((2.0 ** 111, 1e34, 3.3e38)):
        block = x[:, 32 * i:32 * i + 32]
        x[:, 32 * i:32 * i + 32] = block / block.abs().amax(1, keepdim=True) * top
    ck = L.ckpt_pack(x.to(torch.bfloat16))
    dy = sample(f, t, n, dy_dtype) * 1e-10
    dy[:, ::5] = 0
    ref = dy.double().T @ ck.restore(torch.float32).double()
    assert bool(torch.isfinite(ref).all())
    dw = L.ckpt_wgrad(dy, ck, dtype=dt("f32"))
    assert L.ckpt_status() == 0
    for k in range(0, f, 32):
        assert rel(dw[:, k:k + 32], ref[:, k:k + 32]) <= 1e-5, k


def exact_scores(seed, n, h, hk, dtype, base, spread=0):
    """q, k, v, dout of n rows with head_dim 64 whose scores are computed
    without rounding: whole numbers, and a scale of 1/8.  The scores are `base`
    (a multiple of 504), plus up to `spread` eighths."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = torch.full((n, h, 64), 64.0, device="cuda"), torch.full((n, hk, 64), float(base // 504), device="cuda")
    whole = lambda m, *shape: torch.randint(-m, m + 1, shape, generator=g, device="cuda").float()  # noqa: E731
    q[..., 0] = whole(2, n, h) if spread else 0.0
    k[..., 0] = whole(max(1, spread // 2), n, hk)
    v, do = (torch.randn(n, x, 64, generator=g, device="cuda") for x in (hk, h))
    return [x.to(dt(dtype)) for x in (q, k, v, do)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("base", [504 * 2, 504 * 64, 504 * 124, -504 * 124], ids=str)
def test_one_key_however_large_the_score(base, dtype):
    """p = 1 and the log-sum is the score itself, a number that fp32 holds: the
    output is the value and dv the output's gradient, to the bit."""
    import torch
    n, h, hk = 200, 2, 2
    q, k, v, do = exact_scores(1, n, h, hk, dtype, base)
    plan = plan_for(h, hk, 64, n, [1] * n, dtype)
    out, lse = plan.forward(q, k, v)
    dv = plan.backward(q, k, v, out, lse, do)[2]
    assert plan.status() == 0
    assert torch.equal(lse, torch.full_like(lse, float(base)))
    assert torch.equal(out, v) and torch.equal(dv, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("base", [504 * 64, 504 * 124], ids=str)
def test_many_keys_of_large_scores(base, dtype):
    """Scores around 32256 and 62496 that differ by up to 4.  Tolerances of
    ordinary scores; the fp32 log-sum adds half of its last place, 2^-10 or 2^-9,
    to the exponent of the backward pass."""
    n, h, hk, lengths = 700, 4, 2, [300, 1, 399]
    q, k, v, do = exact_scores(2, n, h, hk, dtype, base, 16)
    plan = plan_for(h, hk, 64, n, lengths, dtype)
    ref = reference(q, k, v, do, lengths)
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    assert plan.status() == 0
    half = 2.0 ** (-10 if base < 2 ** 15 else -9)
    assert float((lse.double() - ref[1]).abs().max()) <= 1.01 * half
    assert err(out, ref[0]) <= TOL[dtype, "fwd"]
    for x, r, m in zip(grads, ref[2:5], ref[5]):
        assert err(x, r, m) <= TOL[dtype, "bwd"] + half


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_swiglu_element_by_element(dtype):
    """Gates from -87 (below, exp(gate) leaves fp32's normal numbers) to 100,
    each element against its own size.  fp32: an exponential of 2 units in the
    last place, a quotient of 2, and three other roundings of a half, 5.5 *
    2^-23 = 6.6e-7; the backward pass has two roundings more and is measured
    against its terms before they cancel.  bf16: one rounding, 2^-8, besides."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    tol = 8e-7 + (2.0 ** -8 if dtype == "bf16" else 0)
    gate = torch.linspace(-87, 100, 64 * 96, device="cuda").view(64, 96).to(dt(dtype))
    up, dh = (sample(i, 64, 96, dtype) for i in (1, 2))
    h, cg, cu = L.ckpt_swiglu(gate, up)
    g, u = gate.double(), up.double()
    ref = g * torch.sigmoid(g) * u
    assert bool(((h.double() - ref).abs() <= tol * ref.abs() + 2.0 ** -126).all())
    g, u, d = cg.restore(torch.float32).double(), cu.restore(torch.float32).double(), dh.double()
    s = torch.sigmoid(g)
    dgate, dup = (x.double() for x in L.ckpt_swiglu_backward(cg, cu, dh))
    assert bool(((dup - d * g * s).abs() <= tol * (d * g * s).abs() + 2.0 ** -126).all())
    terms = (d * u * s).abs() * (1 + g.abs() * (1 - s))
    assert bool(((dgate - d * u * s * (1 + g * (1 - s))).abs() <= tol * terms + 2.0 ** -126).all())


def test_second_derivatives_are_refused():
    """The backward passes fill their results outside autograd: a second
    derivative would miss their terms without a word."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    leaf = lambda *shape: torch.randn(*shape, device="cuda").to(torch.bfloat16).requires_grad_()  # noqa: E731
    q, k, v = leaf(40, 2, 64), leaf(40, 1, 64), leaf(40, 1, 64)
    plan = plan_for(2, 1, 64, 40, [40], "bf16")
    for f, leaves in ((plan, (q, k, v)), (L.linear, (leaf(40, 64), leaf(32, 64))), (L.swiglu, (leaf(40, 64), leaf(40, 64)))):
        grads = torch.autograd.grad((f(*leaves) ** 2).sum(), leaves, create_graph=True)
        for g in grads:
            with pytest.raises(RuntimeError, match="once_differentiable"):
                (g ** 2).sum().backward(retain_graph=True)


def test_backward_pass_of_other_lengths_is_refused():
    import torch
    q, k, v, do = make(3, 64, 2, 1, 64, "bf16")
    plan = plan_for(2, 1, 64, 64, [40, 24], "bf16")
    want = plan.backward(q, k, v, *plan.forward(q, k, v), do)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    out = plan(*leaves)
    plan.set_lengths([24, 40])
    with pytest.raises(RuntimeError, match="lengths changed"):
        torch.autograd.grad(out, leaves, do, retain_graph=True)
    plan.set_lengths(torch.tensor([40, 24]))           # the call's lengths again
    for x, y in zip(torch.autograd.grad(out, leaves, do), want):
        assert torch.equal(x, y)


def test_stream_argument():
    """Work on a stream given by argument: the same bits, and outputs that do
    not lie where the current stream still has work to do."""
    import torch
    n, h, hk = 1024, 2, 1
    q, k, v, do = make(4, n, h, hk, 64, "bf16")
    plan = plan_for(h, hk, 64, n, [1000], "bf16")
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def while_memory_is_in_use(shapes, f):
        held = [torch.full(s, 3.0, dtype=t, device="cuda") for s, t in shapes]
        torch.cuda._sleep(200_000_000)               # a tenth of a second
        copies = [x.clone() for x in held]
        del held                                     # what is still to be copied is free for others
        got = f()
        torch.cuda.synchronize()
        for x in copies:
            assert bool((x == 3.0).all())
        return got
    o2, l2 = while_memory_is_in_use([(out.shape, out.dtype), (lse.shape, lse.dtype)],
                                    lambda: plan.forward(q, k, v, stream=side))
    g2 = while_memory_is_in_use([(x.shape, x.dtype) for x in grads],
                                lambda: plan.backward(q, k, v, out, lse, do, stream=side))
    assert plan.status(side) == 0
    for x, y in zip((o2, l2, *g2), (out, lse, *grads)):
        assert torch.equal(x, y)
    o3, g3 = torch.empty_like(out), torch.empty_like(grads[0])   # given outputs
    side.wait_stream(torch.cuda.current_stream())
    assert plan.forward(q, k, v, out=o3, stream=side)[0] is o3
    assert plan.backward(q, k, v, out, lse, do, dq=g3, stream=side)[0] is g3
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o3, out) and torch.equal(g3, grads[0])


def test_a_wait_that_gave_up_is_reported_by_the_next_call():
    """With test_stall one CTA loads nothing: its waits give up after two seconds
    and the kernel ends.  No call of the plan then passes, the differentiable
    form's neither, until its status has been asked."""
    import torch
    from paper_2609_36692_gb300 import normpre as C
    q, k, v, do = make(6, 500, 2, 1, 64, "bf16")
    plan = plan_for(2, 1, 64, 500, [300, 200], "bf16")
    out, lse = plan.forward(q, k, v)
    plan.close()
    plan.plan = C.normpre_attn_init(C.normpre_attn_config(2, 1, 64, 2, 500, C.NORMPRE_BF16, 0.0, 1))
    plan.set_lengths([300, 200])
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    got = plan(*leaves)                       # asynchronous: nothing to report yet
    torch.cuda.synchronize()
    for f in (lambda: got.backward(do), lambda: plan(*leaves), lambda: plan.backward(q, k, v, out, lse, do)):
        with pytest.raises(C.NormPreError, match="gave up") as e:
            f()
        assert e.value.status == C.NORMPRE_ERR_TIMEOUT
    assert plan.status(raise_on_error=False) == C.NORMPRE_ERR_TIMEOUT
    assert plan.status() == C.NORMPRE_OK
    grads = plan.backward(q, k, v, out, lse, do)   # the context is usable, and the plan too
    assert plan.status() == C.NORMPRE_OK
    for x, r, m in zip(grads, *(lambda ref: (ref[2:5], ref[5]))(reference(q, k, v, do, [300, 200]))):
        assert err(x, r, m) <= TOL["bf16", "bwd"]


def test_checkpoint_capture_in_a_graph():
    """Pack, weight gradient, restore and SwiGLU captured in a process that has
    made no call of theirs before."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2609_36692_gb300 import layers as L
x, dy, up = (torch.randn(300, n, device="cuda").to(torch.bfloat16) for n in (256, 136, 256))
def calls():
    ck = L.ckpt_pack(x)
    h, cg, cu = L.ckpt_swiglu(x, up)
    return (ck.restore(), L.ckpt_wgrad(dy, ck), h, *L.ckpt_swiglu_backward(cg, cu, x))
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = calls()
for _ in range(2):
    for y in got:
        y.zero_()
    g.replay()
assert L.ckpt_status() == 0
assert all(torch.equal(a, b) for a, b in zip(got, calls()))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("shape", [(96,), (3, 40, 96), (2, 0, 96)], ids=str)
def test_linear_of_any_leading_dimensions(shape):
    """As many dimensions as the call takes when no gradient is kept; the bits of
    the same rows as a matrix."""
    import torch
    from paper_2609_36692_gb300 import layers as L
    x = torch.randn(*shape, device="cuda").to(torch.bfloat16)
    w = torch.randn(64, 96, device="cuda").requires_grad_()
    rows = [x.reshape(-1, 96).clone().requires_grad_(), w.detach().clone().requires_grad_()]
    y2 = L.linear(*rows)
    x.requires_grad_()
    y = L.linear(x, w)
    with torch.no_grad():
        assert y.shape == L.linear(x, w).shape == (*shape[:-1], 64)
    dy = torch.randn_like(y)
    y.backward(dy)
    y2.backward(dy.reshape(-1, 64))
    assert torch.equal(w.grad, rows[1].grad)
    # the library's products of other shapes may sum in another order
    assert x.grad.shape == x.shape and rel(x.grad.reshape(-1, 96), rows[0].grad.double()) <= 2.0 ** -8
    # a gradient that is expanded, or has its rows elsewhere
    w.grad = None
    L.linear(x, w).sum().backward()
    ref = torch.ones(64, 1, device="cuda").double() @ L.ckpt_pack(x.detach().reshape(-1, 96)).restore().double().sum(0, keepdim=True)
    assert rel(w.grad, ref) <= 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_and_calls_on_different_streams(dtype):
    """A call uses the lengths that were set before it, on whatever stream, and
    not those that are set while it waits for its turn."""
    import torch
    n, h, hk = 600, 2, 1
    packs = ([600], [37] * 16, [1, 300, 299])
    q, k, v, do = make(7, n, h, hk, 64, dtype)
    plan = plan_for(h, hk, 64, n, packs[1], dtype)

    def both(stream=None):
        out, lse = plan.forward(q, k, v, stream=stream)
        return (out, lse, *plan.backward(q, k, v, out, lse, do, stream=stream))
    want = []
    for lengths in packs:
        plan.set_lengths(lengths)
        want.append(both())
    side = torch.cuda.Stream()
    got = []
    for lengths in packs:
        torch.cuda._sleep(20_000_000)                  # the copy of the lengths waits on the current stream
        plan.set_lengths(lengths)
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)              # and the calls on theirs
        got.append(both(side))
    # lengths copied on the other stream, calls on the current one
    side.wait_stream(torch.cuda.current_stream())
    for lengths in packs:
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        plan.set_lengths(lengths, stream=side)
        got.append(both())
    torch.cuda.synchronize()
    assert plan.status() == 0
    for i, outs in enumerate(got):
        for x, y in zip(outs, want[i % 3]):
            assert torch.equal(x, y), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replay_under_other_lengths_stays_in_range(dtype):
    """A captured call knows the number of blocks of its own lengths.  Replayed
    with the lists of others it writes no row but the call's, ends, and gives the
    right bits again once its lengths are back."""
    import torch
    h, hk, d, n, room = 4, 2, 64, 700, 64
    own, others = [123, 277], [[700], [1] * 100, [5] * 140, [0, 400], []]
    # a process whose plans take up to 700 rows; the call's are 400, with rows around them that nobody owns
    names = [("q", h), ("k", hk), ("v", hk), ("o", h), ("do", h), ("dq", h), ("dk", hk), ("dv", hk)]
    big = {name: torch.full((400 + 2 * room, x, d), 7.0, device="cuda", dtype=dt(dtype)) for name, x in names}
    t = {name: x[room:room + 400] for name, x in big.items()}
    for name, x in zip(("q", "k", "v", "do"), make(8, 400, h, hk, d, dtype)):
        t[name].copy_(x)
    lse = torch.full((h, 400), 7.0, device="cuda")
    plan = plan_for(h, hk, d, n, [1] * 140, dtype)
    plan.set_lengths(own)

    def calls():
        plan.forward(t["q"], t["k"], t["v"], out=t["o"], lse=lse)
        plan.backward(t["q"], t["k"], t["v"], t["o"], lse, t["do"], t["dq"], t["dk"], t["dv"])
    calls()
    torch.cuda.synchronize()
    want = {name: x.clone() for name, x in big.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for lengths in others:
        plan.set_lengths(lengths)
        g.replay()
        torch.cuda.synchronize()
        plan.status(raise_on_error=False)
        for name, x in big.items():
            assert bool((x[:room] == 7.0).all()) and bool((x[room + 400:] == 7.0).all()), name
        plan.set_lengths(own)
        g.replay()
        torch.cuda.synchronize()
        assert plan.status() == 0
        for name, x in big.items():
            assert torch.equal(x, want[name]), name
