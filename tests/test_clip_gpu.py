"""The global norm of gradients and clipping by it, against 64 bits.

Tolerances.  A thread sums the squares of 16 fp32 or 32 bf16 values in fp32, one
rounding of 2^-24 each, and all else is summed in 64 bits: the sum is off by at
most 32 * 2^-24, the norm by half of that plus its own rounding, 17 * 2^-24.  A
clipped value carries the norm's 16, the factor's rounding and the product's,
18 * 2^-24; in bf16 one rounding of 2^-8 besides.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-6


def dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def make(sizes, dtypes, seed=0, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale * 10.0 ** (i % 3 - 1)).to(dt(t))
            for i, (n, t) in enumerate(zip(sizes, dtypes))]


def exact(grads, max_norm, eps=EPS):
    square = sum(float((g.double() ** 2).sum()) for g in grads)
    n = math.sqrt(square)
    return n, min(1.0, max_norm / (n + eps))


def close(x, ref, c, n_tol=18 * U):
    """x = c ref, element by element."""
    import torch
    want = ref.double() * c
    tol = n_tol + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0)
    # numbers below 2^-126 have fixed steps
    assert bool(((x.double() - want).abs() <= tol * 1.01 * want.abs() + 2.0 ** -133).all())


LISTS = [[1], [0], [0, 0, 5], [7, 1, 333], [4096, 4095, 4097, 8192, 8191], [100000, 3, 70001], [1 << 20, 17], [2] * 65,
         [37] * 1000, [5000] * 130 + [0] + [1] * 900]


@pytest.mark.parametrize("to", ["place", "f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_norm_and_clip(sizes, dtype, to):
    import torch
    from paper_2609_36692_gb300 import optim
    dtypes = [("f32", "bf16")[i % 2] for i in range(len(sizes))] if dtype == "mixed" else [dtype] * len(sizes)
    grads = make(sizes, dtypes, len(sizes))
    keep = [g.clone() for g in grads]
    n, _ = exact(grads, 1.0)
    got = optim.grad_norm(grads)
    assert abs(float(got) - n) <= 17 * U * n
    for part in (0.37, 1.5):
        limit = part * n
        c = exact(grads, limit)[1]
        out = None if to == "place" else [torch.full_like(g, 7.0, dtype=dt(to)) for g in grads]
        same = optim.clip_grads(grads, limit, out=out)
        assert torch.equal(same, got)
        for g, k, o in zip(grads, keep, out or grads):
            if part > 1 and o.dtype == k.dtype:
                assert torch.equal(o, k)
            else:
                close(o, k, c)
            if out is not None:
                assert torch.equal(g, k)
            g.copy_(k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-44, 1e-38, 1e-30, 1e-19, 1.0, 1e18, 1e25, 3e38])
def test_squares_beyond_the_range_of_fp32(size, dtype):
    import torch
    from paper_2609_36692_gb300 import optim
    g = torch.full((5000,), size, device="cuda").to(dt(dtype))
    g[::7] = 0
    keep = g.clone()
    n = exact([g], 1.0)[0]
    got = float(optim.grad_norm([g]))
    if n < 3.4e38:
        assert abs(got - n) <= 17 * U * n + 2.0 ** -149
    else:
        assert got == math.inf
    out = torch.empty_like(g)
    optim.clip_grads([g], 0.25 * min(n, 1e38), eps=0.0, out=[out])
    # the library's max_norm is an fp32 number
    limit = float(torch.tensor(0.25 * min(n, 1e38), dtype=torch.float32))
    close(out, keep, min(1.0, limit / n) if n else 1.0)


def test_not_finite():
    import torch
    from paper_2609_36692_gb300 import optim
    for bad, norm in ((math.nan, math.nan), (math.inf, math.inf), (-math.inf, math.inf)):
        a, b = make([1000, 50], ["f32", "bf16"])
        a[777] = bad
        got = optim.clip_grads([a, b], 1.0)
        assert str(float(got)) == str(norm)
        if math.isnan(norm):
            assert bool(torch.isnan(a).all()) and bool(torch.isnan(b).all())
        else:                                     # finite values times zero
            assert math.isnan(float(a[777])) and not bool(torch.cat([a[:777], a[778:], b.float()]).any())
        a[777] = bad
        a[3] = math.nan
        assert math.isnan(float(optim.grad_norm([a, b])))


def test_zeros_and_limits():
    import torch
    from paper_2609_36692_gb300 import optim
    z = torch.zeros(100, device="cuda")
    for limit in (0.0, 1.0):
        assert float(optim.clip_grads([z], limit, eps=0.0)) == 0.0 and not bool(z.any())
    g = torch.tensor([3.0, 4.0], device="cuda")
    assert float(optim.clip_grads([g], 5.0, eps=0.0)) == 5.0 and g.tolist() == [3.0, 4.0]
    assert float(optim.clip_grads([g], 2.5, eps=0.0)) == 5.0 and g.tolist() == [1.5, 2.0]
    optim.clip_grads([g], 0.0)
    assert g.tolist() == [0.0, 0.0]
    assert float(optim.clip_grads([], 1.0)) == 0.0 == float(optim.grad_norm([]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("to", ["place", "f32", "bf16"])
def test_layouts_of_memory(dtype, to):
    """Slices at every offset of one buffer, transposed matrices, and outputs at
    offsets of their own: nothing around them changes."""
    import torch
    from paper_2609_36692_gb300 import optim
    sizes = [1, 2, 3, 5, 9, 17, 4099, 16385, 20000]
    base = torch.full((sum(sizes) + len(sizes) + 1,), 7.0, device="cuda").to(dt(dtype))
    buf = torch.full((sum(sizes) + 2 * len(sizes),), 7.0, device="cuda").to(dt(dtype if to == "place" else to))
    src = make(sizes, [dtype] * len(sizes), 3)
    grads, outs, at, to_at, hold, to_hold = [], [], 1, 0, [], []
    for x in src:
        grads.append(base[at:at + x.numel()])
        grads[-1].copy_(x)
        outs.append(buf[to_at:to_at + x.numel()])
        hold.append(at + x.numel())
        to_hold += [to_at + x.numel(), to_at + x.numel() + 1]
        at += x.numel() + 1
        to_at += x.numel() + 2
    m = torch.randn(60, 90, device="cuda").to(dt(dtype)).t()
    grads.append(m)
    src.append(m.clone())
    outs.append(torch.empty_strided(m.shape, m.stride(), dtype=buf.dtype, device="cuda"))
    n, c = exact(src, 2.0)
    got = optim.clip_grads(grads, 2.0, out=None if to == "place" else outs)
    assert abs(float(got) - n) <= 17 * U * n
    for x, o in zip(src, grads if to == "place" else outs):
        close(o, x, c)
    assert bool((base[hold] == 7.0).all()) and bool((buf[to_hold] == 7.0).all()) and float(base[0]) == 7.0


def test_same_bits_streams_and_capture():
    import torch
    from paper_2609_36692_gb300 import optim
    grads = make([50000, 7, 123457, 64], ["f32", "bf16", "bf16", "f32"], 9)
    out = [torch.empty_like(g) for g in grads]
    want_n = optim.clip_grads(grads, 1.0, out=out)
    want = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in out:
            o.zero_()
        got_n = optim.clip_grads(grads, 1.0, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got_n, want_n) and all(torch.equal(a, b) for a, b in zip(out, want))
    torch.cuda.synchronize()
    # two graphs with workspaces of their own, replayed at once
    graphs, norms = [torch.cuda.CUDAGraph() for _ in range(2)], []
    outs = [[torch.zeros_like(g) for g in grads] for _ in range(2)]
    for g, o in zip(graphs, outs):
        with torch.cuda.graph(g):
            norms.append(optim.clip_grads(grads, 1.0, out=o))
    for x in grads:
        x.mul_(2.0)                               # replays read what is there by then
    torch.cuda.synchronize()
    for s, g in zip((side, torch.cuda.Stream()), graphs):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    want_n = optim.clip_grads(grads, 1.0, out=out)
    for k, o in zip(norms, outs):
        assert torch.equal(k, want_n) and all(torch.equal(a, b) for a, b in zip(o, out))


def test_large():
    """Offsets past 2^31 elements."""
    import torch
    from paper_2609_36692_gb300 import optim
    g = torch.full(((1 << 31) + 5,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    g[-1] = 64.0
    n = math.sqrt(((1 << 31) + 4) * 2.0 ** -20 + 4096.0)
    got = optim.clip_grads([g], 0.5 * n, eps=0.0)
    assert abs(float(got) - n) <= 17 * U * n
    assert float(g[-1]) == 32.0 and bool((g[:-1] == 2.0 ** -11).all())


def test_parameters():
    """``clip_grad_norm_`` between a backward pass and a step."""
    import torch
    from paper_2609_36692_gb300.optim import NormPreOptimizer, clip_grad_norm_
    torch.manual_seed(0)
    w = [torch.nn.Parameter(torch.randn(64, 96, device="cuda")) for _ in range(3)]
    x = torch.randn(8, 96, device="cuda")
    (10 * (x @ w[0].t()).square().sum() + (x @ w[1].t()).sum()).backward()
    assert w[2].grad is None
    keep = [p.grad.clone() for p in w[:2]]
    n, c = exact(keep, 1.0)
    got = clip_grad_norm_(w, 1.0)
    assert abs(float(got) - n) <= 17 * U * n
    for p, k in zip(w, keep):
        close(p.grad, k, c)
    n = exact([w[0].grad], 1.0)[0]
    assert abs(float(clip_grad_norm_(w[0], 1e9)) - n) <= 17 * U * n
    w[2].grad = torch.zeros_like(w[2])
    opt = NormPreOptimizer(w, lr=0.01)
    before = [p.detach().clone() for p in w]
    opt.step()
    assert all(not torch.equal(a, p.detach()) for a, p in zip(before[:2], w[:2]))


def test_refusals():
    import torch
    from paper_2609_36692_gb300 import normpre as C
    from paper_2609_36692_gb300 import optim
    g = torch.ones(64, device="cuda")
    big = torch.ones(96, device="cuda")
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        optim.grad_norm([g, g.half()])
    for bad in (g.cpu(), torch.ones(8, 8, device="cuda")[:, :4], torch.ones(1, device="cuda").expand(5),
                torch.ones(4, 4, device="cuda").to_sparse()):
        with pytest.raises(ValueError):
            optim.grad_norm([g, bad])
    with pytest.raises(ValueError, match="tensor for each"):
        optim.clip_grads([g], 1.0, out=[])
    with pytest.raises(ValueError, match="shape"):
        optim.clip_grads([g], 1.0, out=[big])
    with pytest.raises(ValueError, match="strides"):
        optim.clip_grads([torch.ones(4, 6, device="cuda").t()], 1.0, out=[torch.ones(6, 4, device="cuda")])
    # memory that would be clipped twice, or overwritten while it is read
    h, half = torch.ones_like(g), big.view(torch.bfloat16)
    for grads, out in (([g, g], None), ([big[:64], big[32:]], None), ([big[:64]], [big[32:]]),
                       ([g, big[:64]], [big[32:], h]), ([g, h], [big[:64], big[32:]]), ([big], [half[:96]]),
                       ([g, h], [g, g])):
        with pytest.raises(C.NormPreError) as e:
            optim.clip_grads(grads, 1.0, out=out)
        assert e.value.status == C.NORMPRE_ERR_ARG
    for limit, eps in ((-1.0, 0.0), (math.nan, 0.0), (math.inf, 0.0), (1.0, -1.0), (1.0, math.nan)):
        with pytest.raises(C.NormPreError) as e:
            optim.clip_grads([g], limit, eps)
        assert e.value.status == C.NORMPRE_ERR_ARG
    assert bool((g == 1.0).all()) and bool((big == 1.0).all())
    optim.grad_norm([g, g])                        # read twice: the norm alone takes it
