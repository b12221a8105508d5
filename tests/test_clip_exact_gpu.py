"""The norm and the clip factor by themselves: where the squares' sum is a whole
number that all sums hold exactly, both are their 64-bit values rounded once."""
import math

import pytest

pytestmark = pytest.mark.gpu


def half_ulp(x):
    """Half a step of fp32 at x (a normal number)."""
    return 2.0 ** (math.frexp(x)[1] - 25)


@pytest.mark.parametrize("shift", [0, -40, 40])
def test_norm_and_factor_are_rounded_once(shift):
    """A gradient of whole numbers, times 2^shift, of which one is 1: its clipped
    value is the factor (times 2^shift, exactly).  The library's own error before
    the last rounding, 2^-45, is below 2^-20 of half a step."""
    import numpy as np
    import torch
    from paper_2609_36692_gb300 import optim
    rng = np.random.default_rng(5)
    unit = 2.0 ** shift
    for i in range(150):
        x = np.concatenate([[1], rng.integers(-300, 301, size=int(rng.integers(1, 60)))])
        g = (torch.from_numpy(x).float() * unit).cuda()
        n = math.sqrt(float((x.astype(np.int64) ** 2).sum())) * unit
        limit = float(np.float32(n * rng.uniform(0.01, 0.99)))
        eps = float(np.float32(rng.choice([0.0, 1e-6, 0.1]) * unit))
        out = [torch.empty_like(g)]
        norm = float(optim.clip_grads([g], limit, eps=eps, out=out))
        assert abs(norm - n) <= half_ulp(n) * (1 + 2.0 ** -20)
        c = min(1.0, limit / (n + eps))
        assert abs(float(out[0][0]) / unit - c) <= half_ulp(c) * (1 + 2.0 ** -20), (i, limit, eps)
        assert float(optim.grad_norm([g])) == norm


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_each_value_once(dtype):
    """Slices of one buffer side by side, which share lines of memory with their
    neighbours in other CTAs: each value is halved once, whoever is first."""
    import torch
    from paper_2609_36692_gb300 import optim
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    sizes = [1 + (i * 7919) % 9001 for i in range(400)]
    buf = torch.ones(sum(sizes) + 2, dtype=t, device="cuda")
    grads = list(buf[1:-1].split(sizes))
    n = math.sqrt(sum(sizes))
    for i in range(10):
        # the norm is n 2^-i, the limit half of it, both rounded once; the factor is within 2^-22 of a half
        c = float(torch.tensor(0.5 * n * 2.0 ** -i, dtype=torch.float32)) / (n * 2.0 ** -i)
        before = buf.clone()
        optim.clip_grads(grads, c * n * 2.0 ** -i, eps=0.0)
        want = before[1:-1].float() * torch.tensor(c, dtype=torch.float32, device="cuda")
        assert bool((buf[1:-1].float() - want).abs().max() <= 2.0 ** -22 * want.max() + (2.0 ** -8 * want.max() if dtype == "bf16" else 0))
        assert float(buf[0]) == 1.0 == float(buf[-1])
        buf[1:-1] = 2.0 ** -(i + 1)


def test_an_infinite_limit_asks_for_the_norm_alone():
    import torch
    from paper_2609_36692_gb300 import optim
    p = [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (9, 16, 5)]
    assert float(optim.clip_grad_norm_(p, math.inf)) == 0.0
    p[0].grad, p[1].grad = (torch.full_like(x, y) for x, y in zip(p, (1.0, 2.5)))
    p[0].grad[3] = 0.0
    keep = [x.grad.clone() for x in p[:2]]
    for limit in (math.inf, torch.tensor(math.inf)):
        assert float(optim.clip_grad_norm_(p, limit)) == float(torch.tensor(math.sqrt(108.0), dtype=torch.float32))
        assert all(torch.equal(x.grad, k) for x, k in zip(p, keep))
    assert float(optim.clip_grad_norm_(p[0], math.inf)) == float(torch.tensor(math.sqrt(8.0), dtype=torch.float32))
    for bad in (-math.inf, math.nan):
        with pytest.raises(RuntimeError):
            optim.clip_grad_norm_(p, bad)
