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
