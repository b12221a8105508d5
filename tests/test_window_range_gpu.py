"""Windowed attention where scores are sharp, so that the running maximum is raised
in every kind of block, and where values are large.

Tolerances: those of test_attention_gpu, and what a score of size s carries into an
exponential: d products added in fp32, sqrt(d) 2^-24 s with random signs, once
in the score and once in the log-sum.
"""
import math

import pytest

from test_attention_gpu import TOL, err, make, plan_for
from test_window_gpu import reference

pytestmark = pytest.mark.gpu

LAYOUTS = [(2, 2, 64), (4, 2, 128), (3, 1, 128)]
WINDOWS = [(300, 7), (300, 0), (600, 4), (200, 40), (1000, 0)]    # both kinds of kernels, with and without sinks
LENGTHS = [1700, 450, 1]


def sharp(mode, layout, window, sinks, dtype):
    """Ordinary scores and, in the first dimension, s nats that keys add: 20 more for
    each 128 keys further on ("steps"; odd heads: less, so that the maximum moves at
    every block on the way down), or only some keys, 30 nats above all others
    ("spikes": one of them in each window, at every distance, and two sinks more)."""
    import torch
    h, hk, d = layout
    n = sum(LENGTHS) + 5
    q, k, v, do = (x.contiguous() for x in make(window + d, n, h, hk, d, dtype))
    at = torch.cat([torch.arange(m, device="cuda") for m in LENGTHS + [5]])
    if mode == "steps":
        s, sign = at * (20.0 / 128), [1.0 if i % 2 else -1.0 for i in range(h)]
    else:
        s, sign = torch.where(at % (window - 10) == window // 2, 30.0, 0.0), [1.0] * h
        if sinks:
            s[at == sinks - 1] = 60.0
    k[:, :, 0] = (s * (math.sqrt(d) / 4.0)).to(k.dtype)[:, None]
    q[:, :, 0] = 4.0 * torch.tensor(sign, device="cuda")
    return q, k, v, do


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("window, sinks", WINDOWS)
@pytest.mark.parametrize("mode", ["steps", "spikes"])
def test_the_maximum_moves(mode, window, sinks, layout, dtype):
    h, hk, d = layout
    q, k, v, do = sharp(mode, layout, window, sinks, dtype)
    n = sum(LENGTHS)
    plan = plan_for(h, hk, d, n + 5, LENGTHS, dtype, window=window, sinks=sinks)
    ref = reference(q, k, v, do, LENGTHS, window, sinks)
    out, lse = plan.forward(q, k, v)
    grads = plan.backward(q, k, v, out, lse, do)
    assert plan.status() == 0
    size = float(ref[1][:, :n].abs().max())
    assert float((lse[:, :n].double() - ref[1][:, :n]).abs().max()) <= 2e-5 * max(1.0, size)
    more = 2 * math.sqrt(d) * 2.0 ** -24 * size
    for name, x, r in zip(("out", "dq", "dk", "dv"), (out, *grads), (ref[0], *ref[2:5])):
        tol, terms = TOL[dtype, "fwd" if name == "out" else "bwd"], ref[5][name]
        assert err(x, r, float(terms.sum()) ** 0.5) <= tol + more, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_large_values(window, sinks, layout, dtype):
    """Values of 2^108 behind keys that are 15 nats (a factor of 2^22) above those
    that a row meets first: what is summed on the way stays in fp32's range, as
    without a window (up to 2^120 over the number of keys)."""
    import torch
    h, hk, d = layout
    q, k, v, do = sharp("spikes", layout, window, sinks, dtype)
    k[:, :, 0] = torch.clamp(k[:, :, 0], max=15.0 * math.sqrt(d) / 4.0)
    q[:, :, 1:] *= 0.1                               # the others do not add to it
    v = v * 2.0 ** 108
    n = sum(LENGTHS)
    plan = plan_for(h, hk, d, n + 5, LENGTHS, dtype, window=window, sinks=sinks)
    ref = reference(q, k, v, do, LENGTHS, window, sinks)
    out, lse = plan.forward(q, k, v)
    assert plan.status() == 0
    assert bool(torch.isfinite(out).all())
    assert err(out, ref[0], float(ref[5]["out"].sum()) ** 0.5) <= TOL[dtype, "fwd"] + 2 * math.sqrt(d) * 2.0 ** -24 * 30
