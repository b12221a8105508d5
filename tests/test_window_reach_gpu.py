"""How far a value that is not finite reaches in the backward pass of windowed
attention: the blocks of 128 keys that its row's block of 128 rows meets."""
import math

import pytest

from test_attention_gpu import make, plan_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [(2, 1, 64), (3, 3, 128)], ids=str)
@pytest.mark.parametrize("sinks", [0, 2])
@pytest.mark.parametrize("which", ["q", "do", "out", "lse"])
def test_rows_that_are_not_finite(which, sinks, layout, dtype):
    """Row 700 lies in block 5 (640 .. 767), which meets the keys from 441 on: blocks
    3 to 5, and with sinks block 0."""
    import torch
    h, hk, d = layout
    n, row = 1000, 700
    q, k, v, do = (x.contiguous() for x in make(9, n, h, hk, d, dtype))
    plan = plan_for(h, hk, d, n, [n], dtype, window=200, sinks=sinks)
    out, lse = plan.forward(q, k, v)
    want = plan.backward(q, k, v, out, lse, do)
    x = {"q": q.clone(), "do": do.clone(), "out": out.clone(), "lse": lse.clone()}
    if which == "lse":
        x["lse"][:, row] = math.nan
    else:
        x[which][row] = math.nan
    got = plan.backward(x["q"], k, v, x["out"], x["lse"], x["do"])
    assert plan.status() == 0
    others = torch.arange(n, device="cuda") != row
    assert torch.equal(got[0][others], want[0][others])
    assert bool(torch.isnan(got[0][row]).all())
    seen = slice(row - 199, row + 1)
    for a, b in zip(got[1:], want[1:]):
        for keys in (slice(0 if sinks == 0 else 128, 384), slice(768, n)):
            assert torch.equal(a[keys], b[keys])
    # o reaches dk through delta, which dv does not need
    assert bool(torch.isnan(got[1][seen]).all())
    assert which == "out" or bool(torch.isnan(got[2][seen]).all())
    if which == "out":
        assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_that_are_not_finite(dtype):
    """Key 300 lies in block 2 (256 .. 383); the rows of its own block and those up to
    383 + 199 meet it, blocks 2 to 4."""
    import torch
    h, hk, d, n = 2, 1, 64, 1000
    q, k, v, do = (x.contiguous() for x in make(9, n, h, hk, d, dtype))
    plan = plan_for(h, hk, d, n, [n], dtype, window=200, sinks=2)
    out, lse = plan.forward(q, k, v)
    want = plan.backward(q, k, v, out, lse, do)
    for i in (1, 2):
        x = [q, k.clone(), v.clone()]
        x[i][300] = math.nan
        o2, l2 = plan.forward(*x)
        got = plan.backward(*x, out, lse, do)
        for rows in (slice(0, 256), slice(640, n)):
            assert torch.equal(o2[rows], out[rows]) and torch.equal(l2[:, rows], lse[:, rows])
            assert torch.equal(got[0][rows], want[0][rows])
    assert plan.status() == 0
