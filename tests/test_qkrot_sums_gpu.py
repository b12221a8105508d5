"""The sums over rows in the weights' gradients of the query and key norms.

All terms here are exact: rows of 1 and -1 have the inverse root 1 with this eps,
and position 0 turns nothing, so that a term is dz times 1 or -1.  What is left is
the sums' own rounding.
"""
import pytest

from test_qkrot_gpu import U, dt

pytestmark = pytest.mark.gpu


def calls(dtype, h, hk, d, value):
    """dq_weight and dk_weight of rows whose terms are value(tokens, heads)."""
    import torch
    from paper_2609_36692_gb300.layers import QKNormRotary
    g = torch.Generator(device="cuda").manual_seed(d)
    plan = QKNormRotary(h, hk, d, eps=1e-30, dtype=dt(dtype))
    v = [value(n).double() for n in (h, hk)]
    x = [torch.randint(0, 2, y.shape, generator=g, device="cuda") * 2.0 - 1.0 for y in v]
    dz = [(a * b).to(dt(dtype)) for a, b in zip(x, v)]
    x = [a.to(dt(dtype)) for a in x]
    w = torch.ones(d, device="cuda")
    pos = torch.zeros(x[0].shape[0], dtype=torch.int64, device="cuda")
    got = plan.backward(*x, pos, *dz, w, w)[2:]
    return list(zip(got, v))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_large_row_among_many(dtype):
    """Terms of 1 behind one of 2^24 in three hundred.  At most 16 rows are added in
    one fp32 number, 15 roundings of 2^-24; what two fp32 numbers and fp64 numbers
    add to that is below 2^-40, and the result is rounded once.  A lane's 300 rows
    in one fp32 number would lose half of them."""
    import torch
    n, d = 60000, 128

    def value(heads):
        v = torch.ones(n, heads, d, device="cuda")
        v[torch.arange(n, device="cuda") // 2 % 18 == 0, 0] = 2.0 ** 24
        return v
    for got, v in calls(dtype, 16, 8, d, value):
        want = v.sum((0, 1))
        assert float(((got.double() - want).abs() / (16 * U * want)).max()) <= 1.01


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens, layout", [(1, (4, 2, 64)), (77, (5, 3, 64)), (2999, (3, 1, 128)), (20000, (16, 8, 128))])
def test_every_row_once(tokens, layout, dtype):
    """Whole numbers whose partial sums stay below 2^24: equal, whatever the order."""
    import torch
    h, hk, d = layout
    g = torch.Generator(device="cuda").manual_seed(tokens)
    for got, v in calls(dtype, h, hk, d, lambda n: torch.randint(-3, 8, (tokens, n, d), generator=g, device="cuda")):
        assert torch.equal(got.double(), v.sum((0, 1)))
