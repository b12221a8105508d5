"""The layer operators where their work no longer fits one round: more items
than are dealt out to the CTAs beforehand, more items a CTA than it looks up at
once, every number of CTAs that can share a weight gradient's tile, and more
tiles than clusters.  References and tolerances are those of the operators'
other tests.
"""
import pytest

from test_attention_gpu import check_backward, check_forward, make, plan_for
from test_checkpoint_gpu import definition, rel, sample, unpacked

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [(64, 64, 8), (64, 2, 64)], ids=str)
@pytest.mark.parametrize("seqs", [100, 130], ids=str)
def test_many_items(seqs, layout, dtype):
    h, hk, d = layout
    lengths = [1 + (29 * i) % 128 for i in range(seqs)]
    q, k, v, do = make(seqs + d, sum(lengths), h, hk, d, dtype)
    plan = plan_for(h, hk, d, sum(lengths), lengths, dtype)
    out, lse, ref = check_forward(plan, q, k, v, do, lengths, dtype)
    check_backward(plan, q, k, v, do, out, lse, ref, lengths, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sequences_of_one_token(dtype):
    """Every row sees itself alone: its output is its value, and its gradient
    reaches v only."""
    h, hk, d, n = 4, 2, 64, 700
    q, k, v, do = make(1, n, h, hk, d, dtype)
    plan = plan_for(h, hk, d, n, [1] * n, dtype)
    out, lse, ref = check_forward(plan, q, k, v, do, [1] * n, dtype)
    check_backward(plan, q, k, v, do, out, lse, ref, [1] * n, dtype)


def test_many_backward_passes_in_a_row():
    """No wait gives up and the bits stay the same over a long queue of passes."""
    import torch
    for h, hk, d, lengths in ((32, 8, 64, [2048] * 2), (8, 4, 128, [1700, 1, 900])):
        q, k, v, do = make(2, sum(lengths), h, hk, d, "bf16")
        plan = plan_for(h, hk, d, sum(lengths), lengths, "bf16")
        out, lse = plan.forward(q, k, v)
        first = plan.backward(q, k, v, out, lse, do)
        grads = [torch.empty_like(x) for x in first]
        for _ in range(6):
            for _ in range(250):
                plan.backward(q, k, v, out, lse, do, *grads)
            assert plan.status() == 0
            for a, b in zip(first, grads):
                assert torch.equal(a, b)


# tiles of 128 features x 256 outputs: 18, 25, 30, 36, 49 and 66 of them leave
# room for 8, 6, 5, 4, 3 and 2 CTAs each
@pytest.mark.parametrize("tiles", [(3, 6), (5, 5), (5, 6), (6, 6), (7, 7), (6, 11), (1, 1)], ids=str)
@pytest.mark.parametrize("tokens", [1100, 200], ids=str)
def test_weight_gradient_shared_tiles(tiles, tokens):
    import torch
    from paper_2609_36692_gb300 import layers as L
    n, f = 256 * tiles[0] - 8, 128 * tiles[1] - 5
    ck = L.ckpt_pack(sample(n + tokens, tokens, f, "bf16"))
    dy = sample(f, tokens, n, "bf16")
    ref = dy.double().T @ ck.restore(torch.float32).double()
    dw = L.ckpt_wgrad(dy, ck, dtype=torch.float32)
    assert L.ckpt_status() == 0
    assert rel(dw, ref) <= 1e-5
    assert torch.equal(dw, L.ckpt_wgrad(dy, ck, dtype=torch.float32))


# two, three and four rounds over the clusters; odd numbers of feature tiles
@pytest.mark.parametrize("shape", [(5000, 1145), (5000, 1153), (6144, 2176), (8192, 2700), (200, 33000)], ids=str)
@pytest.mark.parametrize("tokens", [1, 130, 700], ids=str)
def test_weight_gradient_several_rounds(shape, tokens):
    import torch
    from paper_2609_36692_gb300 import layers as L
    n, f = shape
    ck = L.ckpt_pack(sample(n + tokens, tokens, f, "bf16"))
    dy = sample(f, tokens, n, "bf16")
    ref = dy.double().T @ ck.restore(torch.float32).double()
    dw = L.ckpt_wgrad(dy, ck, dtype=torch.float32)
    assert L.ckpt_status() == 0
    assert rel(dw, ref) <= 1e-5
    L.ckpt_wgrad(dy, ck, out=dw, accumulate=True)
    assert rel(dw, 2 * ref) <= 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(9000, 300), (40001, 65), (3, 70001)], ids=str)
def test_pack_of_many_blocks(shape, dtype):
    import numpy as np
    import torch
    from paper_2609_36692_gb300 import layers as L
    x = sample(shape[0], *shape, dtype)
    ck = L.ckpt_pack(x)
    codes, steps, values = definition(x.float().cpu().numpy())
    got_codes, got_steps = unpacked(ck)
    assert np.array_equal(got_codes, codes) and np.array_equal(got_steps, steps)
    assert np.array_equal(ck.restore(torch.float32).cpu().numpy().astype(np.float64), values)


@pytest.mark.parametrize("shape", [(9000, 300), (40001, 65), (3, 70001)], ids=str)
def test_swiglu_of_many_blocks(shape):
    import torch
    from paper_2609_36692_gb300 import layers as L
    g, u, dh = (sample(i, *shape, "f32").clamp(-30, 30) for i in range(3))
    h, cg, cu = L.ckpt_swiglu(g, u)
    s = torch.sigmoid(g.double())
    assert rel(h, g.double() * s * u.double()) <= 2e-6
    g, u = cg.restore(torch.float32).double(), cu.restore(torch.float32).double()
    dg, du = L.ckpt_swiglu_backward(cg, cu, dh)
    s = torch.sigmoid(g)
    assert rel(dg, dh.double() * u * s * (1 + g * (1 - s))) <= 2e-6
    assert rel(du, dh.double() * g * s) <= 2e-6
