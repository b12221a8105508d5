"""The layer operators at the ends of their ranges: steps near the largest fp32
number in the weight gradient.

References are in 64 bits; each test derives its tolerance.
"""
import pytest

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
