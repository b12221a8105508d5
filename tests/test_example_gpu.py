"""The packed language model example learns: attention, 8-bit checkpoints, gated
activation and the NormPre step run together as a user would run them."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_packed_language_model_learns():
    from examples.train_packed_lm import train
    losses = train(steps=240)
    assert all(math.isfinite(x) for x in losses)
    # the uniform guess costs ln 256 = 5.55; repeating the phrase costs little
    assert abs(losses[0] - math.log(256)) < 0.5
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0]


def test_one_step_against_plain_torch():
    """Loss and gradients of the first step against the same model in fp32 with
    plain torch operations.  bf16 activations round by 2^-8 at each of a dozen
    operations and 8-bit checkpoints add about 1% to the matrices' gradients."""
    import torch
    import torch.nn.functional as F
    from examples import train_packed_lm as T
    from paper_2609_36692_gb300 import layers

    torch.manual_seed(3)
    model = T.Model(64, 128, 2, 1, 192, 2, 128).cuda()
    lengths, ids, places, targets = T.batch(torch.Generator().manual_seed(4), 512, 64, 128)
    attention = layers.PackedAttention(2, 1, 64, max_tokens=512, max_seqs=64)
    attention.set_lengths(lengths)
    loss = F.cross_entropy(model(ids, places, attention), targets, ignore_index=-100)
    loss.backward()
    got = {n: p.grad.clone() for n, p in model.named_parameters()}
    model.zero_grad(set_to_none=True)

    seq = torch.repeat_interleave(torch.arange(len(lengths) + 1), torch.tensor(lengths + [512 - sum(lengths)])).cuda()
    at = torch.arange(512, device="cuda")
    # a padding row sees itself, so that the plain softmax has something to sum
    seen = ((seq[:, None] == seq) & (at <= at[:, None]) & (seq < len(lengths))[:, None]) | torch.eye(512, device="cuda").bool()
    x = model.tokens[ids] + model.places[places]
    for b in model.blocks:
        y = F.rms_norm(x, x.shape[-1:], b.norm1) @ b.qkv.t()
        q, k, v = y.view(512, 4, 64).split([2, 1, 1], 1)
        s = torch.einsum("ihd,jkd->hij", q, k) / 8
        p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
        x = x + torch.einsum("hij,jd->ihd", p, v[:, 0]).reshape(512, 128) @ b.out.t()
        y = F.rms_norm(x, x.shape[-1:], b.norm2)
        x = x + (F.silu(y @ b.gate.t()) * (y @ b.up.t())) @ b.down.t()
    ref = F.cross_entropy(F.rms_norm(x, x.shape[-1:], model.norm) @ model.tokens.t(), targets, ignore_index=-100)
    ref.backward()
    assert abs(float(loss.detach()) - float(ref.detach())) < 2e-2
    for n, p in model.named_parameters():
        err = float((got[n] - p.grad).norm() / p.grad.norm())
        assert err < 6e-2, (n, err)
