"""The packed language model with windowed layers, rotated queries and keys and
clipped gradients: the operators as a training step uses them together."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_it_runs():
    from examples.train_packed_lm import train
    losses = train(steps=4, window=40, sinks=3, rotary=True, clip=1.0)
    assert len(losses) == 4 and all(math.isfinite(x) for x in losses)


@pytest.mark.parametrize("window, sinks", [(20, 0), (33, 4)])
def test_one_step_against_plain_torch(window, sinks):
    """Loss, gradients, their norm and the clipped gradients of a step against the
    same model in fp32 with plain torch operations; the tolerances of the model
    without these operators: bf16 activations round by 2^-8 at each of a dozen
    operations, and 8-bit checkpoints add about 1 % to the matrices' gradients.
    The norm is off by no more than the gradients are; clipping itself adds 1e-6."""
    import torch
    import torch.nn.functional as F
    from examples import train_packed_lm as T
    from paper_2609_36692_gb300 import layers
    from paper_2609_36692_gb300.optim import clip_grad_norm_

    torch.manual_seed(3)
    model = T.Model(64, 128, 2, 1, 192, 2, 128, rotary=True).cuda()
    with torch.no_grad():
        for b in model.blocks:
            for w in (b.q_norm, b.k_norm):
                w.copy_(1 + 0.3 * torch.randn_like(w))
    lengths, ids, places, targets = T.batch(torch.Generator().manual_seed(4), 512, 64, 128)
    plans = [layers.PackedAttention(2, 1, 64, max_tokens=512, max_seqs=64, window=w, sinks=s) for w, s in ((window, sinks), (0, 0))]
    for p in plans:
        p.set_lengths(lengths)
    loss = F.cross_entropy(model(ids, places, *plans), targets, ignore_index=-100)
    loss.backward()
    for p in plans:
        assert p.status() == 0
    got = {n: p.grad.clone() for n, p in model.named_parameters()}
    model.zero_grad(set_to_none=True)

    n = sum(lengths)
    seq = torch.repeat_interleave(torch.arange(len(lengths) + 1), torch.tensor(lengths + [512 - n])).cuda()
    at = torch.arange(512, device="cuda")
    whole = (seq[:, None] == seq) & (at <= at[:, None]) & (at < n)[:, None]
    near = (at[:, None] - at < window) | (places < sinks)[None, :]
    f = 10000.0 ** (-torch.arange(0, 64, 2, device="cuda") / 64)
    a = places[:, None, None] * f
    c, s = torch.cos(a), torch.sin(a)

    def turned(y, w):
        y = F.rms_norm(y, (64,), w, 1e-6)
        y1, y2 = y.split(32, -1)
        return torch.cat([y1 * c - y2 * s, y1 * s + y2 * c], -1)
    x = model.tokens[ids]
    for i, b in enumerate(model.blocks):
        y = F.rms_norm(x, x.shape[-1:], b.norm1) @ b.qkv.t()
        q, k, v = y.view(512, 4, 64).split([2, 1, 1], 1)
        # a padding row sees itself, so that the plain softmax has something to sum; it gives nothing
        seen = (whole & near if i == 0 else whole) | torch.eye(512, device="cuda").bool()
        z = torch.einsum("ihd,jkd->hij", turned(q, b.q_norm), turned(k, b.k_norm)) / 8
        p = torch.softmax(z.masked_fill(~seen, -math.inf), -1)
        o = torch.einsum("hij,jd->ihd", p, v[:, 0]) * (at < n)[:, None, None]
        x = x + o.reshape(512, 128) @ b.out.t()
        y = F.rms_norm(x, x.shape[-1:], b.norm2)
        x = x + (F.silu(y @ b.gate.t()) * (y @ b.up.t())) @ b.down.t()
    ref = F.cross_entropy(F.rms_norm(x, x.shape[-1:], model.norm) @ model.tokens.t(), targets, ignore_index=-100)
    ref.backward()
    assert abs(float(loss.detach()) - float(ref.detach())) < 2e-2
    for name, p in model.named_parameters():
        err = float((got[name] - p.grad).norm() / p.grad.norm())
        assert err < 6e-2, (name, err)
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in got.values()))
    want = math.sqrt(sum(float((p.grad.double() ** 2).sum()) for p in model.parameters()))
    assert abs(norm - want) < 6e-2 * want
    for name, p in model.named_parameters():
        p.grad = got[name].clone()
    assert abs(float(clip_grad_norm_(model.parameters(), 0.5 * norm)) - norm) < 1e-5 * norm
    for name, p in model.named_parameters():
        assert float((p.grad - 0.5 * got[name]).abs().max()) <= 1e-5 * float(got[name].abs().max())


def test_together_in_a_graph():
    """Norms with rotation, windowed attention, their gradients and clipping in one
    captured step: the bits of the calls one by one, replay after replay."""
    import torch
    from paper_2609_36692_gb300 import layers, optim
    torch.manual_seed(0)
    t, h, hk, d = 300, 4, 2, 64
    x = torch.randn(t, h + 2 * hk, d, device="cuda").bfloat16().requires_grad_()
    qw, kw = (torch.ones(d, device="cuda", requires_grad=True) for _ in range(2))
    places, dout = torch.arange(t, device="cuda"), torch.randn(t, h, d, device="cuda").bfloat16()
    rotary = layers.QKNormRotary(h, hk, d)
    attention = layers.PackedAttention(h, hk, d, t, 4, window=40, sinks=3)
    attention.set_lengths([200, 90])

    def step():
        q, k = rotary(x[:, :h], x[:, h:h + hk], places, qw, kw, used=290)
        out = attention(q, k, x[:, h + hk:])
        grads = torch.autograd.grad(out, (x, qw, kw), dout)
        clipped = [torch.empty_like(g) for g in grads]
        norm = optim.clip_grads(grads, 1.0, out=clipped)
        return [out.detach(), norm, *clipped]
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        for y in got:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert attention.status() == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want))
