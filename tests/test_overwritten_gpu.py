"""Calls that write tensors of the caller's tell autograd: a backward pass that
needs what such a tensor held raises instead of running on other values."""
import pytest

from test_attention_gpu import make, plan_for

pytestmark = pytest.mark.gpu

MODIFIED = "modified by an inplace operation"


def test_clipped_gradients():
    import torch
    from paper_2609_36692_gb300 import optim
    x = torch.randn(50, 30, device="cuda", requires_grad=True)
    for clip in (lambda g: optim.clip_grads([g], 1e-3), lambda g: optim.clip_grads([torch.ones_like(g)], 1.0, out=[g])):
        g, = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
        penalty = (g ** 2).sum()                      # keeps g
        clip(g.detach())
        with pytest.raises(RuntimeError, match=MODIFIED):
            penalty.backward()
    p = torch.nn.Parameter(torch.randn(50, 30, device="cuda"))
    (p ** 2).sum().backward(create_graph=True)
    penalty = (p.grad ** 2).sum()
    optim.clip_grad_norm_([p], 1e-3)
    with pytest.raises(RuntimeError, match=MODIFIED):
        penalty.backward()
    # the norm alone writes nothing
    g, = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
    penalty = (g ** 2).sum()
    optim.grad_norm([g])
    penalty.backward()


def saved_by(x):
    """A result whose backward pass needs x."""
    import torch
    w = torch.ones_like(x, requires_grad=True)
    return (x * w).sum()


def test_norms_over_their_inputs():
    import torch
    from paper_2609_36692_gb300.layers import QKNormRotary
    q, k, v, do = (x.contiguous() for x in make(1, 40, 4, 2, 64, "bf16"))
    plan = QKNormRotary(4, 2, 64)
    pos = torch.arange(40, device="cuda")
    for name in ("q_out", "k_out"):
        x = {"q_out": q, "k_out": k}[name]
        kept = saved_by(x)
        plan.forward(q, k, pos, **{name: x})
        with pytest.raises(RuntimeError, match=MODIFIED):
            kept.backward()
    for name in ("dq", "dk"):
        dz = {"dq": do.clone(), "dk": k.clone()}
        kept = saved_by(dz[name])
        plan.backward(q, k, pos, dz["dq"], dz["dk"], **{name: dz[name]})
        with pytest.raises(RuntimeError, match=MODIFIED):
            kept.backward()
    kept = saved_by(q), saved_by(k)
    plan.forward(q, k, pos)
    plan.backward(q, k, pos, do, k)
    for x in kept:
        x.backward()


def test_attention_and_checkpoints():
    import torch
    from paper_2609_36692_gb300 import layers
    q, k, v, do = (x.contiguous() for x in make(2, 300, 4, 2, 64, "bf16"))
    plan = plan_for(4, 2, 64, 300, [300], "bf16", window=100)
    out, lse = plan.forward(q, k, v)
    dq, dk, dv = plan.backward(q, k, v, out, lse, do)
    ck = layers.ckpt_pack(q.view(300, 256))
    r, w = ck.restore(), layers.ckpt_wgrad(do.view(300, 256), ck)
    for x, call in ((out, lambda: plan.forward(q, k, v, out=out)), (lse, lambda: plan.forward(q, k, v, lse=lse)),
                    (dq, lambda: plan.backward(q, k, v, out, lse, do, dq=dq)),
                    (dk, lambda: plan.backward(q, k, v, out, lse, do, dk=dk)),
                    (dv, lambda: plan.backward(q, k, v, out, lse, do, dv=dv)),
                    (r, lambda: ck.restore(out=r)), (w, lambda: layers.ckpt_wgrad(do.view(300, 256), ck, out=w)),
                    (w, lambda: layers.ckpt_wgrad(do.view(300, 256), ck, out=w, accumulate=True))):
        kept = saved_by(x)
        call()
        with pytest.raises(RuntimeError, match=MODIFIED):
            kept.backward()
    assert plan.status() == 0


def test_inference_tensors():
    """They have no versions; the calls take them, inside the mode and outside."""
    import torch
    from paper_2609_36692_gb300 import optim
    with torch.inference_mode():
        g = torch.ones(64, device="cuda")
        assert float(optim.clip_grads([g], 4.0, eps=0.0)) == 8.0
    assert float(optim.clip_grads([g], 2.0, eps=0.0)) == 4.0
    assert bool((g == 0.25).all())
