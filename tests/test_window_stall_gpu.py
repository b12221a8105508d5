"""A wait of the backward pass that gives up: the merged launch skips its second
walk, ends, and is reported; the context and the plan stay usable.  One CTA loads
no queries (test_stall); its waits are bounded by two seconds."""
import pytest

from test_attention_gpu import make, plan_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [(4, 2, 64), (3, 1, 128)], ids=str)
@pytest.mark.parametrize("window, sinks", [(0, 0), (100, 4), (130, 200), (600, 0)])
def test_backward_gives_up(window, sinks, layout):
    import torch
    from paper_2609_36692_gb300 import normpre as C
    h, hk, d = layout
    lengths, room = [1500, 333], 64
    n = sum(lengths) + 3
    q, k, v, do = make(6, n, h, hk, d, "bf16")
    plan = plan_for(h, hk, d, n, lengths, "bf16", window=window, sinks=sinks)
    out, lse = plan.forward(q, k, v)
    want = plan.backward(q, k, v, out, lse, do)
    plan.close()
    plan.plan = C.normpre_attn_init_window(C.normpre_attn_config(h, hk, d, 2, n, C.NORMPRE_BF16, 0.0, 2), window, sinks)
    plan.set_lengths(lengths)
    wide = [torch.full((n + 2 * room, x, d), 7.0, dtype=torch.bfloat16, device="cuda") for x in (h, hk, hk)]
    plan.backward(q, k, v, out, lse, do, *(x[room:room + n] for x in wide))
    torch.cuda.synchronize()
    for f in (lambda: plan.forward(q, k, v), lambda: plan.backward(q, k, v, out, lse, do)):
        with pytest.raises(C.NormPreError, match="gave up") as e:
            f()
        assert e.value.status == C.NORMPRE_ERR_TIMEOUT
    assert plan.status(raise_on_error=False) == C.NORMPRE_ERR_TIMEOUT
    for x in wide:
        assert bool((x[:room] == 7.0).all()) and bool((x[room + n:] == 7.0).all())
    # the plan's forward pass, and another plan's backward pass
    again = plan.forward(q, k, v)
    assert plan.status() == C.NORMPRE_OK
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    other = plan_for(h, hk, d, n, lengths, "bf16", window=window, sinks=sinks)
    for a, b in zip(other.backward(q, k, v, out, lse, do), want):
        assert torch.equal(a, b)
    assert other.status() == C.NORMPRE_OK


def test_other_values_are_refused():
    from paper_2609_36692_gb300 import normpre as C
    for bad in (-1, 3):
        with pytest.raises(C.NormPreError) as e:
            C.normpre_attn_init(C.normpre_attn_config(4, 2, 64, 2, 100, C.NORMPRE_BF16, 0.0, bad))
        assert e.value.status == C.NORMPRE_ERR_ARG
