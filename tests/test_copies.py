"""Copies of what holds memory of the library's: a module that has a plan is copied
(``copy.deepcopy``, ``pickle``), and both are used and released."""
import os
import subprocess
import sys

import pytest

from test_layers_cpu import C  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

COPIES = """
import copy, pickle, torch
from paper_2609_36692_gb300 import layers

class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.rotary = layers.QKNormRotary(4, 2, 64, rotary_dim=32, base=500.0, interleaved=True, eps=1e-5)
model = Model()
for other in (copy.deepcopy(model), pickle.loads(pickle.dumps(model))):
    a, b = model.rotary, other.rotary
    assert a.plan != b.plan and a._made == b._made and len(b._made["frequencies"]) == 16
    assert (b.n_heads, b.n_kv_heads, b.head_dim, b.rotary_dim, b.dtype) == (4, 2, 64, 32, torch.bfloat16)
    c = copy.copy(b)
    b.close()
    assert c.plan and copy.deepcopy(b).plan is None
    del c
del model, other, a, b
print("released")
"""


def test_plans(C):
    """In a process of its own: a plan released twice ends it."""
    r = subprocess.run([sys.executable, "-c", COPIES], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "released", r.stderr


@pytest.mark.gpu
def test_attention_plans_and_checkpoints():
    import copy
    import pickle
    import torch
    from paper_2609_36692_gb300 import layers
    from test_attention_gpu import make, plan_for
    q, k, v, _ = (x.contiguous() for x in make(3, 500, 4, 2, 64, "bf16"))
    plan = plan_for(4, 2, 64, 500, [300, 190], "bf16", window=100, sinks=3)
    want = plan.forward(q, k, v)
    others = [copy.deepcopy(plan), pickle.loads(pickle.dumps(plan))]
    plan.close()
    for p in others:
        assert p.lengths == (300, 190) and p.plan
        assert all(torch.equal(a, b) for a, b in zip(p.forward(q, k, v), want))
        assert p.status() == 0
    assert copy.deepcopy(plan).plan is None
    ck = layers.ckpt_pack(q.view(500, 256))
    want = ck.restore()
    others = [copy.deepcopy(ck), pickle.loads(pickle.dumps(ck))]
    assert all(x.codes_ptr != ck.codes_ptr for x in others)
    ck.data.zero_()
    assert all(torch.equal(x.restore(), want) for x in others)
