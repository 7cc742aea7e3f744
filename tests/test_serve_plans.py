"""Plans of the serving operators as Python objects: copies, threads, and what autograd is told.  Nothing here needs a GPU;
where a call would reach the device, a stand-in takes its place."""
import copy
import gc
import pickle
import threading
import types

import pytest
import torch

from paper_2002_12798_b200 import binding as B
from paper_2002_12798_b200 import ops


# ----------------------------------------------------------------------------------------------------------------------
# copies
# ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))])
def test_a_copied_rope_plan_owns_its_own(how, monkeypatch):
    freed = []
    real = ops._lib.amap_rope_destroy
    monkeypatch.setattr(ops, "_lib", types.SimpleNamespace(amap_rope_plan=ops._lib.amap_rope_plan, amap_serve_error=ops._lib.amap_serve_error,
                                                           amap_rope_destroy=lambda h: freed.append(h)))
    plan = ops.RopePlan(64, 32, base=500.0, sections=[4, 12], pairs="adjacent", scale=0.5)
    plan.name = "what a user hangs on it"
    other = how(plan)
    handles = {plan._h, other._h}
    assert len(handles) == 2 and type(other) is ops.RopePlan
    assert (other.head_dim, other.rotary_dim, other.n_axes, other.name) == (64, 32, 2, plan.name)
    module = torch.nn.Module()
    module.rope = plan
    third = copy.deepcopy(module)
    handles.add(third.rope._h)
    assert len(handles) == 3
    del plan, other, third, module
    gc.collect()
    assert sorted(freed) == sorted(handles)  # each once
    for h in freed:
        real(h)


def test_a_rope_plan_that_was_refused_is_freed_quietly():
    with pytest.raises(B.AmapError):
        ops.RopePlan(64, scale=float("inf"))
    gc.collect()
