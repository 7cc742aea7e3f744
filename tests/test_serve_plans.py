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


def attend_plan(monkeypatch):
    """An AttendPlan without its device memory, and a list of what its calls do in which order."""
    done = []

    def make(plan):
        plan._lock, plan._raw, plan._at = threading.Lock(), 1, object()

    monkeypatch.setattr(ops.AttendPlan, "_make", make, raising=False)
    plan = object.__new__(ops.AttendPlan)
    plan.max_requests, plan.q_heads, plan.kv_heads, plan.head_dim = 4, 8, 2, 64
    plan.scale, plan.window, plan.softcap, plan.device, plan._device = 0.125, 0, 0.0, torch.device("cuda", 0), 0
    make(plan)
    return plan, done


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))])
def test_a_copied_attend_plan_has_a_workspace_of_its_own(how, monkeypatch):
    plan, _ = attend_plan(monkeypatch)
    plan.window = 77
    other = how(plan)
    assert other._at is not plan._at and other._lock is not plan._lock
    assert (other.max_requests, other.q_heads, other.kv_heads, other.head_dim, other.scale, other.window, other.device) == (4, 8, 2, 64, 0.125, 77, plan.device)


def test_calls_from_two_threads_keep_their_order(monkeypatch):
    """Between a call's taking its place behind the plan's last stream and its launch, no other call takes one."""
    plan, done = attend_plan(monkeypatch)
    streams = {}
    inside, go_on = threading.Event(), threading.Event()

    def order(self):
        me = streams[threading.get_ident()]
        done.append(("waits for", self._raw, me))
        self._raw = me
        if me == 2:
            inside.set()
            go_on.wait(2)

    monkeypatch.setattr(ops.AttendPlan, "_order", order)
    monkeypatch.setattr(ops, "_raw_stream", lambda device: streams[threading.get_ident()])
    monkeypatch.setattr(ops, "_entry", types.SimpleNamespace(attend=lambda *a: done.append(("launched on", streams[threading.get_ident()]))))
    cache = types.SimpleNamespace(_at=0, _maps_at=0, _device=0)

    def call(stream):
        streams[threading.get_ident()] = stream
        plan.attend(None, cache, None, None)

    first, second = threading.Thread(target=call, args=(2,)), threading.Thread(target=call, args=(3,))
    first.start()
    assert inside.wait(5)
    second.start()
    second.join(0.3)
    go_on.set()
    first.join(5)
    second.join(5)
    assert done == [("waits for", 1, 2), ("launched on", 2), ("waits for", 2, 3), ("launched on", 3)]


# ----------------------------------------------------------------------------------------------------------------------
# autograd, with the turn in plain torch in the entry's place
# ----------------------------------------------------------------------------------------------------------------------
@pytest.fixture
def plain_entry(monkeypatch):
    calls = []

    def rotate(h, dim, axes, xs, positions, inverse, outs):
        calls.append(("rotate", bool(inverse)))
        with torch.no_grad():
            c, s = positions.double().cos()[:, None, None], positions.double().sin()[:, None, None] * (-1 if inverse else 1)
            got = [torch.cat([x[..., : dim // 2] * c - x[..., dim // 2 :] * s, x[..., dim // 2 :] * c + x[..., : dim // 2] * s], -1) for x in xs]
            if outs is not None:
                for o, g in zip(outs, got):
                    o.copy_(g)
            return got if outs is None else list(outs)

    def append(h, dim, axes, q, k, v, positions, slots, at, device, out):
        calls.append(("append",))
        if ops._tracked((q, k, v)):
            return NotImplemented
        return q.detach() * 2 if out is None else out

    def attend(*a):
        calls.append(("attend",))
        q, lse = a[4], a[11]
        if ops._tracked((q,)):
            return NotImplemented
        got = q.detach() * 3
        return (got, got.sum(-1)) if lse else got

    monkeypatch.setattr(ops, "_entry", types.SimpleNamespace(rotate=rotate, append=append, attend=attend))
    return calls


def doubles(*shape):
    return torch.randn(*shape, dtype=torch.float64)


def test_rotate_has_derivatives_of_every_order(plain_entry):
    torch.manual_seed(0)
    plan, pos = ops.RopePlan(4), torch.tensor([0.3, 1.0, 2.0])
    q, k = doubles(3, 2, 4).requires_grad_(), doubles(3, 1, 4).requires_grad_()
    assert torch.autograd.gradcheck(lambda q, k: tuple(plan.rotate([q, k], pos)), (q, k))
    assert torch.autograd.gradgradcheck(lambda q, k: tuple(plan.rotate([q, k], pos)), (q, k))
    # a penalty on the gradient: its own gradient goes through the gradient's turn
    weight = doubles(3, 2, 4).requires_grad_()
    (g,) = torch.autograd.grad((plan.rotate([q], pos)[0] * weight).sum(), [q], create_graph=True)
    assert g.requires_grad
    (gw,) = torch.autograd.grad((g * g).sum(), [weight])
    assert torch.allclose(gw, 2 * weight)  # a turn keeps lengths


def test_rotate_carries_tangents(plain_entry):
    from torch.autograd import forward_ad

    plan, pos = ops.RopePlan(4), torch.tensor([0.3, 1.0, 2.0])
    q, k, t = doubles(3, 2, 4), doubles(3, 1, 4), doubles(3, 2, 4)
    with torch.no_grad(), forward_ad.dual_level():
        a, b = plan.rotate([forward_ad.make_dual(q, t), k], pos, inverse=True)
        value, tangent = forward_ad.unpack_dual(a)
        other = forward_ad.unpack_dual(b).tangent
        assert torch.equal(value, plan.rotate([q], pos, inverse=True)[0])
        assert torch.equal(tangent, plan.rotate([t], pos, inverse=True)[0])
        assert other is None or not other.any()
        with pytest.raises(ValueError, match="outs"):
            plan.rotate([forward_ad.make_dual(q, t)], pos, outs=[torch.empty_like(q)])


CACHE = types.SimpleNamespace(_at=0, _maps_at=0, _device=0)


def test_append_and_attend_say_that_they_have_no_derivative(plain_entry, monkeypatch):
    """Their results are what they were; asking for the gradient raises instead of leaving it out."""
    from torch.autograd import forward_ad

    rope, (attention, _) = ops.RopePlan(4), attend_plan(monkeypatch)
    monkeypatch.setattr(ops, "_raw_stream", lambda device: attention._raw)
    q, k = doubles(3, 2, 4), doubles(3, 1, 4)
    for call in (lambda q, k, **o: rope.append(q, k, k, None, None, CACHE, **o), lambda q, k, **o: attention.attend(q, CACHE, None, None, **o)):
        plain = call(q, k)
        assert not plain.requires_grad
        asked = call(q.clone().requires_grad_(), k)
        assert torch.equal(asked.detach(), plain)
        with pytest.raises(RuntimeError, match="not differentiable"):
            asked.sum().backward()
        with pytest.raises(ValueError, match="out"):
            call(q.clone().requires_grad_(), k, out=torch.empty_like(q))
        with torch.no_grad():
            assert not call(q.clone().requires_grad_(), k).requires_grad
            with forward_ad.dual_level(), pytest.raises(RuntimeError, match="not differentiable"):
                call(forward_ad.make_dual(q, q), k)
    with pytest.raises(RuntimeError, match="not differentiable"):  # k and v, too
        rope.append(q, k.clone().requires_grad_(), k, None, None, CACHE).sum().backward()
    out, lse = attention.attend(q.clone().requires_grad_(), CACHE, None, None, return_lse=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        lse.sum().backward()


@pytest.mark.gpu
def test_rotate_has_derivatives_on_the_gpu():
    from torch.autograd import forward_ad

    torch.manual_seed(1)
    plan, pos = ops.RopePlan(64, 32), torch.arange(7, dtype=torch.int32, device="cuda")
    q, k, w, t = (torch.randn(7, n, 64, device="cuda") for n in (4, 1, 4, 4))
    q.requires_grad_(), w.requires_grad_()
    (g,) = torch.autograd.grad((plan.rotate([q, k], pos)[0] * w).sum(), [q], create_graph=True)
    (gw,) = torch.autograd.grad((g * g).sum(), [w])
    assert torch.allclose(gw, 2 * w, rtol=1e-5, atol=1e-5)
    with torch.no_grad(), forward_ad.dual_level():
        a, b = plan.rotate([forward_ad.make_dual(q.detach(), t), k], pos)
        assert torch.equal(forward_ad.unpack_dual(a).tangent, plan.rotate([t], pos)[0])
        assert not torch.count_nonzero(forward_ad.unpack_dual(b).tangent)


@pytest.mark.gpu
def test_append_and_attend_say_so_on_the_gpu():
    k, v = (torch.randn(2, 16, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache, rope, attention = ops.PagedCache(k, v), ops.RopePlan(64), ops.AttendPlan(1, 4, 2, 64)
    q, kk = torch.randn(1, 4, 64, device="cuda", dtype=torch.bfloat16), torch.randn(1, 2, 64, device="cuda", dtype=torch.bfloat16)
    one = dict(dtype=torch.int32, device="cuda")
    pos, slot, table, n = torch.tensor([3], **one), torch.tensor([-1], **one), torch.tensor([[1, 0]], **one), torch.tensor([20], **one)
    for call in (lambda q: rope.append(q, kk, kk, pos, slot, cache), lambda q: attention.attend(q, cache, table, n),
                 lambda q: attention.attend(q, cache, table, n, return_lse=True)[1]):
        plain, asked = call(q), call(q.clone().requires_grad_())
        assert torch.equal(plain, asked.detach()) and not plain.requires_grad
        with pytest.raises(RuntimeError, match="not differentiable"):
            asked.float().sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("stream", [False, True])
def test_reset_makes_a_failed_plan_fit_for_use(stream):
    """A kernel that gave up is played by the host: the mark set, counters and parts left as they may be."""
    torch.manual_seed(2)
    n = 5000
    k, v = (torch.randn(n // 16 + 1, 16, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache, attention = ops.PagedCache(k, v), ops.AttendPlan(3, 8, 2, 64)
    q = torch.randn(3, 8, 64, device="cuda", dtype=torch.bfloat16)
    table = torch.arange(n // 16 + 1, dtype=torch.int32, device="cuda").repeat(3, 1)
    lens = torch.tensor([n, 100, n - 7], dtype=torch.int32, device="cuda")
    want = attention.attend(q, cache, table, lens)
    assert not attention.failed()
    attention._workspace.fill_(1)
    assert attention.failed()
    side = torch.cuda.Stream() if stream else torch.cuda.current_stream()
    with torch.cuda.stream(side):
        attention.reset()
    got = attention.attend(q, cache, table, lens)
    assert not attention.failed() and torch.equal(got, want)
