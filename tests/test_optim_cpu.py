"""Host-side parts of the torch.optim integration (no GPU needed)."""
import contextlib
import math

import pytest
import torch

from paper_2609_15037_amd import moara as M
from paper_2609_15037_amd.optim import moara_targets, warmup_cosine


def test_warmup_cosine_schedule_shape():
    # Appendix D: 10 % linear warmup, cosine decay to 0.1 of the peak
    f = warmup_cosine(100)
    assert f(0) == pytest.approx(0.1) and f(9) == pytest.approx(1.0)
    assert f(10) == pytest.approx(1.0)
    assert f(55) == pytest.approx(0.1 + 0.9 * 0.5 * (1 + math.cos(math.pi * 0.5)))
    assert f(100) == pytest.approx(0.1) and f(1000) == pytest.approx(0.1)
    vals = [f(s) for s in range(10, 101)]
    assert all(a >= b for a, b in zip(vals, vals[1:]))


def test_targets_are_the_projection_weights():
    class Attn(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.q_proj = torch.nn.Linear(8, 8, bias=False)
            self.k_proj = torch.nn.Linear(8, 4, bias=False)
            self.o_proj = torch.nn.Linear(8, 8, bias=True)
            self.norm = torch.nn.LayerNorm(8)

    class Net(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.embed = torch.nn.Embedding(10, 8)
            self.attn = Attn()
            self.down_proj = torch.nn.Linear(16, 8, bias=False)

    net = Net()
    t, o = moara_targets(net)
    assert [(p.shape, m) for p, m in t] == [(net.attn.q_proj.weight.shape, M.MOARA_Q),
                                             (net.attn.k_proj.weight.shape, M.MOARA_K),
                                             (net.attn.o_proj.weight.shape, M.MOARA_O),
                                             (net.down_proj.weight.shape, M.MOARA_DOWN)]
    assert len(o) == 4   # embedding, o_proj bias, norm weight and bias


def test_expert_projections_take_the_expert_types():
    class Expert(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.gate_proj = torch.nn.Linear(8, 12, bias=False)
            self.down_proj = torch.nn.Linear(12, 8, bias=False)

    class Moe(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.experts = torch.nn.ModuleList([Expert(), Expert()])
            self.up_proj = torch.nn.Linear(8, 12, bias=False)   # a dense MLP projection

    t, _ = moara_targets(Moe())
    assert [m for _, m in t] == [M.MOARA_EXP_GATE, M.MOARA_EXP_DOWN, M.MOARA_EXP_GATE, M.MOARA_EXP_DOWN,
                                 M.MOARA_UP]


def _own_adamw(shapes, bits=32):
    from paper_2609_15037_amd.optim import _AdamW
    params = [torch.nn.Parameter(torch.zeros(s)) for s in shapes]
    return _AdamW(params, M.moara_adamw_config(beta1=0.9, beta2=0.999, eps=1e-6, bits=bits), 0.0, 0)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("mine,theirs", [([(7,), (33,)], [(7,), (1,)]), ([(7,), (4, 6)], [(7,), (6, 4)]), ([(3,)], [(4,)])])
def test_adamw_state_of_other_shapes_is_refused_whole(mine, theirs, bits):
    """Moments of one element would fill a longer parameter's, those of a transposed matrix lie elsewhere."""
    a, b = _own_adamw(mine, bits), _own_adamw(theirs, bits)
    sd = b.state_dict()
    for s in sd["state"]:
        for t in s:
            if t is not None:
                t.fill_(5)
    sd["steps"] = [9] * len(theirs)
    before = a.state_dict()
    for drop in ((), ("form",)):
        bad = {k: v for k, v in sd.items() if k not in drop}
        if drop and mine[-1] == (4, 6):     # as many elements: without the shapes there is nothing to compare
            continue
        with pytest.raises(ValueError):
            a.load_state_dict(bad)
        after = a.state_dict()
        assert after["steps"] == before["steps"] and after["form"] == before["form"]
        assert all(x is None or torch.equal(x, y) for s, t in zip(after["state"], before["state"]) for x, y in zip(s, t))
    good = a.state_dict()
    with pytest.raises(ValueError):
        a.load_state_dict({**good, "steps": [3]} if len(mine) > 1 else {**good, "steps": [3, 3]})
    good["steps"] = [4] * len(mine)
    a.load_state_dict(good)
    assert a.steps.tolist() == [4] * len(mine)


class _Stream:
    """A stream that writes down who waits for whom."""

    def __init__(self, name, handle, log, look):
        self.name, self.cuda_stream, self.log, self.look = name, handle, log, look

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name, self.look()))


@pytest.mark.parametrize("side", [True, False])
@pytest.mark.parametrize("clip", [None, 1.0])
def test_step_on_a_side_stream_waits_both_ways(side, clip, monkeypatch):
    """The library's step runs on the default stream. It waits for the current one, after the gradients' copies, and
    the current one for it; on the default stream nobody waits."""
    from paper_2609_15037_amd import optim
    log = []
    w = torch.nn.Parameter(torch.zeros(4, 6, dtype=torch.bfloat16))
    opt = None
    copied = lambda: opt._g32[0] is not None and torch.equal(opt._g32[0], w.grad.float())
    default = _Stream("default", 0, log, copied)
    here = _Stream("here", 77, log, copied) if side else default
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: here)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: default)
    monkeypatch.setattr(optim.MoARa, "_device", lambda self: contextlib.nullcontext())
    monkeypatch.setattr(optim.MoARa, "_clip", lambda self: None)
    monkeypatch.setattr(M, "moara_default_config", lambda **kw: None)
    monkeypatch.setattr(M, "moara_create_state", lambda cfg, descs: "state")
    monkeypatch.setattr(M, "moara_step_mixed", lambda st, *a, **kw: log.append("step"))
    opt = optim.MoARa([(w, M.MOARA_Q)], [], max_grad_norm=clip)
    w.grad = torch.full_like(w, 3.0)
    opt.step()
    assert log == ([("default", "waits for", "here", True), "step", ("here", "waits for", "default", True)] if side else ["step"])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_library_adamw_refuses_other_types_at_the_start(dtype, monkeypatch):
    from paper_2609_15037_amd import optim
    monkeypatch.setattr(M, "moara_default_config", lambda **kw: None)
    monkeypatch.setattr(M, "moara_adamw_default_config", lambda **kw: M.moara_adamw_config(**kw))
    w, p = torch.nn.Parameter(torch.zeros(4, 6)), torch.nn.Parameter(torch.zeros(5, dtype=dtype))
    for bits in (8, 32):
        with pytest.raises(ValueError):
            optim.MoARa([(w, M.MOARA_Q)], [p], adamw_bits=bits)
        optim.MoARa([(w, M.MOARA_Q)], [torch.nn.Parameter(p.detach().bfloat16())], adamw_bits=bits)
    optim.MoARa([(w, M.MOARA_Q)], [p])


def test_a_refused_state_leaves_the_rates(monkeypatch):
    from paper_2609_15037_amd import optim
    monkeypatch.setattr(M, "moara_default_config", lambda **kw: None)
    monkeypatch.setattr(M, "moara_adamw_default_config", lambda **kw: M.moara_adamw_config(**kw))
    make = lambda n, lr: optim.MoARa([(torch.nn.Parameter(torch.zeros(4, 6)), M.MOARA_Q)], [torch.nn.Parameter(torch.zeros(n))],
                                     lr=lr, adamw_bits=8)
    a, b = make(5, 1e-2), make(7, 3e-3)
    with pytest.raises(ValueError):
        a.load_state_dict(b.state_dict())
    assert [g["lr"] for g in a.param_groups] == [1e-2] * 2
    make(7, 1e-2).load_state_dict(b.state_dict())
