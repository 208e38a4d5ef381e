"""The operators of a training step together: MoARa with the library's AdamW and clipping, the router
module, and the example that trains with all of them."""
import importlib.util
import math
import os
import weakref

import numpy as np
import pytest
import torch

from tests.conftest import ROOT
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs an MI355X GPU")]


class Net(torch.nn.Module):
    def __init__(self, seed):
        super().__init__()
        torch.manual_seed(seed)
        self.embed = torch.nn.Embedding(96, 64)
        self.q_proj = torch.nn.Linear(64, 64, bias=False)
        self.down_proj = torch.nn.Linear(64, 64, bias=False)
        self.norm = torch.nn.LayerNorm(64)
        self.head = torch.nn.Linear(64, 96)

    def forward(self, x):
        h = self.embed(x)
        h = h + self.down_proj(torch.relu(self.q_proj(h)))
        return self.head(self.norm(h))


def _opt(net, **kw):
    from paper_2609_15037_amd.optim import MoARa, moara_targets
    targets, others = moara_targets(net)
    assert len(targets) == 2 and len(others) == 5
    return MoARa(targets, others, lr=1e-2, rank_table=[16] * 10, block_size=32, refresh_interval=5, **kw)


def _backward(net, step, seed=0):
    x = torch.randint(0, 96, (32,), generator=torch.Generator().manual_seed(seed + step)).cuda()
    loss = torch.nn.functional.cross_entropy(net(x).float(), (x + 1) % 96)
    loss.backward()
    return loss


def _same_grads(a, b):
    for p, q in zip(a.parameters(), b.parameters()):
        q.grad = None if p.grad is None else p.grad.detach().clone()


def test_library_adamw_follows_torch_adamw_in_the_optimizer():
    a, b = Net(1).cuda(), Net(1).cuda()
    oa, ob = _opt(a), _opt(b, adamw_bits=32)
    for step in range(6):
        _backward(a, step)
        _same_grads(a, b)
        for o in (oa, ob):
            o.step()
            o.zero_grad()
    for (n, p), q in zip(a.named_parameters(), b.parameters()):   # six updates of about 1e-2, a few roundings each
        torch.testing.assert_close(q, p, rtol=4e-6, atol=4e-6, msg=n)


@pytest.mark.parametrize("bits", [None, 8, 32])
@pytest.mark.parametrize("limit", [0.05, 1e6])
def test_clipping_in_step_equals_clipping_before_it(limit, bits):
    a, b = Net(2).cuda(), Net(2).cuda()
    oa, ob = _opt(a, adamw_bits=bits), _opt(b, adamw_bits=bits, max_grad_norm=limit)
    for step in range(3):
        _backward(a, step)
        _same_grads(a, b)
        norm = torch.nn.utils.clip_grad_norm_(a.parameters(), limit)
        oa.step()
        ob.step()
        assert abs(float(ob.grad_norm) / float(norm) - 1) < 1e-6
        for o in (oa, ob):
            o.zero_grad()
    for (n, p), q in zip(a.named_parameters(), b.parameters()):
        if bits == 8 and "proj" not in n:       # a code may round the other way: a sixteenth of an update
            torch.testing.assert_close(q, p, rtol=0, atol=3e-2 / 16, msg=n)
        else:   # Adam's first steps are near sign(g): an element of G near zero may move either way
            assert float((q - p).abs().max()) <= 6e-2 and float((q - p).norm() / p.norm()) < 2e-3, n


def test_a_norm_that_is_not_finite_skips_the_other_parameters():
    net = Net(3).cuda()
    opt = _opt(net, adamw_bits=8, max_grad_norm=1.0)
    _backward(net, 0)
    opt.step()
    opt.zero_grad()
    before = [p.detach().clone() for p in net.parameters()]
    saved = opt.state_dict()["adamw_own"]["state"]
    _backward(net, 1)
    net.head.bias.grad[3] = math.inf
    opt.step()
    after = opt.state_dict()["adamw_own"]["state"]
    for (n, p), q in zip(net.named_parameters(), before):
        assert torch.isfinite(p).all()
        assert ("proj" in n) or torch.equal(p.detach(), q), n
    assert all(torch.equal(x, y) for s, t in zip(saved, after) for x, y in zip(s, t))


@pytest.mark.parametrize("bits", [8, 32])
def test_weight_decay_is_for_matrices(bits):
    """With gradients of zero and fresh moments the update is the decay alone, one rounding of the product."""
    net = Net(8).cuda()
    opt = _opt(net, adamw_bits=bits, adamw_weight_decay=0.5)
    before = {n: p.detach().clone() for n, p in net.named_parameters()}
    for p in net.parameters():
        p.grad = torch.zeros_like(p)
    opt.step()
    for n, p in net.named_parameters():
        if "proj" not in n:
            want = before[n] * (1 - 1e-2 * 0.5) if p.dim() > 1 else before[n]
            torch.testing.assert_close(p.detach(), want, rtol=2.0 ** -22, atol=0, msg=n)


@pytest.mark.parametrize("bits", [8, 32])
def test_checkpoint_of_the_library_adamw(bits):
    a = Net(4).cuda()
    oa = _opt(a, adamw_bits=bits, adamw_seed=7)
    for step in range(3):
        _backward(a, step)
        if step == 1:
            a.norm.bias.grad = None         # a parameter that misses a step
        oa.step()
        oa.zero_grad()
    b = Net(5).cuda()
    b.load_state_dict(a.state_dict())
    ob = _opt(b, adamw_bits=bits)
    ob.load_state_dict(oa.state_dict())
    assert sorted(oa.state_dict()["adamw_own"]["steps"]) == [2, 3, 3, 3, 3]
    _backward(a, 9)
    _same_grads(a, b)
    oa.step()
    ob.step()
    assert all(torch.equal(p, q) for p, q in zip(a.parameters(), b.parameters()))
    for other in (40 - bits, None):
        with pytest.raises(ValueError):
            _opt(b, adamw_bits=other).load_state_dict(oa.state_dict())
    with pytest.raises(ValueError):
        _opt(b, adamw_bits=bits).load_state_dict(_opt(b).state_dict())


def test_parameters_replaced_and_transposed_between_steps():
    net = Net(6).cuda()
    net.head.weight = torch.nn.Parameter(net.head.weight.detach().t().contiguous().t())
    opt = _opt(net, adamw_bits=32)
    for step in range(2):
        _backward(net, step)
        before = net.head.weight.detach().clone()
        opt.step()
        opt.zero_grad()
        assert not torch.equal(net.head.weight.detach(), before)
        net.embed.weight.data = net.embed.weight.data.clone()     # other storage
    assert opt._own.steps.tolist() == [2] * 5


def test_router_module_gradients_and_load():
    from paper_2609_15037_amd import moara as M
    from paper_2609_15037_amd.route import ExpertRouter
    torch.manual_seed(7)
    r = ExpertRouter(32, 16, 3, score=M.MOARA_SIGMOID, renormalise=1).cuda()
    x = torch.randn(50, 32, device="cuda", requires_grad=True)
    index, weight = r(x)
    c = torch.randn(50, 3, device="cuda")
    (weight * c).sum().backward()
    w64 = r.weight.detach().double().requires_grad_(True)
    x64 = x.detach().double().requires_grad_(True)
    s = torch.sigmoid(x64 @ w64.t()).gather(1, index.long())
    ((s / s.sum(1, keepdim=True)) * c).sum().backward()
    torch.testing.assert_close(r.weight.grad.double(), w64.grad, rtol=1e-4, atol=1e-5)
    torch.testing.assert_close(x.grad.double(), x64.grad, rtol=1e-4, atol=1e-5)
    assert r.load().sum() == 150
    weight2 = r(x)[1]
    weight2.sum().backward()                # a gradient that is an expanded scalar
    assert r.load().sum() == 300
    load = r.load().copy()
    with torch.autocast("cuda", dtype=torch.bfloat16):
        again = r(x)
    assert torch.equal(again[0], index) and torch.equal(again[1], weight)
    load = r.load().copy()
    r.balance(0.25)
    assert not r.load().any()
    assert np.array_equal(r.bias.cpu().numpy(), 0.25 * np.sign(load.mean() - load))


@pytest.mark.parametrize("bits", [8, 32])
def test_example_trains(bits):
    spec = importlib.util.spec_from_file_location("train_moe", os.path.join(ROOT, "examples", "train_moe.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses, share = ex.train(steps=40, bits=bits, say=lambda s: print("[moe]", s, flush=True))
    assert np.isfinite(losses).all()
    assert losses[-1] < 0.8 * losses[0], losses
    assert max(share) <= 0.5        # top-2 of 8 experts: an even share is an eighth, one expert always chosen a half


def _other_strides(p):
    """The same elements, rows first or columns first in memory."""
    p.data = p.data.t().contiguous().t() if p.data.is_contiguous() else p.data.contiguous()


@pytest.mark.parametrize("bits", [8, 32])
def test_moments_stay_with_their_elements_when_strides_change(bits):
    """One copy's head changes its strides twice between steps; both take the same gradients: the same bits."""
    a, b = Net(9).cuda(), Net(9).cuda()
    oa, ob = _opt(a, adamw_bits=bits), _opt(b, adamw_bits=bits)
    for step in range(4):
        _backward(a, step)
        _same_grads(a, b)
        if step in (1, 3):
            _other_strides(b.head.weight)
        for o in (oa, ob):
            o.step()
            o.zero_grad()
        assert b.head.weight.is_contiguous() == (step in (0, 3))
        for (n, p), q in zip(a.named_parameters(), b.parameters()):
            assert torch.equal(p, q), (step, n)


@pytest.mark.parametrize("bits", [8, 32])
def test_checkpoint_of_a_transposed_parameter(bits):
    """Saved with a transposed head, loaded for a contiguous one, and on from there: the same bits. A state that
    does not say its strides is taken to be in the order of the parameters that it is loaded for."""
    a, b = Net(9).cuda(), Net(9).cuda()
    _other_strides(a.head.weight)
    oa, ob = _opt(a, adamw_bits=bits), _opt(b, adamw_bits=bits)
    for step in range(2):
        _backward(a, step)
        oa.step()
        oa.zero_grad()
    b.load_state_dict(a.state_dict())
    ob.load_state_dict(oa.state_dict())
    bare = oa.state_dict()
    del bare["adamw_own"]["form"]
    c = Net(9).cuda()
    _other_strides(c.head.weight)
    oc = _opt(c, adamw_bits=bits)
    c.load_state_dict(a.state_dict())
    oc.load_state_dict(bare)
    for step in (9, 10):
        _backward(a, step)
        for net, opt in ((b, ob), (c, oc)):
            _same_grads(a, net)
            opt.step()
        oa.step()
        oa.zero_grad()
        for (n, p), q, r in zip(a.named_parameters(), b.parameters(), c.parameters()):
            assert torch.equal(p, q) and torch.equal(p, r), n


def test_a_parameter_of_another_shape_than_its_moments_is_refused():
    net = Net(9).cuda()
    opt = _opt(net, adamw_bits=8)
    _backward(net, 0)
    opt.step()
    opt.zero_grad()
    net.head.weight.data = net.head.weight.data.t()
    net.head.weight.grad = torch.zeros_like(net.head.weight)
    with pytest.raises(ValueError):
        opt.step()


@pytest.mark.parametrize("bits", [None, 8, 32])
def test_clipping_keeps_no_gradient(bits):
    """After zero_grad() the gradients' memory is free again: nothing of the step holds one."""
    net = Net(3).cuda()
    opt = _opt(net, adamw_bits=bits, max_grad_norm=1.0)
    for step in range(2):
        _backward(net, step)
        grads = [weakref.ref(p.grad) for p in net.parameters()]
        opt.step()
        opt.zero_grad()
        assert all(g() is None for g in grads)


@pytest.mark.parametrize("clip", [None, 0.05])
def test_training_on_a_side_stream_equals_the_default_one(clip):
    """Forward, backward, step and zero_grad on a side stream, nothing waited for between: the same bits."""
    nets, opts = [Net(11).cuda() for _ in range(2)], []
    opts = [_opt(n, adamw_bits=32, max_grad_norm=clip) for n in nets]
    for step in range(8):
        _backward(nets[0], step)
        opts[0].step()
        opts[0].zero_grad()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for step in range(8):
            _backward(nets[1], step)
            opts[1].step()
            opts[1].zero_grad()
    side.synchronize()
    for (n, p), q in zip(nets[0].named_parameters(), nets[1].parameters()):
        assert torch.equal(p, q), n


@pytest.mark.parametrize("bits", [None, 8, 32])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_what_a_norm_that_is_not_finite_does_to_each_adamw(bad, bits):
    """torch's AdamW takes a step of zero gradients, bit for bit; the library's changes nothing. Nothing turns NaN."""
    net, ref = Net(12).cuda(), Net(12).cuda()
    opt, oref = _opt(net, adamw_bits=bits, max_grad_norm=1.0), _opt(ref, adamw_bits=bits, max_grad_norm=1.0)
    for o, n in ((opt, net), (oref, ref)):
        _backward(n, 0)
        o.step()
        o.zero_grad()
    before = {n: p.detach().clone() for n, p in net.named_parameters()}
    _backward(net, 1)
    net.norm.weight.grad[5] = bad
    opt.step()
    for p in ref.parameters():
        p.grad = torch.zeros_like(p)
    oref.step()
    for (n, p), q in zip(net.named_parameters(), ref.parameters()):
        assert torch.isfinite(p).all()
        if bits is None or "proj" in n:
            assert torch.equal(p, q), n
        else:
            assert torch.equal(p.detach(), before[n]), n
        if bits is None and "proj" not in n:
            assert not torch.equal(p.detach(), before[n]), n        # it moves by its momentum


@pytest.mark.parametrize("bits", [None, 8, 32])
def test_gradients_of_any_order_are_scaled_in_place(bits):
    """Transposed gradients stay the caller's tensors, scaled where the class says so; expanded ones, whose elements
    share memory, are replaced. The steps equal those of contiguous gradients."""
    a, b = Net(6).cuda(), Net(6).cuda()
    oa, ob = _opt(a, adamw_bits=bits, max_grad_norm=0.05), _opt(b, adamw_bits=bits, max_grad_norm=0.05)
    g = torch.Generator(device="cuda").manual_seed(1)
    for n, p in a.named_parameters():
        if n == "norm.bias":
            p.grad = torch.full((1,), 0.5, device="cuda").expand(p.shape)
        else:
            p.grad = torch.randn(p.shape[::-1], generator=g, device="cuda").t() if p.dim() == 2 else \
                torch.randn(p.shape, generator=g, device="cuda")
    for p, q in zip(a.parameters(), b.parameters()):
        q.grad = p.grad.contiguous().clone()
    held = {n: p.grad for n, p in a.named_parameters()}
    before = {n: x.clone() for n, x in held.items()}
    oa.step()
    ob.step()
    for (n, p), q in zip(a.named_parameters(), b.parameters()):
        torch.testing.assert_close(p, q, rtol=1e-5, atol=1e-6, msg=n)      # the norm's order of summation differs
        torch.testing.assert_close(p.grad, q.grad, rtol=1e-6, atol=0, msg=n)
        if n == "norm.bias":
            assert torch.equal(held[n], before[n])
            continue
        assert p.grad is held[n], n
        scaled = bits is None or "proj" in n
        assert torch.equal(p.grad, before[n]) != scaled, n


def test_router_in_a_bf16_model():
    """Cast with its model, the router takes bf16 rows, has bf16 gradients, and its bias moves in fp32."""
    from paper_2609_15037_amd.route import ExpertRouter
    torch.manual_seed(13)
    r = torch.nn.Sequential(ExpertRouter(32, 16, 3, renormalise=1)).cuda().bfloat16()[0]
    same = ExpertRouter(32, 16, 3, renormalise=1).cuda()
    same.load_state_dict({"weight": r.weight.float(), "bias": r.bias, "counts": r.counts})
    for step in range(3):
        x = torch.randn(50, 32, device="cuda").bfloat16()
        c = torch.randn(50, 3, device="cuda")
        out, want = r(x), same(x.float())
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        (out[1] * c).sum().backward()
        (want[1] * c).sum().backward()
        assert r.weight.grad.dtype == torch.bfloat16 and torch.equal(r.weight.grad, same.weight.grad.bfloat16())
        r.weight.grad = same.weight.grad = None
        r.balance(1e-3)
        same.balance(1e-3)
        assert r.bias.dtype == torch.float32 and torch.equal(r.bias, same.bias) and r.bias.any()


def _example():
    spec = importlib.util.spec_from_file_location("train_moe", os.path.join(ROOT, "examples", "train_moe.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


@pytest.mark.parametrize("reentrant", [None, False, True])
def test_counts_are_those_of_training(reentrant):
    """A layer of the example: evaluated, trained, and with its activations recomputed; output and gradients alike."""
    from torch.utils.checkpoint import checkpoint
    torch.manual_seed(14)
    layer = _example().Layer(32, 2, 48, 8, 2).cuda()
    x = torch.randn(2, 9, 32, device="cuda", requires_grad=True)
    layer.eval()
    want = layer(x)
    want.square().sum().backward()
    grads = [p.grad for p in layer.parameters()]
    assert not layer.router.load().any()
    layer.train()
    layer.zero_grad()
    out = layer(x) if reentrant is None else checkpoint(layer, x, use_reentrant=reentrant)
    assert torch.equal(out, want)
    out.square().sum().backward()
    assert layer.router.load().sum() == 36
    for p, g in zip(layer.parameters(), grads):
        assert (p.grad is None) == (g is None)
        if g is not None:
            torch.testing.assert_close(p.grad, g, rtol=1e-4, atol=1e-5)     # attention's sums in any order


def test_balancing_spreads_the_example_tokens():
    """The bias moves by 0.4 in 40 steps, between scores from 0 to 1. Towards an even load no layer's busiest expert has
    over twice an even share (an eighth); the other way those above the mean stay there and gain, fewer and fewer."""
    even = _example().train(steps=40, rate=1e-2, say=lambda s: print("[moe]", s, flush=True))[1]
    uneven = _example().train(steps=40, rate=-1e-2, say=lambda s: print("[moe]", s, flush=True))[1]
    assert max(even) <= 0.25, even
    assert min(uneven) > max(even), (even, uneven)
