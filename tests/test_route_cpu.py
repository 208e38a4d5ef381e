"""The router module's host side, with a stand-in for the library's call (no GPU needed)."""
import pytest
import torch

R = pytest.importorskip("paper_2609_15037_amd.route")
M = R.M


@pytest.fixture
def router(monkeypatch):
    """A router of 6 experts whose routing takes the two largest logits, on the CPU."""
    monkeypatch.setattr(M, "moara_route_default_config", lambda **kw: M.moara_route_config(**kw))

    def fake(logits, cfg, bias=None, mask=None, counts=None):
        assert bias.dtype == torch.float32 and logits.dtype == torch.float32
        index = (logits + bias).topk(2, dim=1)[1]
        if counts is not None:
            assert counts.dtype == torch.int64
            counts += torch.bincount(index.flatten(), minlength=6)
        return index.int(), logits.softmax(1).gather(1, index)
    monkeypatch.setattr(R, "route", fake)
    torch.manual_seed(0)
    return R.ExpertRouter(8, 6, 2)


@pytest.mark.parametrize("cast", [lambda r: r.bfloat16(), lambda r: r.half(), lambda r: r.to(torch.bfloat16),
                                  lambda r: torch.nn.Sequential(r).to(torch.bfloat16)[0], lambda r: r.bfloat16().float()])
def test_casts_leave_the_bias_in_fp32(router, cast):
    router.bias += torch.arange(6) * 1e-3 + 1.0     # values that bf16 does not hold
    before = router.bias.clone()
    r = cast(router)
    assert r is router and torch.equal(r.bias, before) and r.bias.dtype == torch.float32
    assert "bias" in dict(r.named_buffers()) and torch.equal(r.state_dict()["bias"], before)
    index, weight = r(torch.randn(5, 8, dtype=r.weight.dtype))
    weight.sum().backward()
    assert r.weight.grad.dtype == r.weight.dtype


def test_evaluation_counts_nothing(router):
    x = torch.randn(7, 8)
    router.eval()
    router(x)
    assert not router.load().any()
    router.train()
    router(x)
    with torch.no_grad():
        router(x)
    assert router.load().sum() == 28


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_recomputed_pass_counts_once(router, reentrant):
    from torch.utils.checkpoint import checkpoint
    x = torch.randn(7, 8, requires_grad=True)
    passes = []

    def block(x):
        passes.append(1)
        return router(x)[1] * x[:, :2]
    checkpoint(block, x, use_reentrant=reentrant).sum().backward()
    assert len(passes) == 2 and router.load().sum() == 14
    assert router.weight.grad.any()
    checkpoint(block, x, use_reentrant=reentrant).sum().backward()
    assert len(passes) == 4 and router.load().sum() == 28
