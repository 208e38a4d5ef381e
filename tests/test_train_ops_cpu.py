"""The operators beside the projected update without a GPU: refusals of the C ABI before anything is
enqueued, and the oracle against hand-written values."""
import ctypes
import math
import os

import numpy as np
import pytest

from oracle import train_oracle as O

M = pytest.importorskip("paper_2609_15037_amd.moara")

P = 1 << 20         # an address that no refused call may touch


@pytest.fixture(autouse=True)
def _built():
    if not os.path.exists(M.LIB_PATH):
        pytest.skip("libmoara.so not built")


def _grads(**kw):
    return (M.moara_grad_tensor * 1)(M.moara_grad_tensor(**{**dict(grad=P, count=8, dtype=M.MOARA_F32), **kw}))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), M.MOARA_E_ARG), (dict(count=-1), M.MOARA_E_SHAPE), (dict(count=(1 << 40) + 1), M.MOARA_E_SHAPE),
    (dict(count=(1 << 33) + 1), M.MOARA_E_SHAPE),
    (dict(grad=P + 2), M.MOARA_E_ARG), (dict(grad=P + 1, dtype=M.MOARA_BF16), M.MOARA_E_ARG)])
def test_gradient_lists_are_refused(kw, status):
    L, t = M.lib(), _grads(**kw)
    assert L.moara_grad_norm(ctypes.addressof(t), 1, 1.0, P, P, None) == status
    assert L.moara_grad_scale(ctypes.addressof(t), 1, P, None) == status


@pytest.mark.parametrize("args", [(None, 1, 1.0, P, P), (None, -1, 1.0, P, P), (None, 0, 0.0, P, P), (None, 0, math.nan, P, P),
                                  (None, 0, 1.0, None, P), (None, 0, 1.0, P, None), (None, 0, 1.0, P + 1, P),
                                  (None, 0, 1.0, P, P + 4)])
def test_norm_arguments_are_refused(args):
    assert M.lib().moara_grad_norm(*args, None) == M.MOARA_E_ARG
    assert M.moara_last_error()


def test_scale_without_a_coefficient_is_refused():
    t = _grads()
    assert M.lib().moara_grad_scale(ctypes.addressof(t), 1, None, None) == M.MOARA_E_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(param_dtype=2), M.MOARA_E_ARG), (dict(grad_dtype=-1), M.MOARA_E_ARG), (dict(count=-5), M.MOARA_E_SHAPE),
    (dict(count=(1 << 33) + 1), M.MOARA_E_SHAPE),
    (dict(param=None), M.MOARA_E_ARG), (dict(exp_avg=None), M.MOARA_E_ARG), (dict(exp_avg_sq=None), M.MOARA_E_ARG),
    (dict(scales=None), M.MOARA_E_ARG), (dict(param=P + 2), M.MOARA_E_ARG), (dict(grad=P + 1), M.MOARA_E_ARG),
    (dict(step=0), M.MOARA_E_ARG), (dict(lr=math.nan), M.MOARA_E_ARG), (dict(weight_decay=math.inf), M.MOARA_E_ARG)])
def test_adamw_tensors_are_refused(kw, status):
    t = (M.moara_adamw_tensor * 1)(M.moara_adamw_tensor(**{**dict(
        param=P, grad=P, exp_avg=P, exp_avg_sq=P, scales=P, count=8, step=1, lr=0.1, weight_decay=0.0,
        param_dtype=M.MOARA_F32, grad_dtype=M.MOARA_F32), **kw}))
    cfg = M.moara_adamw_default_config(bits=8)
    assert M.lib().moara_adamw_step(ctypes.byref(cfg), ctypes.addressof(t), 1, None, 0, None) == status


def test_adamw_configurations_are_refused():
    for kw in (dict(bits=16), dict(beta1=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=math.inf)):
        cfg = M.moara_adamw_default_config(**kw)
        assert M.lib().moara_adamw_step(ctypes.byref(cfg), None, 0, None, 0, None) == M.MOARA_E_ARG, kw
    assert M.lib().moara_adamw_step(None, None, 0, None, 0, None) == M.MOARA_E_ARG
    cfg = M.moara_adamw_default_config()
    assert M.lib().moara_adamw_step(ctypes.byref(cfg), None, 1, None, 0, None) == M.MOARA_E_ARG
    assert M.lib().moara_adamw_step(ctypes.byref(cfg), None, 0, P + 2, 0, None) == M.MOARA_E_ARG
    assert M.lib().moara_adamw_step(ctypes.byref(cfg), None, 0, None, 0, None) == M.MOARA_OK     # nothing to do


@pytest.mark.parametrize("kw,status", [
    (dict(experts=0), M.MOARA_E_ARG), (dict(top_k=0), M.MOARA_E_ARG), (dict(top_k=65), M.MOARA_E_ARG),
    (dict(groups=5), M.MOARA_E_ARG), (dict(groups=4, top_groups=5), M.MOARA_E_ARG), (dict(groups=0), M.MOARA_E_ARG),
    (dict(groups=32, top_groups=2), M.MOARA_E_ARG), (dict(group_best=3), M.MOARA_E_ARG), (dict(score=2), M.MOARA_E_ARG),
    (dict(logits_dtype=3), M.MOARA_E_ARG), (dict(scale=math.inf), M.MOARA_E_ARG),
    (dict(experts=1025), M.MOARA_E_UNSUPPORTED), (dict(experts=128, top_k=65), M.MOARA_E_UNSUPPORTED),
    (dict(experts=256, groups=128, top_groups=128), M.MOARA_E_UNSUPPORTED)])
def test_routing_configurations_are_refused(kw, status):
    cfg = M.moara_route_default_config(**kw)
    E = cfg.experts
    assert M.lib().moara_route(ctypes.byref(cfg), P, 4, E, None, None, P, P, None, None) == status
    assert M.lib().moara_route_backward(ctypes.byref(cfg), P, 4, E, P, P, P, None) == status


def test_routing_arguments_are_refused():
    cfg = M.moara_route_default_config()
    c = ctypes.byref(cfg)
    f, b = M.lib().moara_route, M.lib().moara_route_backward
    for args, status in (((None, P, 4, 64, None, None, P, P, None), M.MOARA_E_ARG), ((c, None, 4, 64, None, None, P, P, None), M.MOARA_E_ARG),
                         ((c, P, -1, 64, None, None, P, P, None), M.MOARA_E_SHAPE), ((c, P, 4, 63, None, None, P, P, None), M.MOARA_E_SHAPE),
                         ((c, P + 2, 4, 64, None, None, P, P, None), M.MOARA_E_ARG), ((c, P, 4, 64, None, None, None, P, None), M.MOARA_E_ARG),
                         ((c, P, 4, 64, None, None, P, None, None), M.MOARA_E_ARG), ((c, P, 4, 64, P + 1, None, P, P, None), M.MOARA_E_ARG),
                         ((c, P, 4, 64, None, None, P, P, P + 4), M.MOARA_E_ARG)):
        assert f(*args, None) == status, args
    for args in ((c, P, 4, 64, None, P, P), (c, P, 4, 64, P, None, P), (c, P, 4, 64, P, P, None), (c, P, 4, 64, P, P, P + 1)):
        assert b(*args, None) == M.MOARA_E_ARG, args
    for args in ((0, P, P, 0.1), (1025, P, P, 0.1), (64, None, P, 0.1), (64, P, None, 0.1), (64, P + 4, P, 0.1), (64, P, P, math.nan)):
        assert M.lib().moara_route_balance(*args, None) == M.MOARA_E_ARG, args


# ---------------------------------------------------------------- the oracle

def test_oracle_codes_of_known_values():
    m = np.zeros(32)
    m[:7] = [448.0, 1.0, -1.0625, 17.0, 2.0 ** -9, 2.0 ** -11, 0.0]
    e = O.block_exponents(m, 18)
    assert e.tolist() == [135]                  # 448 = 1.75 2^8
    c = O.encode_m(m, e)
    assert c[:7].tolist() == [0x7E, 0x38, 0xB8, 0x58, 1, 0, 0]      # -1.0625 and 17 are ties: to the even codes
    np.testing.assert_array_equal(O.decode_m(c, e)[:7], [448.0, 1.0, -1.0, 16.0, 2.0 ** -9, 0, 0])
    m[0] = 449.0
    assert O.block_exponents(m, 18).tolist() == [136]
    v = np.zeros(32)
    v[:5] = [1.75, 1.0, 1.0 + 1 / 32, 1e-30, 0.0]
    ev = O.block_exponents(v, 35)
    assert ev.tolist() == [127]
    low = O.encode_v(v, ev, np.zeros(32, np.int64))
    assert low[:5].tolist() == [254, 248, 248, 1, 0]
    high = O.encode_v(v, ev, np.full(32, 65535))
    assert high[:5].tolist() == [254, 248, 249, 1, 0]
    np.testing.assert_array_equal(O.decode_v(low, ev)[:4], [1.75, 1.0, 1.0, 2.0 ** -33])


def test_oracle_random_bits_are_even():
    r = O.random16(0, 1 << 16, 12345, 3)
    bits = (r[:, None] >> np.arange(16)) & 1
    n = r.size
    assert np.all(np.abs(bits.mean(axis=0) - 0.5) <= 5 * 0.5 / math.sqrt(n))
    for lag in (1, 2, 3, 32, 64):
        a, b = r[:-lag] - 32767.5, r[lag:] - 32767.5
        assert abs((a * b).mean() / (65536 ** 2 / 12)) <= 5 / math.sqrt(n)
    for other in (O.random16(0, n, 12346, 3), O.random16(0, n, 12345, 4), O.random16(0, n, 12345 + (1 << 32), 3),
                  O.random16(1 << 33, n, 12345, 3)):
        assert abs(((r - 32767.5) * (other - 32767.5)).mean() / (65536 ** 2 / 12)) <= 5 / math.sqrt(n)
    assert np.array_equal(O.random16(1000, 77, 12345, 3), r[1000:1077])


def test_oracle_routing_of_a_known_row():
    x = np.log(np.array([[1.0, 2.0, 4.0, 1.0, 6.0, 2.0]]))
    i, w, _ = O.route(x, 2, False)
    assert i.tolist() == [[4, 2]]
    np.testing.assert_allclose(w, [[6 / 16, 4 / 16]])
    i, w, _ = O.route(x, 3, False, renorm=True, scale=2.0)
    assert i.tolist() == [[4, 2, 1]]
    np.testing.assert_allclose(w, [[1.0, 4 / 6, 2 / 6]])
    i, _, _ = O.route(x, 2, False, groups=3, top_groups=1, group_best=2)    # groups of 3/16, 5/16, 8/16
    assert i.tolist() == [[4, 5]]
    i, _, _ = O.route(x, 2, False, groups=3, top_groups=1, group_best=1, bias=np.array([0, 0, 0.5, 0, 0, 0]))
    assert i.tolist() == [[2, 3]]
    i, w, _ = O.route(x, 2, True, bias=np.array([-np.inf] * 5 + [0]))
    assert i.tolist() == [[5, -1]]
    np.testing.assert_allclose(w, [[2 / 3, 0]])


@pytest.mark.parametrize("plant", ["no_rounding_up", "ties_to_odd", "bias_in_weight", "highest_index"])
def test_oracle_pins_catch_planted_mistakes(plant, monkeypatch):
    if plant == "no_rounding_up":
        real = O.encode_v
        monkeypatch.setattr(O, "encode_v", lambda v, ev, r: real(v, ev, 0 * r))
        pin = test_oracle_codes_of_known_values
    elif plant == "ties_to_odd":
        real_m = O.encode_m
        monkeypatch.setattr(O, "encode_m", lambda m, em: real_m(m * (1 + 1e-9), em))
        pin = test_oracle_codes_of_known_values
    elif plant == "bias_in_weight":
        real_s = O.weights
        monkeypatch.setattr(O, "weights", lambda l, i, s, r, c: real_s(l, i, s, r, c) + 0.5)
        pin = test_oracle_routing_of_a_known_row
    else:
        real_c = O.selection
        monkeypatch.setattr(O, "selection", lambda *a: real_c(*a) + 0 * 1e-3 + np.arange(6) * 1e-1)
        pin = test_oracle_routing_of_a_known_row
    with pytest.raises(AssertionError):
        pin()


# ---------------------------------------------------------------- the binding

def test_a_shared_routing_configuration_is_not_written(monkeypatch):
    """Calls on logits of both types, interleaved as threads may, each with its own type and the caller's other fields."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(M, "_on_gpu", lambda t, device, what: 0)
    cfg = M.moara_route_config(experts=6, top_k=2, groups=3, top_groups=2, group_best=2, score=M.MOARA_SIGMOID, renormalise=1,
                               logits_dtype=M.MOARA_F32, scale=2.5)
    before = bytes(cfg)
    half, dev, tokens, ld = M._route_logits(cfg, torch.zeros(4, 6, dtype=torch.bfloat16))
    full = M._route_logits(cfg, torch.zeros(4, 6))[0]
    assert bytes(cfg) == before
    assert half.logits_dtype == M.MOARA_BF16 and full.logits_dtype == M.MOARA_F32 and (dev, tokens, ld) == (0, 4, 6)
    for name, _ in M.moara_route_config._fields_:
        if name != "logits_dtype":
            assert getattr(half, name) == getattr(full, name) == getattr(cfg, name)


class _OnGpu:
    """What the binding asks a tensor for, on a GPU that is not here."""

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_a_given_stream_is_one_of_the_tensors_gpu(monkeypatch):
    """With the tensors on GPU 1 and GPU 0 current: handles are of GPU 1, streams of GPU 0 are refused, and the call
    sees the stream as the current one."""
    torch = pytest.importorskip("torch")
    now = []

    class Stream:
        def __init__(self, handle, device_index):
            self.cuda_stream, self.device_index = handle, device_index

    class Current:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            now.append(self.stream)

        def __exit__(self, *exc):
            now.pop()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0, 0 if device is None else device))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle, 0 if device is None else device))
    monkeypatch.setattr(torch.cuda, "stream", Current)
    call = M._streamed(lambda *a, **kw: (now[-1].cuda_stream, now[-1].device_index, [list(x) for x in a if isinstance(x, list)])
                       if now else None)
    t, cpu = _OnGpu(1), _OnGpu(-1)
    marshalled = M.GradArgs.__new__(M.GradArgs)
    marshalled.device = 1
    cfg = M.moara_route_config()
    for args, kw in (((t,), {}), ((cfg, t), {}), (([None, cpu, t],), {}), ((None, 1.0), dict(args=marshalled)),
                     (({0: t}.values(), 1.0), {}), ((None, 1.0), dict(lr=np.float32(1), steps=np.zeros(2), grads=(t,)))):
        assert call(*args, **kw) is None
        assert call(*args, stream=0, **kw)[:2] == (0, 1)
        assert call(*args, stream=77, **kw)[:2] == (77, 1)
        assert call(*args, stream=Stream(5, 1), **kw)[:2] == (5, 1)
        with pytest.raises(ValueError):
            call(*args, stream=Stream(5, 0), **kw)
    assert call((x for x in (None, t)), stream=77) == (77, 1, [[None, t]])      # a generator is read once
    assert call([], stream=77)[:2] == (77, 0) and call([], stream=Stream(5, 1))[:2] == (5, 1)
