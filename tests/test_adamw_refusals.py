"""What adamw_step, adamw_unpack and their binding refuse, before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2002_03629_amd import binding as B


def config(**kw):
    base = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, param_dtype=B.MADE_F32,
                grad_dtype=B.MADE_F32, moment_bits=32)
    base.update(kw)
    return B.adamw_config(*base.values())


def call(cfg, sizes=(5,), null=None, copies=False, scalars=None, n=None):
    """null: index of the pointer array (params, grads, m, v, m_scale, v_scale) whose pointer is NULL"""
    arr = [(C.c_void_p * len(sizes))(*[None if i == null else 4096] * len(sizes)) for i in range(7)]
    if not copies:
        arr[6] = None
    return B.lib().adamw_step(C.byref(cfg) if cfg else None, len(sizes) if n is None else n, (C.c_int64 * len(sizes))(*sizes), *arr, scalars, None)


BAD = [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=-1e-9), dict(eps=float("inf")), dict(weight_decay=float("nan")),
       dict(lr=float("inf")), dict(grad_scale=float("nan")), dict(step=0), dict(param_dtype=2), dict(grad_dtype=-1), dict(moment_bits=16)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_bad_numbers(bad):
    assert call(config(**bad)) == B.MADE_ERR_ARG
    assert "adamw_step" in B.made_last_error()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [1e-40, 1e-300, 1e39])
def test_eps_that_is_no_normal_fp32_number(eps, bits):
    """rounded to fp32 it would be zero, or its reciprocal or itself infinite"""
    assert call(config(eps=eps, moment_bits=bits)) == B.MADE_ERR_ARG
    assert "eps" in B.made_last_error()


def test_a_tensor_of_more_than_a_launch_takes():
    assert call(config(), sizes=((1 << 36),)) == B.MADE_ERR_ARG
    assert "elements" in B.made_last_error()


def test_bad_arguments():
    assert call(None) == B.MADE_ERR_ARG
    assert call(config(), n=-1) == B.MADE_ERR_ARG
    assert call(config(), sizes=(4, -1)) == B.MADE_ERR_ARG
    for i in range(4):
        assert call(config(), null=i) == B.MADE_ERR_ARG
    for i in range(6):
        assert call(config(moment_bits=8), null=i) == B.MADE_ERR_ARG
    assert call(config(param_dtype=B.MADE_BF16), copies=True) == B.MADE_ERR_ARG
    L = B.lib()
    assert L.adamw_step(C.byref(config()), 1, None, *[None] * 7, None, None) == B.MADE_ERR_ARG
    assert L.adamw_unpack(1, (C.c_int64 * 1)(3), *[None] * 6, None) == B.MADE_ERR_ARG
    assert L.adamw_unpack(-1, None, *[None] * 6, None) == B.MADE_ERR_ARG


def test_no_tensors_and_empty_tensors_need_no_pointers():
    assert call(config(), n=0) == B.MADE_OK
    L = B.lib()
    none = (C.c_void_p * 2)()
    assert L.adamw_step(C.byref(config()), 2, (C.c_int64 * 2)(0, 0), none, none, none, none, None, None, None, None, None) == B.MADE_OK
    assert L.adamw_unpack(0, None, *[None] * 6, None) == B.MADE_OK


def test_the_binding_refuses_tensors_of_the_host():
    t = [torch.zeros(4)]
    with pytest.raises(ValueError, match="GPU"):
        B.adamw_step(t, t, t, t, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    with pytest.raises(ValueError):
        B.adamw_moments(t, 4)
    with pytest.raises(ValueError):
        B.PreparedAdamW([], [], [], [])


def test_zeroed_moments():
    m, v, ms, vs = B.adamw_moments([torch.zeros(3, 100), torch.zeros(1)], 8)
    assert [x.dtype for x in (m[0], v[0], ms[0], vs[0])] == [torch.int8, torch.uint8, torch.float32, torch.float32]
    assert [x.shape for x in m] == [(3, 100), (1,)] and [x.numel() for x in ms] == [2, 1]


def test_calls_of_one_prepared_step_have_their_own_numbers(monkeypatch):
    """a call made while another of the same object is under way (two threads) does not change the other's numbers"""
    seen = []

    class Library:
        @staticmethod
        def adamw_step(cfg, *args):
            if cfg._obj.step == 1:
                plan(2.0, 0.8, 0.8, 1.0, 0.0, 2, 0.5)
            seen.append((cfg._obj.lr, cfg._obj.beta1, cfg._obj.step, cfg._obj.grad_scale, cfg._obj.moment_bits))
            return B.MADE_OK

    monkeypatch.setattr(B, "_on_device", lambda t, *a: t)              # (tensors of the host, a library that computes nothing)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    plan = B.PreparedAdamW(*[[torch.zeros(4)] for _ in range(4)])
    plan(1.0, 0.9, 0.9, 1.0, 0.0, 1)
    assert seen == [(2.0, 0.8, 2, 0.5, 32), (1.0, 0.9, 1, 1.0, 32)]
