"""Host side of the operators around the layer: what they refuse, before anything is launched, and the
workspace they ask for (no GPU needed; the addresses are never followed)."""
import ctypes
import os
import subprocess

import pytest

import paper_2101_03961_amd as sw

OK = 0x1000   # aligned, never dereferenced
INF, NAN = float("inf"), float("nan")


def linear(**kw):
    base = dict(M=100, K=64, N=128, act_dtype=sw.SW_BF16, activation=sw.SW_ACT_RELU, dropout=0.0, flags=0, seed=1)
    base.update(kw)
    return sw.SwitchLinearConfig(*[base[k] for k, _ in sw.SwitchLinearConfig._fields_])


def balance(**kw):
    base = dict(T=100, E=8, k=2, n_groups=1, alpha=0.01, flags=0)
    base.update(kw)
    return sw.SwitchBalanceConfig(*[base[k] for k, _ in sw.SwitchBalanceConfig._fields_])


def forward(cfg, x=OK, W=OK, bias=OK, residual=OK, y=OK, z=OK, ws=OK, size=1 << 40):
    return sw.switch_linear(cfg, x, W, bias, residual, y, z, ws, size, check=False)


def backward(cfg, dy=OK, x=OK, W=OK, z=OK, dx=OK, dW=OK, db=OK, ws=OK, size=1 << 40):
    return sw.switch_linear_backward(cfg, dy, x, W, z, dx, dW, db, ws, size, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), -2), (dict(M=1 << 31), -2), (dict(K=0), -2), (dict(N=0), -2), (dict(K=-8), -2),
    (dict(K=60), -2), (dict(N=124), -2), (dict(K=1 << 21), -2), (dict(N=1 << 21), -2),
    (dict(act_dtype=sw.SW_F32, K=62), -2), (dict(act_dtype=sw.SW_F32, N=126), -2),
    (dict(N=1 << 20, activation=sw.SW_ACT_GEGLU), -2),                       # 2 N columns
    (dict(K=1 << 15, N=1 << 15), -2), (dict(K=1 << 15, N=1 << 14, act_dtype=sw.SW_F32), -2),   # W of 2 GB
    (dict(K=1 << 15, N=1 << 14, activation=sw.SW_ACT_GEGLU), -2),
    (dict(act_dtype=2), -4), (dict(act_dtype=-1), -4), (dict(activation=4), -4), (dict(activation=-1), -4),
    (dict(dropout=1.0), -3), (dict(dropout=-0.1), -3), (dict(dropout=NAN), -3), (dict(flags=1), -3)])
def test_linear_configurations_refused(kw, status):
    assert ctypes.sizeof(sw.SwitchLinearConfig) == 48   # the header's struct
    cfg = linear(**kw)
    for back in (False, True):
        with pytest.raises(sw.SwitchError) as e:
            sw.switch_linear_workspace_size(cfg, back)
        assert e.value.status == status
    assert forward(cfg) == status and backward(cfg) == status


def test_linear_pointers_refused():
    cfg = linear()
    for name in ("x", "W", "y"):
        assert forward(cfg, **{name: None}) == -1
    for name in ("x", "W", "bias", "residual", "y", "z"):
        assert forward(cfg, **{name: OK + 8}) == -6
    for name in ("dy", "x", "W", "z"):
        assert backward(cfg, **{name: None}) == -1
    for name in ("dy", "x", "W", "z", "dx", "dW", "db"):
        assert backward(cfg, **{name: OK + 8}) == -6
    assert backward(cfg, dx=None, dW=None, db=None) == -1
    need = sw.switch_linear_workspace_size(cfg, True)
    assert need >= 100 * 128 * 2
    assert backward(cfg, size=need - 1) == -5
    assert backward(cfg, ws=None) == -5 and backward(cfg, ws=OK + 16) == -5
    need = sw.switch_linear_workspace_size(linear(M=16, K=8192, N=256, activation=sw.SW_ACT_NONE), False)
    if need:
        assert forward(linear(M=16, K=8192, N=256, activation=sw.SW_ACT_NONE), size=need - 1) == -5


def test_no_rows_is_no_work():
    cfg = linear(M=0)
    assert sw.switch_linear_workspace_size(cfg, False) == 0 and sw.switch_linear_workspace_size(cfg, True) == 0
    assert forward(cfg, x=None, W=None, bias=None, residual=None, y=None, z=None, ws=None, size=0) == 0
    # only dx, which has no rows: nothing to write
    assert backward(cfg, dy=None, x=None, W=None, z=None, dW=None, db=None, ws=None, size=0) == 0
    assert sw.switch_dropout(0, sw.SW_F32, 0.1, 1, None, None, None, check=False) == 0
    assert sw.switch_balance_loss_backward(balance(T=0), 1.0, None, None, None, None, None, check=False) == 0


@pytest.mark.parametrize("args,status", [
    ((8, 2, 0.1, 1, OK, None, OK), -4), ((-1, 0, 0.1, 1, OK, None, OK), -2), ((1 << 40, 0, 0.1, 1, OK, None, OK), -2),
    ((8, 0, 1.0, 1, OK, None, OK), -3), ((8, 0, -0.5, 1, OK, None, OK), -3), ((8, 0, NAN, 1, OK, None, OK), -3),
    ((8, 0, 0.1, 1, None, None, OK), -1), ((8, 0, 0.1, 1, OK, None, None), -1),
    ((8, 0, 0.1, 1, OK + 4, None, OK), -6), ((8, 0, 0.1, 1, OK, OK + 8, OK), -6), ((8, 0, 0.1, 1, OK, None, OK + 2), -6)])
def test_dropout_refusals(args, status):
    assert sw.switch_dropout(*args, check=False) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -2), (dict(T=1 << 31), -2), (dict(E=0), -2), (dict(E=4097), -2), (dict(k=0), -2), (dict(k=9), -2),
    (dict(T=1 << 30, k=2), -2), (dict(n_groups=-1), -2), (dict(n_groups=3), -2), (dict(T=65536, n_groups=65536), -2),
    (dict(alpha=NAN), -3), (dict(alpha=INF), -3), (dict(flags=2), -3)])
def test_balance_configurations_refused(kw, status):
    assert ctypes.sizeof(sw.SwitchBalanceConfig) == 40
    cfg = balance(**kw)
    with pytest.raises(sw.SwitchError) as e:
        sw.switch_balance_workspace_size(cfg)
    assert e.value.status == status
    assert sw.switch_balance_loss(cfg, *([OK] * 7), 1 << 40, check=False) == status
    assert sw.switch_balance_loss_backward(cfg, 1.0, *([OK] * 5), check=False) == status


def test_balance_pointers_refused():
    cfg = balance()
    need = sw.switch_balance_workspace_size(cfg)
    call = lambda i, v, size=need: sw.switch_balance_loss(cfg, *[v if j == i else OK for j in range(7)], size, check=False)
    for i in (0, 1, 3, 4, 5):
        assert call(i, None) == -1
        assert call(i, OK + 4) == -6
    assert call(6, None) == -5 and call(6, OK + 16) == -5 and call(6, OK, need - 1) == -5
    back = lambda i, v: sw.switch_balance_loss_backward(cfg, 1.0, *[v if j == i else OK for j in range(5)], check=False)
    for i in (0, 2, 3, 4):
        assert back(i, None) == -1
        assert back(i, OK + 4) == -6
    for d in (NAN, INF):
        assert sw.switch_balance_loss_backward(cfg, d, *([OK] * 5), check=False) == -3
    assert sw.switch_balance_loss(balance(T=0), None, None, None, None, OK, OK, None, 0, check=False) == -1


def test_null_configuration_and_size():
    lib = ctypes.CDLL(sw.library_path())
    size = ctypes.c_size_t()
    assert lib.switch_linear_workspace_size(None, 0, ctypes.byref(size)) == -1
    assert lib.switch_linear_workspace_size(ctypes.byref(linear()), 0, None) == -1
    assert lib.switch_balance_workspace_size(None, ctypes.byref(size)) == -1
    assert lib.switch_balance_workspace_size(ctypes.byref(balance()), None) == -1
