"""Host-side checks of the training operators' C entry points (no GPU needed):
sizes, and refusals before any device call."""
import ctypes

import pytest

B = pytest.importorskip("paper_2307_15034_amd.binding")

BAD = B.FNO_ERR_INVALID_ARGUMENT


def _norm(**kw):
    a = dict(batch=2, points=100, channels=12, groups=3)
    a.update(kw)
    return B.make_norm_desc(**a)


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(points=0), dict(channels=0), dict(groups=0), dict(groups=5),
    dict(groups=24), dict(batch=-1), dict(channels=70000, groups=1), dict(dtype=3),
    dict(dtype=-1), dict(layout=2), dict(activation=3), dict(eps=-1e-5), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(points=1 << 38), dict(points=1 << 62), dict(batch=1 << 62)])
def test_norm_descriptor_refused(kw):
    with pytest.raises(B.FnoError) as e:
        B.fno_group_norm_act_workspace_size(_norm(**kw), B.FNO_OP_FWD)
    assert e.value.status == BAD


def test_norm_workspace_and_pointer_refusals():
    d = _norm()
    for op in (B.FNO_OP_FWD, B.FNO_OP_BWD):
        n = B.fno_group_norm_act_workspace_size(d, op)
        assert n >= 256 and n % 256 == 0
    for op in (B.FNO_OP_BWD_DATA, B.FNO_OP_BWD_WEIGHT, 9):
        with pytest.raises(B.FnoError):
            B.fno_group_norm_act_workspace_size(d, op)
    a = 1 << 20  # an aligned address that is never reached
    fwd = dict(x=a, gamma=a, beta=a, residual=a, out=a, stats=a, ws=a, ws_bytes=1 << 30, stream=0)
    for k, v in (("x", 0), ("out", 0), ("ws", 0), ("x", a + 2), ("out", a + 8), ("gamma", a + 4),
                 ("beta", a + 4), ("residual", a + 2), ("stats", a + 4), ("ws", a + 8)):
        assert B.fno_group_norm_act_fwd(d, **{**fwd, k: v}, check=False) == BAD, (k, v)
    assert B.fno_group_norm_act_fwd(d, **{**fwd, "ws_bytes": 0},
                                    check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL
    bwd = dict(x=a, gamma=a, beta=a, stats=a, g_out=a, gx=a, g_gamma=a, g_beta=a, ws=a,
               ws_bytes=1 << 30, stream=0)
    for k, v in (("x", 0), ("stats", 0), ("g_out", 0), ("gx", 0), ("ws", 0), ("gx", a + 2),
                 ("g_gamma", a + 4), ("g_beta", a + 4), ("stats", a + 4)):
        assert B.fno_group_norm_act_bwd(d, **{**bwd, k: v}, check=False) == BAD, (k, v)
    assert B.fno_group_norm_act_bwd(d, **{**bwd, "ws_bytes": 0},
                                    check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL


def _list(**kw):
    a = 1 << 20
    t = dict(param=a, master=None, grad=2 * a, exp_avg=3 * a, exp_avg_sq=4 * a, exp_avg_scale=None,
             exp_avg_sq_scale=None, n=100, param_dtype=B.FNO_DTYPE_F32, grad_dtype=B.FNO_DTYPE_F32,
             state_bits=32, weight_decay=0.01)
    t.update(kw)
    return (B.FnoAdamwTensor * 1)(B.FnoAdamwTensor(**t))


OPT = B.FnoAdamwDesc(1e-3, 0.9, 0.999, 1e-8)
A = 1 << 24


@pytest.mark.parametrize("kw", [
    dict(param=0), dict(param=(1 << 20) + 4), dict(grad=0), dict(exp_avg=0), dict(exp_avg_sq=0),
    dict(exp_avg=4 << 20), dict(n=-1), dict(n=(1 << 34) + 1), dict(param_dtype=3),
    dict(grad_dtype=B.FNO_DTYPE_F16), dict(state_bits=16), dict(state_bits=8),
    dict(state_bits=8, exp_avg_scale=A), dict(exp_avg_scale=A), dict(master=A),
    dict(param_dtype=B.FNO_DTYPE_F16, master=A + 4), dict(weight_decay=-1.0),
    dict(weight_decay=float("nan")), dict(weight_decay=float("inf")),
    dict(param_dtype=B.FNO_DTYPE_F16, grad_dtype=B.FNO_DTYPE_BF16)])
def test_adamw_tensor_refused(kw):
    assert B.fno_adamw_step(OPT, _list(**kw), 1, 1, 0, 0, check=False) == BAD


@pytest.mark.parametrize("hyper", [
    (-1e-3, 0.9, 0.999, 1e-8), (float("nan"), 0.9, 0.999, 1e-8), (float("inf"), 0.9, 0.999, 1e-8),
    (1e-3, 1.0, 0.999, 1e-8), (1e-3, -0.1, 0.999, 1e-8), (1e-3, 0.9, 1.0, 1e-8),
    (1e-3, 0.9, float("nan"), 1e-8), (1e-3, 0.9, 0.999, -1e-8), (1e-3, 0.9, 0.999, float("inf"))])
def test_adamw_hyper_refused(hyper):
    assert B.fno_adamw_step(B.FnoAdamwDesc(*hyper), _list(), 1, 1, 0, 0, check=False) == BAD


def test_adamw_call_refused():
    t = _list()
    assert B.fno_adamw_step(OPT, t, 1, 0, 0, 0, check=False) == BAD        # steps count from 1
    assert B.fno_adamw_step(OPT, t, 1, 1, A + 8, 0, check=False) == BAD    # control alignment
    assert B.fno_adamw_step(OPT, t, -1, 1, 0, 0, check=False) == BAD
    assert B.fno_adamw_step(OPT, None, 1, 1, 0, 0, check=False) == BAD
    assert B.fno_adamw_step(OPT, t, 0, 1, 0, 0, check=False) == B.FNO_OK   # nothing to do
    assert B.fno_adamw_step(OPT, None, 0, 1, 0, 0, check=False) == B.FNO_OK


def test_grad_norm_refused():
    t = _list()
    n = B.fno_grad_norm_workspace_size(t, 1)
    assert n >= 256 and n % 256 == 0
    assert B.fno_grad_norm_workspace_size(None, 0) >= 256
    ok = dict(max_norm=1.0, inv_loss_scale=1.0, control=A, ws=A, ws_bytes=n, stream=0)
    for k, v, st in (("max_norm", 0.0, BAD), ("max_norm", float("nan"), BAD),
                     ("inv_loss_scale", 0.0, BAD), ("inv_loss_scale", float("inf"), BAD),
                     ("inv_loss_scale", float("nan"), BAD), ("control", 0, BAD),
                     ("control", A + 8, BAD), ("ws", 0, BAD), ("ws", A + 8, BAD),
                     ("ws_bytes", n - 1, B.FNO_ERR_WORKSPACE_TOO_SMALL)):
        assert B.fno_grad_norm(OPT, t, 1, **{**ok, k: v}, check=False) == st, (k, v)
    assert B.fno_grad_norm(OPT, _list(grad=0), 1, **ok, check=False) == BAD
    with pytest.raises(B.FnoError):
        B.fno_grad_norm_workspace_size(_list(n=-1), 1)


def test_moments_refused():
    p = (ctypes.c_void_p * 1)(A)
    t8 = _list(state_bits=8, exp_avg_scale=A, exp_avg_sq_scale=A)
    assert B.fno_adamw_moments(_list(), 1, B.FNO_DTYPE_F32, p, p, 0, check=False) == BAD
    assert B.fno_adamw_moments(t8, 1, 7, p, p, 0, check=False) == BAD
    assert B.fno_adamw_moments(t8, 1, B.FNO_DTYPE_F32, None, p, 0, check=False) == BAD
    assert B.fno_adamw_moments(t8, 1, B.FNO_DTYPE_F32, (ctypes.c_void_p * 1)(A + 2), p, 0,
                               check=False) == BAD
    assert B.fno_adamw_moments(t8, 0, B.FNO_DTYPE_F32, p, p, 0, check=False) == B.FNO_OK
