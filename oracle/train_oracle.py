"""float64 CPU oracle of the training operators beside the spectral layer:
group norm with an activation, the gradient norm and the AdamW step with 32-
and 8-bit states (test infrastructure only, written from the definitions; it
shares no code with the HIP path).

`adamw_step32` is the same step in numpy float32, one rounded operation at a
time in the order that the C header states: what a device step has to give bit
for bit.
"""
from __future__ import annotations

import numpy as np
import scipy.special

ACT_NONE, ACT_GELU, ACT_SILU = "none", "gelu", "silu"
BLOCK = 256


def act(z, kind):
    if kind == ACT_GELU:
        return z * 0.5 * (1.0 + scipy.special.erf(z / np.sqrt(2.0)))
    if kind == ACT_SILU:
        return z * scipy.special.expit(z)
    return z


def act_grad(z, kind):
    if kind == ACT_GELU:
        return (0.5 * (1.0 + scipy.special.erf(z / np.sqrt(2.0)))
                + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi))
    if kind == ACT_SILU:
        s = scipy.special.expit(z)
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def _grouped(x, groups):
    """[B, C, P] -> [B, G, C/G, P] in float64."""
    x = np.asarray(x, np.float64)
    return x.reshape(x.shape[0], groups, x.shape[1] // groups, x.shape[2])


def group_norm_act_fwd(x, gamma, beta, groups, eps, kind, residual=None):
    """x [B, C, P] -> (out [B, C, P], stats [B, G, 2])."""
    v = _grouped(x, groups)
    mean = v.mean((2, 3))
    var = ((v - mean[:, :, None, None]) ** 2).mean((2, 3))
    rstd = 1.0 / np.sqrt(var + eps)
    xh = ((v - mean[:, :, None, None]) * rstd[:, :, None, None]).reshape(x.shape)
    z = xh * np.asarray(gamma, np.float64)[None, :, None] + np.asarray(beta, np.float64)[None, :, None]
    out = act(z, kind)
    if residual is not None:
        out = out + np.asarray(residual, np.float64)
    return out, np.stack([mean, rstd], -1)


def group_norm_act_bwd(x, gamma, beta, groups, eps, kind, g_out):
    """(gx, g_gamma, g_beta, scale, |g_gamma| sum, |g_beta| sum): scale [B, C, P] is
    rstd gamma h, the size of the terms whose difference gx is; the last two
    are the parameter gradients' sums over absolute values."""
    _, stats = group_norm_act_fwd(x, gamma, beta, groups, eps, kind)
    v = _grouped(x, groups)
    rstd = stats[:, :, 1][:, :, None, None]
    xh = (v - stats[:, :, 0][:, :, None, None]) * rstd
    ga = np.asarray(gamma, np.float64).reshape(1, groups, -1, 1)
    be = np.asarray(beta, np.float64).reshape(1, groups, -1, 1)
    h = _grouped(g_out, groups) * act_grad(xh * ga + be, kind)
    hx = h * xh
    c = np.asarray(gamma).size
    sums = [t.sum((0, 3)).reshape(c) for t in (hx, h, np.abs(hx), np.abs(h))]
    gh = ga * h
    a = gh.mean((2, 3), keepdims=True)
    d = (gh * xh).mean((2, 3), keepdims=True)
    gx = rstd * (gh - a - xh * d)
    return gx.reshape(x.shape), sums[0], sums[1], (rstd * gh).reshape(x.shape), sums[2], sums[3]


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
def grad_norm(grads, max_norm, inv_scale):
    """(norm, scale, finite)."""
    total = sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads)
    norm = np.sqrt(total) * inv_scale
    return norm, inv_scale * min(1.0, max_norm / norm if norm > 0 else 1.0), bool(np.isfinite(total))


def adamw_step(p, g, m, v, t, lr, b1, b2, eps, wd, scale=1.0):
    """One step in float64: (p, m, v)."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    mh, vh = m / (1 - b1 ** t), v / (1 - b2 ** t)
    return p * (1 - lr * wd) - lr * mh / (np.sqrt(vh) + eps), m, v


def adamw_step32(p, g, m, v, t, lr, b1, b2, eps, wd, scale=1.0):
    """The step in float32, each operation rounded: (p, m, v, sqrt(v))."""
    f = np.float32
    p, g, m, v = (np.asarray(a, f) for a in (p, g, m, v))
    with np.errstate(all="ignore"):
        g = g * f(scale)
        m = m * f(b1) + g * f(1 - b1)
        v = v * f(b2) + (g * g) * f(1 - b2)
        w = np.sqrt(v)
        size, root = f(lr / (1 - b1 ** t)), f(1 / np.sqrt(1 - b2 ** t))
        p = p * f(1 - lr * wd) - (m * size) / (w * root + f(eps))
    return p, m, v, w


def _blocks(x):
    pad = np.zeros(-(-x.size // BLOCK) * BLOCK, x.dtype)
    pad[:x.size] = x.reshape(-1)
    return pad.reshape(-1, BLOCK)


def encode8(m, w):
    """Codes and scales of m and w = sqrt(v) (float32, finite): (qm, qv, A, B)."""
    f = np.float32
    mb, wb = _blocks(np.asarray(m, f)), _blocks(np.asarray(w, f))
    a, b = np.abs(mb).max(1), wb.max(1)
    one = f(1)
    qm = np.rint(np.sqrt(np.abs(mb) / np.where(a > 0, a, one)[:, None]) * f(127)) * np.sign(mb)
    qv = np.rint(np.sqrt(wb / np.where(b > 0, b, one)[:, None]) * f(255))
    qv = np.where((wb > 0) & (qv < 1), one, qv)
    n = np.asarray(m).size
    return (qm.reshape(-1)[:n].astype(np.int8), qv.reshape(-1)[:n].astype(np.uint8), a, b)


def decode8(qm, qv, a, b):
    """(m, v) in float32."""
    f = np.float32
    n = qm.size
    qm, qv = qm.astype(f), qv.astype(f)
    am, bv = np.repeat(a, BLOCK)[:n], np.repeat(b, BLOCK)[:n]
    m = (am * f(1 / 16129)) * (qm * np.abs(qm))
    s = (bv * f(1 / 65025)) * (qv * qv)
    return m, s * s
