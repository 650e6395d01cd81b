"""Every element of the residual norm's results against the float64 oracle, with
a bound of its own for each.

E = 2^-24, a rounding to fp32.  A row's sums are formed by threads that hold up
to 16 values each and joined over up to 2^10 threads: at most D = 32 roundings of
E on the sum of absolute terms.  For rows v that are themselves off by dv:
  mean    dm  = mean(dv) + D E mean|v|
  d       dd  = E (|v| + |mean|) + dv + dm                (d = v - mean)
  r       rho = mean(|d| dd) r^2 + (D + 6) E, relative    (r = 1 / sqrt(var + eps))
  xh      r dd + |xh| (rho + 2 E)
and, with t off by dt, for a norm's gradient r (t - m - xh q):
  m       mean(dt) + D E mean|t|
  q       mean(dt |xh| + |t| dxh) + (D + 2) E mean|t xh|
  result  r (dt + dm + dxh |q| + |xh| dq + 4 E (|t| + |m| + |xh q|)) + rho |result|
Parameters' sums are chains of at most 128 additions, a tree over a work-group's
threads (at most 2^6) and doubles: (128 + 12) E of the sum of absolute terms,
beside the terms' own errors.  A stored result is rounded once: u |result| and
half the spacing of the type's subnormals.
"""
import numpy as np

from oracle import channel_oracle as C

E = 2.0 ** -24
D = 32
CHAIN = 140
U = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
SUB = {"fp32": 2.0 ** -150, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}


def _mean(v):
    return v.mean(1, keepdims=True)


def norm_err(v, dv, kind, eps):
    """(xh, r, dxh, rho)."""
    xh, r = C.norm_rows(v, kind, eps)
    m = _mean(v) if kind == "layer" else 0.0
    dm = _mean(dv) + D * E * _mean(np.abs(v)) if kind == "layer" else 0.0
    dd = E * (np.abs(v) + np.abs(m)) + dv + dm
    rho = _mean(np.abs(v - m) * dd) * r * r + (D + 6) * E
    return xh, r, r * dd + np.abs(xh) * (rho + 2 * E), rho


def grad_err(t, dt, xh, dxh, r, rho, kind):
    out = C.norm_rows_grad(t, xh, r, kind)
    m = _mean(t) if kind == "layer" else np.zeros_like(r)
    dm = _mean(dt) + D * E * _mean(np.abs(t)) if kind == "layer" else 0.0
    q = _mean(t * xh)
    dq = _mean(dt * np.abs(xh) + np.abs(t) * dxh) + (D + 2) * E * _mean(np.abs(t * xh))
    big = np.abs(t) + np.abs(m) + np.abs(xh * q)
    return out, r * (dt + dm + dxh * np.abs(q) + np.abs(xh) * dq + 4 * E * big) + rho * np.abs(out)


def _par(p, rows, c):
    one = lambda k: np.ones(c) if p.get(k) is None else p[k]  # noqa: E731
    zero = lambda k: np.zeros(c) if p.get(k) is None else p[k]  # noqa: E731
    gate = np.ones((rows, c)) if p.get("gate") is None else C.spread_gate(p["gate"], rows)
    return one("post_w"), zero("post_b"), gate, one("scale"), one("pre_w"), zero("pre_b")


def forward(x, u, p, kind, eps, dt):
    """{"y", "h"}: (value, bound)."""
    pw, pb, gate, scale, qw, qb = _par(p, *x.shape)
    out, y, dy = {}, x, np.zeros_like(x)
    if u is not None:
        xh, _, dxh, _ = norm_err(u, np.zeros_like(u), kind, eps)
        n = xh * pw + pb
        dn = np.abs(pw) * dxh + 2 * E * (np.abs(pw * xh) + np.abs(pb))
        y = scale * x + gate * n
        dy = np.abs(gate) * dn + 3 * E * (np.abs(scale * x) + np.abs(gate * n))
        out["y"] = (y, dy + (U[dt] * 1.001) * np.abs(y) + SUB[dt])
    xh, _, dxh, _ = norm_err(y, dy, kind, eps)
    h = xh * qw + qb
    dh = np.abs(qw) * dxh + 2 * E * (np.abs(qw * xh) + np.abs(qb))
    out["h"] = (h, dh + (U[dt] * 1.001) * np.abs(h) + SUB[dt])
    return out


def backward(x, u, y, p, kind, eps, g_y, g_h, dt, gate_dt="fp32"):
    """{"g_x", ...}: (value, bound)."""
    rows, c = x.shape
    pw, pb, gate, scale, qw, _ = _par(p, rows, c)
    out = {}
    over = lambda v, dv, axis=0: (v.sum(axis), dv.sum(axis) + CHAIN * E * np.abs(v).sum(axis))  # noqa: E731
    g = np.zeros_like(x) if g_y is None else g_y
    dg = np.zeros_like(x)
    if g_h is not None:
        xh, r, dxh, rho = norm_err(x if u is None else y, np.zeros_like(x), kind, eps)
        out["g_pre_w"] = over(g_h * xh, np.abs(g_h) * (dxh + E * np.abs(xh)))
        out["g_pre_b"] = over(g_h, np.zeros_like(g_h))
        t = g_h * qw
        d, dd = grad_err(t, E * np.abs(t), xh, dxh, r, rho, kind)
        g = g + d
        dg = dd + E * np.abs(g)
    rounded = lambda v, dv: (v, dv + (U[dt] * 1.001) * np.abs(v) + SUB[dt])  # noqa: E731
    out["g_x"] = rounded(g * scale, np.abs(scale) * dg + E * np.abs(g * scale))
    if u is not None:
        xh, r, dxh, rho = norm_err(u, np.zeros_like(u), kind, eps)
        out["g_scale"] = over(g * x, dg * np.abs(x) + E * np.abs(g * x))
        if p.get("gate") is not None:
            n = xh * pw + pb
            dn = np.abs(pw) * dxh + 2 * E * (np.abs(pw * xh) + np.abs(pb))
            v, dv = g * n, np.abs(g) * dn + dg * np.abs(n) + E * np.abs(g * n)
            s = p["gate"].shape[0]
            v, dv = over(v.reshape(s, -1, c), dv.reshape(s, -1, c), 1)
            out["g_gate"] = (v, dv + (U[gate_dt] * 1.001) * np.abs(v) + SUB[gate_dt])
        t = g * gate
        dt_ = dg * np.abs(gate) + E * np.abs(t)
        out["g_post_w"] = over(t * xh, dt_ * np.abs(xh) + np.abs(t) * dxh + E * np.abs(t * xh))
        out["g_post_b"] = over(t, dt_)
        v, dv = grad_err(t * pw, dt_ * np.abs(pw) + E * np.abs(t * pw), xh, dxh, r, rho, kind)
        out["g_u"] = rounded(v, dv)
    return out


def close(name, got, want, bound):
    got = np.asarray(got, np.float64).reshape(want.shape)
    bad = ~(np.abs(got - want) <= bound)  # not a number is bad too
    if bad.any():
        i = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} elements, first {i}: "
                             f"{got[i]!r}, expected {want[i]!r} within {bound[i]:.3e}")
