"""Float64 oracle of the operators over channels: the norms around a block with
gate and residual scale, and products of 8-bit codes with block scales.  Plain
NumPy from the definitions; no code shared with the library."""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------------------
# Residual norm
# ---------------------------------------------------------------------------
def norm_rows(v, kind, eps):
    """(normalised rows, 1 / sqrt(var + eps))."""
    if kind == "layer":
        v = v - v.mean(1, keepdims=True)
    with np.errstate(all="ignore"):
        r = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
        return v * r, r


def norm_rows_grad(t, xh, r, kind):
    """Gradient of the rows from that of the normalised rows."""
    g = t - xh * (t * xh).mean(1, keepdims=True)
    if kind == "layer":
        g = g - t.mean(1, keepdims=True)
    return g * r


def spread_gate(gate, rows):
    """The gate of each row [rows, C]."""
    return np.repeat(gate, rows // gate.shape[0], 0)


def residual_norm_fwd(x, u, p, kind, eps):
    """p: {"post_w", "post_b", "gate", "scale", "pre_w", "pre_b"}, each an array
    or None; u None: the entry form.  Returns (y, h)."""
    one = lambda k: 1.0 if p.get(k) is None else p[k]  # noqa: E731
    zero = lambda k: 0.0 if p.get(k) is None else p[k]  # noqa: E731
    y = x
    if u is not None:
        n = norm_rows(u, kind, eps)[0] * one("post_w") + zero("post_b")
        gate = 1.0 if p.get("gate") is None else spread_gate(p["gate"], len(x))
        y = one("scale") * x + gate * n
    return y, norm_rows(y, kind, eps)[0] * one("pre_w") + zero("pre_b")


def residual_norm_bwd(x, u, y, p, kind, eps, g_y, g_h):
    """Gradients by name; g_h None: no second norm."""
    one = lambda k: 1.0 if p.get(k) is None else p[k]  # noqa: E731
    zero = lambda k: 0.0 if p.get(k) is None else p[k]  # noqa: E731
    out = {}
    g = g_y
    if g_h is not None:
        xh, r = norm_rows(x if u is None else y, kind, eps)
        out["g_pre_w"], out["g_pre_b"] = (g_h * xh).sum(0), g_h.sum(0)
        g = g + norm_rows_grad(g_h * one("pre_w"), xh, r, kind)
    out["g_x"] = g * one("scale")
    if u is not None:
        xh, r = norm_rows(u, kind, eps)
        out["g_scale"] = (g * x).sum(0)
        if p.get("gate") is not None:
            d = g * (xh * one("post_w") + zero("post_b"))
            out["g_gate"] = d.reshape(p["gate"].shape[0], -1, d.shape[1]).sum(1)
            g = g * spread_gate(p["gate"], len(g))
        out["g_post_w"], out["g_post_b"] = (g * xh).sum(0), g.sum(0)
        out["g_u"] = norm_rows_grad(g * one("post_w"), xh, r, kind)
    return out


# ---------------------------------------------------------------------------
# 8-bit codes with a scale for each block of 128
# ---------------------------------------------------------------------------
BLOCK = 128
FORMATS = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}


def decode_table(fmt):
    """The 256 values of a format, from its definition: sign, exponent with bias,
    fraction; e4m3 has NaN at all ones and no infinity, e5m2 is a short fp16."""
    out = np.zeros(256)
    bits, bias = (3, 7) if fmt == "e4m3" else (2, 15)
    for c in range(256):
        e, f = (c & 127) >> bits, c & ((1 << bits) - 1)
        v = (f / 2.0 ** bits) * 2.0 ** (1 - bias) if e == 0 else (1 + f / 2.0 ** bits) * 2.0 ** (e - bias)
        if fmt == "e4m3" and (c & 127) == 127:
            v = np.nan
        if fmt == "e5m2" and e == 31:
            v = np.inf if f == 0 else np.nan
        out[c] = -v if c & 128 else v
    return out


def round8(v, fmt):
    """v to the nearest value of the format, ties to even; |v| at most its
    largest value, or not finite (an infinity becomes NaN in e4m3)."""
    top, bits, low = FORMATS[fmt]
    ok = np.isfinite(v)
    w = np.where(ok, v, 0.0)
    e = np.maximum(np.frexp(w)[1] - 1, low)
    unit = np.ldexp(1.0, e - bits)
    r = np.rint(w / unit) * unit
    bad = np.where(np.isnan(v) | (fmt == "e4m3"), np.nan, v)
    return np.where(ok, r, bad)


def block_scale(a, fmt, kind):
    """Scales of blocks whose largest finite sizes are a."""
    top = FORMATS[fmt][0]
    safe = np.where(a > 0, a, 1.0)
    if kind == "pow2":
        m, e = np.frexp(safe)  # top = 0.875 2^k
        k = np.frexp(top)[1]
        s = np.ldexp(1.0, np.maximum(e - k + (m > 0.875), -126))
    else:
        s = np.maximum(safe.astype(np.float32) * (np.float32(1.0) / np.float32(top)),
                       np.float32(2.0 ** -126)).astype(np.float64)
    return np.where(a > 0, s, 1.0)


def quantize(v, fmt, kind, tile=False):
    """(values of the codes [R, C], scales [C/128, R or R/128]) of v [R, C]."""
    r, c = v.shape
    q, scales = np.zeros((r, c)), []
    for j in range(0, c, BLOCK):
        b = v[:, j:j + BLOCK]
        a = np.where(np.isfinite(b), np.abs(b), 0.0).max(1)
        if tile:
            a = np.array([a[i:i + BLOCK].max() for i in range(0, r, BLOCK)])
        s = block_scale(a, fmt, kind)
        scales.append(s)
        s = np.repeat(s, BLOCK)[:r] if tile else s
        inv = (np.float32(1.0) / s.astype(np.float32)).astype(np.float64)
        t = b * inv[:, None]
        with np.errstate(over="ignore"):
            q[:, j:j + BLOCK] = round8(t if kind == "pow2" else t.astype(np.float32).astype(np.float64), fmt)
    return q, np.stack(scales)


def values(q, s, tile=False):
    out = q.copy()
    for j in range(s.shape[0]):
        f = np.repeat(s[j], BLOCK)[:len(q)] if tile else s[j]
        out[:, j * BLOCK:(j + 1) * BLOCK] *= f[:, None]
    return out
