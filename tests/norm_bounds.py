"""Every element of a group norm's results against the float64 oracle, with a
bound of its own for each.

E = 2^-24, a rounding to fp32.  With exact statistics mean, r and xh = r (x -
mean), m = |mean| r, the kernels' arithmetic is off by at most
  xh     E (4 |xh| + m): the fp32 mean, x - mean, r, the product
  z      E Z, Z = |gamma| (4 |xh| + m) + |beta| + |z|
  act    1.13 E Z + 10 E |z|: the slope is at most 1.13; erfc to 0.75e-7, its
         exponential and reciprocal
  act'   E (0.8 Z + 10): the second derivative is at most 0.8; the fit 3.3e-7
so that h = g_out act'(z) is off by dh = E |g_out| (0.8 Z + 10).  Sums of h and
h xh are chains of at most CHAIN fp32 additions, doubles from there: CHAIN E of
the sum of absolute terms, beside the terms' own errors.  A stored result is
rounded once: u |result|, and half the spacing of the type's subnormals.
"""
import numpy as np
import torch

from oracle import train_oracle as T
from tests.gpu_util import say
from paper_2307_15034_amd.layer import GroupNormAct

E = 2.0 ** -24
CHAIN = 128
U = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
SUB = {"fp32": 2.0 ** -150, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}


def reference(x, gamma, beta, groups, eps, kind, g_out, residual, dt):
    """{name: (value, bound)} of out, gx, g_gamma, g_beta; [B, C, P] arrays."""
    b, c, p = x.shape
    out, stats = T.group_norm_act_fwd(x, gamma, beta, groups, eps, kind, residual)
    gx, gg, gb = T.group_norm_act_bwd(x, gamma, beta, groups, eps, kind, g_out)[:3]
    per = lambda t: np.repeat(t, c // groups, 1)[:, :, None]  # noqa: E731
    mean, r = per(stats[:, :, 0]), per(stats[:, :, 1])
    ga, be = np.abs(gamma)[None, :, None], np.abs(beta)[None, :, None]
    s = (x - mean) * r
    z = s * gamma[None, :, None] + beta[None, :, None]
    s, m, z = np.abs(s), np.abs(mean) * r, np.abs(z)
    big = ga * (4 * s + m) + be + z
    wide = E * (1.13 * big + 10 * z + 2 * np.abs(out))
    if residual is not None:
        wide = wide + 4 * E * np.abs(residual)
    h, dh = 1.13 * np.abs(g_out), E * np.abs(g_out) * (0.8 * big + 10)
    ds = E * (4 * s + m)
    mean_of = lambda t: per(t.reshape(b, groups, -1).mean(2))  # noqa: E731
    d = mean_of(ga * h * s)
    da = mean_of(ga * dh) + (CHAIN + 4) * E * mean_of(ga * h)
    dd = mean_of(ga * (dh * s + h * ds)) + (CHAIN + 4) * E * d
    back = r * (ga * (dh + 4 * E * h) + da + s * dd + (ds + 6 * E * s) * d + 4 * E * mean_of(ga * h))
    rounded = lambda t: U[dt] * np.abs(t) + SUB[dt]  # noqa: E731
    over = lambda t: t.sum((0, 2))  # noqa: E731
    return {"out": (out, rounded(out) * 1.001 + wide),
            "gx": (gx, rounded(gx) * 1.001 + back),
            "g_gamma": (gg, over(dh * s + h * ds) + (CHAIN + 4) * E * over(h * s)),
            "g_beta": (gb, over(dh) + (CHAIN + 4) * E * over(h))}


def rows(t, last):
    """[B, C, P] in float64 of a tensor of either layout."""
    a = t.double().cpu().numpy()
    a = np.moveaxis(a, -1, 1) if last else a
    return a.reshape(a.shape[0], a.shape[1], -1)


def close(name, got, ref, bound):
    off = np.abs(got - ref)
    bad = ~(off <= bound)  # not a number is bad too
    if bad.any():
        i = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} elements, first {i}: "
                             f"{got[i]!r}, expected {ref[i]!r} within {bound[i]:.3e}")


def check_elements(grid, batch, channels, groups, dt, act, last, residual=False, seed=0,
                   eps=1e-5, g_out=None, spread=1.0):
    """Forward and backward into buffers that hold NaN, with inputs of ordinary
    size (x times `spread`; g_out: a constant in place of noise)."""
    from tests.test_gpu_norm import ACT, DT, _inputs
    say(f"norm elements grid={grid} B={batch} C={channels} G={groups} {dt} {act} last={last} "
        f"spread={spread}")
    op = GroupNormAct(grid, batch, channels, groups, DT[dt], ACT[act], last, eps)
    x, ga, be, g, res = _inputs(seed, grid, batch, channels, dt, last)
    if g_out is not None:
        g.fill_(g_out)
    if spread != 1.0:
        x = (x.float() * spread).to(x.dtype)
    nan = float("nan")
    f32 = dict(dtype=torch.float32, device="cuda")
    out, gx = torch.full_like(x, nan), torch.full_like(x, nan)
    stats = torch.full((batch, groups, 2), nan, **f32)
    gg, gb = torch.full((channels,), nan, **f32), torch.full((channels,), nan, **f32)
    op.fwd(x, ga, be, residual=res if residual else None, out=out, stats=stats)
    op.bwd(x, g, stats, ga, be, gx=gx, g_gamma=gg, g_beta=gb)
    par = [t.double().cpu().numpy() for t in (ga, be)]
    want = reference(rows(x, last), *par, groups, eps, act, rows(g, last),
                     rows(res, last) if residual else None, dt)
    for name, got in (("out", rows(out, last)), ("gx", rows(gx, last)),
                      ("g_gamma", gg.double().cpu().numpy()), ("g_beta", gb.double().cpu().numpy())):
        close(name, got, *want[name])
