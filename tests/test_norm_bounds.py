"""The elementwise bounds of the group norm's tests, on the CPU: rounded exact
results pass; one element that is off, missing, or from a mistaken formula does
not."""
import numpy as np
import pytest

pytest.importorskip("torch")

from oracle import train_oracle as T  # noqa: E402
from tests import norm_bounds as N  # noqa: E402

TYPES = {"fp16": np.float16, "fp32": np.float32}


def _case(dt, kind, p=2000):
    r = np.random.default_rng(11)
    f = TYPES[dt]
    x = (r.standard_normal((2, 12, p)) + r.standard_normal((1, 12, 1))).astype(f).astype(float)
    g, res = (r.standard_normal(x.shape).astype(f).astype(float) for _ in range(2))
    ga, be = 1 + 0.2 * r.standard_normal(12), 0.3 * r.standard_normal(12)
    return x, ga, be, g, res, N.reference(x, ga, be, 3, 1e-5, kind, g, res, dt)


@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
@pytest.mark.parametrize("dt", ["fp16", "fp32"])
def test_bounds(dt, kind):
    x, ga, be, g, res, want = _case(dt, kind)
    for name, (v, b) in want.items():
        f = TYPES[dt] if name in ("out", "gx") else np.float32
        got = v.astype(f).astype(float)
        N.close(name, got, v, b)
        at = tuple(s - 1 for s in v.shape)  # the last element
        for wrong in (got[at] + 4 * b[at], np.nan, np.inf):
            bad = got.copy()
            bad[at] = wrong
            with pytest.raises(AssertionError, match=name):
                N.close(name, bad, v, b)


@pytest.mark.parametrize("dt", ["fp16", "fp32"])
def test_mistaken_formulas_are_seen(dt):
    """The last element of a plane left out of the sums; another channel's value
    in one place."""
    x, ga, be, g, res, want = _case(dt, "gelu")
    short = T.group_norm_act_fwd(x[:, :, :-1], ga, be, 3, 1e-5, "gelu", res[:, :, :-1])[0]
    with pytest.raises(AssertionError, match="out"):
        N.close("out", short, *(t[:, :, :-1] for t in want["out"]))
    _, _, gb = T.group_norm_act_bwd(x[:, :, :-1], ga, be, 3, 1e-5, "gelu", g[:, :, :-1])[:3]
    with pytest.raises(AssertionError, match="g_beta"):
        N.close("g_beta", gb, *want["g_beta"])
    shifted = T.group_norm_act_fwd(np.roll(x, 4, 1), np.roll(ga, 4), np.roll(be, 4), 3, 1e-5,
                                   "gelu")[0]
    mixed = want["out"][0].copy()
    mixed[0, 3, 5] = shifted[0, 3, 5]
    with pytest.raises(AssertionError, match="1 of"):
        N.close("out", mixed, *want["out"])
