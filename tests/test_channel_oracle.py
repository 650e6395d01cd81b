"""The oracle of the operators over channels against differences, torch's own
types and brute force (no GPU needed)."""
import numpy as np
import pytest

from oracle import channel_oracle as C
from tests import rownorm_bounds as RB

torch = pytest.importorskip("torch")


def _case(rows, c, gates, seed=0):
    g = np.random.default_rng(seed)
    p = {k: 1 + 0.3 * g.standard_normal(c) for k in ("post_w", "scale", "pre_w")}
    p.update({k: 0.3 * g.standard_normal(c) for k in ("post_b", "pre_b")})
    p["gate"] = g.standard_normal((gates, c)) if gates else None
    return [g.standard_normal((rows, c)) + 0.5 for _ in range(4)], p


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,c,gates", [(1, 1, 0), (6, 5, 1), (6, 7, 3), (4, 6, 4), (6, 3, 0)])
def test_residual_norm_gradients_against_differences(kind, rows, c, gates):
    (x, u, gy, gh), p = _case(rows, c, gates)

    def loss():
        y, h = C.residual_norm_fwd(x, u, p, kind, 1e-3)
        return (y * gy).sum() + (h * gh).sum()

    y = C.residual_norm_fwd(x, u, p, kind, 1e-3)[0]
    got = C.residual_norm_bwd(x, u, y, p, kind, 1e-3, gy, gh)
    step = 1e-5
    for name, a in [("g_x", x), ("g_u", u)] + [("g_" + k, v) for k, v in p.items() if v is not None]:
        for i in np.ndindex(a.shape):
            old = a[i]
            a[i] = old + step
            up = loss()
            a[i] = old - step
            down = loss()
            a[i] = old
            # differences: step^2 times the third derivative, and the loss's rounding over the step
            assert abs(got[name][i] - (up - down) / (2 * step)) <= 1e-5 * (1 + abs(got[name][i])), (name, i)


def test_bounds_catch_a_planted_mistake():
    """The bounds are far below what a wrong formula changes: a mean over one
    channel too many, a gate of the neighbouring sample, a missing term."""
    (x, u, gy, gh), p = _case(24, 40, 4)
    y = C.residual_norm_fwd(x, u, p, "layer", 1e-5)[0]
    want = RB.backward(x, u, y, p, "layer", 1e-5, gy, gh, "fp32")
    for name, (v, b) in want.items():
        RB.close(name, v, v, b)
    wrong = dict(p, gate=np.roll(p["gate"], 1, 0))
    for change in (dict(p=wrong), dict(kind="rms"), dict(g_y=0 * gy)):
        a = dict(x=x, u=u, y=y, p=p, kind="layer", eps=1e-5, g_y=gy, g_h=gh)
        a.update(change)
        got = C.residual_norm_bwd(**a)
        with pytest.raises(AssertionError):
            RB.close("g_u", got["g_u"], *want["g_u"])
    fwd = RB.forward(x, u, p, "layer", 1e-5, "bf16")
    with pytest.raises(AssertionError):
        RB.close("h", C.residual_norm_fwd(x, u, p, "rms", 1e-5)[1], *fwd["h"])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_codes_are_the_types_own(fmt):
    dt = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    table = C.decode_table(fmt)
    own = torch.arange(256, dtype=torch.uint8).view(dt).double().numpy()
    assert np.array_equal(table, own, equal_nan=True)
    g = np.random.default_rng(1)
    top = C.FORMATS[fmt][0]
    v = (g.standard_normal(20000) * np.exp(g.uniform(-14, 5, 20000))).astype(np.float32)
    fin = np.sort(table[np.isfinite(table)])
    v = np.concatenate([v, fin, (fin[1:] + fin[:-1]) / 2, [0.0, -0.0, np.nan]]).astype(np.float32)
    v = np.clip(v, -top, top)
    assert np.array_equal(C.round8(v.astype(np.float64), fmt),
                          torch.from_numpy(v).to(dt).double().numpy(), equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize_keeps_values(fmt, kind, tile):
    """Within half a step of the format at the block's size; the largest code is
    within the format and, with power of two scales, over half of its largest."""
    g = np.random.default_rng(2)
    v = g.standard_normal((131, 259)) * np.exp(g.uniform(-20, 20, (131, 1)))
    v[5] = 0
    v[7, :128] = 0
    q, s = C.quantize(v, fmt, kind, tile)
    top, bits, low = C.FORMATS[fmt]
    assert np.abs(q).max() <= top and s.shape == (3, 2 if tile else 131)
    back = C.values(q, s, tile)
    scale = np.abs(C.values(np.ones_like(q), s, tile))
    assert np.all(np.abs(back - v) <= 2.0 ** -(bits + 1) * np.abs(v) * 1.000001 + scale * 2.0 ** (low - bits - 1) * 1.000001)
    if kind == "pow2":
        assert np.array_equal(np.frexp(s)[0], np.full(s.shape, 0.5))
    if not tile:
        big = np.abs(q[:, :128]).max(1)
        assert np.all((big > top / 2 * 0.99) | (big == 0))


def test_quantize_of_values_that_are_not_finite():
    v = np.ones((2, 130))
    v[0, 3], v[0, 4], v[1, 129] = np.inf, np.nan, -np.inf
    q, s = C.quantize(v, "e4m3", "pow2")
    assert np.isnan(q[0, 3]) and np.isnan(q[0, 4]) and np.isnan(q[1, 129])
    assert q[0, 5] == 256 and s[0, 0] == 2.0 ** -8 and q[1, 0] == 256
    q, _ = C.quantize(v, "e5m2", "f32")
    assert q[0, 3] == np.inf and np.isnan(q[0, 4]) and q[1, 129] == -np.inf
