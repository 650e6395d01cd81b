"""The norms around a block where rows end inside a vector or a gate's share inside a
work-group, and rows as large as fp32; bounds as in test_gpu_residual_norm."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests import rownorm_bounds as RB  # noqa: E402
from tests import test_gpu_residual_norm as R  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd.layer import ResidualNorm  # noqa: E402


@pytest.mark.parametrize("c", [3, 20, 333, 1030, 2050, 4099, 8203, 16381])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_in_place_with_a_short_last_vector(c, dt, kind):
    """A row's last vector is read from the one before it, which another thread (of
    another wave, in large teams) overwrites."""
    rows = 301 if c < 1000 else 150
    gates = rows // 7 if rows % 7 == 0 else rows // 10 if rows % 10 == 0 else 1
    say(f"residual norm in place {rows}x{c} {dt} {kind}")
    op = ResidualNorm(rows, c, R.DT[dt], R.KIND[kind])
    x, u, p, gy, gh = R._inputs(rows, c, dt, gates, "fp32", True, seed=c)
    y, h = op.fwd(x, u, **p)
    want = op.bwd(gy, gh, x=x, u=u, y=y, **p)
    post = {k: v for k, v in p.items() if not k.startswith("pre")}
    y_only, _ = op.fwd(x, u, pre=False, **post)
    for turn in range(3):
        x2, u2 = x.clone(), u.clone()
        op.fwd(x2, u2, y=x2, h=u2, **p)
        assert torch.equal(x2, y) and torch.equal(u2, h), turn
        x2, u2 = x.clone(), u.clone()
        _, h2 = op.fwd(x2, u2, y=u2, **p)
        assert torch.equal(u2, y) and torch.equal(h2, h) and torch.equal(x2, x), turn
        for into in (0, 1):
            x2, u2 = x.clone(), u.clone()
            op.fwd(x2, u2, pre=False, y=(x2, u2)[into], **post)
            assert torch.equal((x2, u2)[into], y_only), turn
        for a, b in (("gy", "u"), ("gy", "gh"), ("gh", "u")):
            t = dict(gy=gy.clone(), gh=gh.clone(), u=u.clone())
            got = op.bwd(t["gy"], t["gh"], x=x, u=t["u"], y=y, out={"g_x": t[a], "g_u": t[b]}, **p)
            for k, v in want.items():
                assert torch.equal(got[k], v), (turn, a, b, k)


@pytest.mark.parametrize("c", [20, 64, 333, 520, 4096])
@pytest.mark.parametrize("each", [2, 3, 5])
@pytest.mark.parametrize("gate_dt", ["fp32", "bf16"])
def test_gates_of_a_few_rows(c, each, gate_dt):
    """Gate rows that serve fewer rows than a work-group holds."""
    R._check(60, c, "bf16", "layer", "both", 60 // each, gate_dt, seed=each)
    R._check(60, c, "bf16", "rms", "exit", 60 // each, gate_dt, seed=each)


@pytest.mark.parametrize("c,each", [(3, 2), (20, 3), (20, 5), (64, 2), (64, 8), (64, 20), (333, 3), (333, 2), (520, 5),
                                    (520, 16), (2050, 7), (4096, 2), (4099, 3), (8192, 2), (16380, 2)])
@pytest.mark.parametrize("dt,gate_dt", [("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")])
def test_many_gates_of_a_few_rows(c, each, dt, gate_dt):
    """So many that teams take whole gate rows (4096 values of the gate for each of its
    rows), and a few more, so that the last unit is not full; in place too."""
    gates = -(-4096 * each // c) + 5
    op, x, u, p, gy, gh, y, h, got = R._check(gates * each, c, dt, "layer", "both", gates, gate_dt, seed=each)
    u2, gy2, x2, u3 = u.clone(), gy.clone(), x.clone(), u.clone()
    again = op.bwd(gy2, gh, x=x, u=u2, y=y, out={"g_x": gy2, "g_u": u2}, **p)
    assert all(torch.equal(again[k], v) for k, v in got.items())
    op.fwd(x2, u3, y=x2, h=u3, **p)
    assert torch.equal(x2, y) and torch.equal(u3, h)
    R._check(gates * each, c, dt, "rms", "exit", gates, gate_dt, seed=each)


@pytest.mark.parametrize("c,each", [(64, 128), (64, 100), (520, 127), (4096, 65)])
def test_gates_of_up_to_128_rows_against_a_gate_a_row(c, each):
    """The longest runs that a team takes: rows and their gradients are those of the
    same gate given for each row, bit for bit, and the gate's gradient is the sum of
    its rows' (chains of up to 128 fp32 additions), which end where the next begins."""
    gates = -(-4096 * each // c) + 3
    rows = gates * each
    say(f"residual norm {rows}x{c}, gates of {each} rows")
    g = torch.Generator(device="cuda").manual_seed(each)
    row = lambda: torch.randn(rows, c, device="cuda", generator=g).half()  # noqa: E731
    x, u, gy, gh = row(), row(), row(), row()
    w = 1 + 0.2 * torch.randn(c, device="cuda", generator=g)
    gate = torch.randn(gates, c, device="cuda", generator=g)
    op = ResidualNorm(rows, c)
    p = dict(post_w=w, scale=w, pre_w=w)
    y, h = op.fwd(x, u, gate=gate, **p)
    got = op.bwd(gy, gh, x=x, u=u, y=y, gate=gate, **p)
    alone = gate.repeat_interleave(each, 0)
    y2, h2 = op.fwd(x, u, gate=alone, **p)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    want = op.bwd(gy, gh, x=x, u=u, y=y, gate=alone, **p)
    assert torch.equal(got["g_x"], want["g_x"]) and torch.equal(got["g_u"], want["g_u"])
    for a in range(0, gates, 1024):
        terms = want["g_gate"][a * each:(a + 1024) * each].double().view(-1, each, c)
        off = (got["g_gate"][a:a + 1024].double() - terms.sum(1)).abs()
        assert bool((off <= each * 2.0 ** -24 * terms.abs().sum(1)).all())
    # either order: chains of up to 128, a tree, doubles, of terms whose sizes are below 4 in the mean
    for k in ("g_post_w", "g_scale", "g_pre_w"):
        assert bool(((got[k] - want[k]).abs() <= 2 * RB.CHAIN * RB.E * rows * 4).all()), k


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("c", [40, 3000])
@pytest.mark.parametrize("size", [2.0 ** 126.5, 3.0e38])
def test_rows_up_to_the_types_largest(dt, kind, c, size):
    """Values beyond 2^126: 1 / deviation is a subnormal fp32 number, half a step of
    which is at most 2^-22 of it, within the bounds' (D + 6) 2^-24."""
    rows = 9
    say(f"residual norm {rows}x{c} {dt} {kind} of {size}")
    g = torch.Generator(device="cuda").manual_seed(c)
    r = lambda: torch.rand(rows, c, device="cuda", generator=g) * 2 - 1  # noqa: E731
    x = (r() * size).to(R.DT[dt])
    gy, gh = r().to(R.DT[dt]), r().to(R.DT[dt])
    assert bool(x.isfinite().all())
    op = ResidualNorm(rows, c, R.DT[dt], R.KIND[kind])
    _, h = op.fwd(x)
    n = dict.fromkeys(op.PARAMS)
    RB.close("h", R._f64(h), *RB.forward(R._f64(x), None, n, kind, 1e-5, dt)["h"])
    got = op.bwd(gy, gh, x=x)
    want = RB.backward(R._f64(x), None, None, n, kind, 1e-5, R._f64(gy), R._f64(gh), dt)
    RB.close("g_x", R._f64(got["g_x"]), *want["g_x"])


def test_rows_whose_distances_from_the_mean_pass_fp32_are_not_a_number():
    """LAYER alone: values are finite, a distance is not.  The row is NaN throughout,
    and alone."""
    rows, c = 12, 200
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, c, device="cuda", generator=g)
    x[4] = 3e38
    x[4, 7] = -3e38
    gy, gh = torch.ones_like(x), torch.ones_like(x)
    keep = torch.arange(rows, device="cuda") != 4
    for kind in ("layer", "rms"):
        op = ResidualNorm(rows, c, torch.float32, R.KIND[kind])
        _, h = op.fwd(x)
        gx = op.bwd(gy, gh, x=x)["g_x"]
        assert bool(h[keep].isfinite().all()) and bool(gx[keep].isfinite().all())
        assert bool(h[4].isnan().all() if kind == "layer" else h[4].isfinite().all())
        assert bool(gx[4].isnan().all() if kind == "layer" else gx[4].isfinite().all())
