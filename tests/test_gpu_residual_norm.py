"""The norms around a block on the GPU, through the layer wrapper, every element
against the float64 oracle within the bounds derived in rownorm_bounds."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from oracle import channel_oracle as C  # noqa: E402
from tests import rownorm_bounds as RB  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.layer import ResidualNorm  # noqa: E402

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
KIND = {"layer": B.FNO_ROW_NORM_LAYER, "rms": B.FNO_ROW_NORM_RMS}
EPS = 1e-5


def _f64(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(rows, c, dt, gates, gate_dt, params, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    row = lambda: ((r(rows, c) + r(c)) * spread).to(DT[dt])  # noqa: E731
    p = {k: 1 + 0.2 * r(c) if params else None for k in ("post_w", "scale", "pre_w")}
    p.update({k: 0.2 * r(c) if params else None for k in ("post_b", "pre_b")})
    p["gate"] = (0.5 + 0.5 * r(gates, c)).to(DT[gate_dt]) if gates else None
    return row(), row(), p, (0.3 * r(rows, c)).to(DT[dt]), r(rows, c).to(DT[dt])


def _check(rows, c, dt, kind="layer", form="both", gates=0, gate_dt="fp32", params=True, seed=0,
           spread=1.0, eps=EPS, with_g_y=True):
    say(f"residual norm {rows}x{c} {dt} {kind} {form} gates={gates} {gate_dt} params={params} "
        f"spread={spread} eps={eps}")
    op = ResidualNorm(rows, c, DT[dt], KIND[kind], eps)
    x, u, p, gy, gh = _inputs(rows, c, dt, gates, gate_dt, params, seed, spread)
    if form == "entry":
        u = None
        for k in ("post_w", "post_b", "gate", "scale"):
            p[k] = None
    if form == "exit":
        gh = p["pre_w"] = p["pre_b"] = None
    nan = float("nan")
    y0 = torch.full_like(x, nan) if u is not None else None
    h0 = torch.full_like(x, nan) if form != "exit" else None
    y, h = op.fwd(x, u, pre=form != "exit", y=y0, h=h0, **p)
    n = {k: _f64(v) for k, v in p.items()}
    want = RB.forward(_f64(x), _f64(u), n, kind, eps, dt)
    if u is not None:
        RB.close("y", _f64(y), *want["y"])
    else:
        assert y is x
    if h is not None:
        RB.close("h", _f64(h), *want["h"])
    out = {"g_x": torch.full_like(x, nan)}
    out.update({"g_" + k: torch.full_like(v, nan) for k, v in p.items() if v is not None})
    got = op.bwd(gy if with_g_y else None, gh, x=x, u=u, y=y, out=dict(out), **p)
    assert all(got[k] is v for k, v in out.items())
    want = RB.backward(_f64(x), _f64(u), _f64(y), n, kind, eps, _f64(gy) if with_g_y else None,
                       _f64(gh), dt, gate_dt)
    for k, v in got.items():
        if v is not None:
            RB.close(k, _f64(v), *want[k])
    assert set(k for k, v in got.items() if v is not None) == \
        {"g_x"} | ({"g_u"} if u is not None else set()) | {"g_" + k for k, v in p.items() if v is not None}
    return op, x, u, p, gy, gh, y, h, got


# channels at each team's edges: vectors of 8 (16-bit) or 4 (fp32) values
@pytest.mark.parametrize("c", [1, 3, 8, 20, 31, 32, 33, 64, 100, 129, 255, 256, 257, 511, 520,
                               1023, 1030, 2048, 2056, 4096, 4099, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
def test_channels(c, dt):
    _check(37 if c < 2048 else 5, c, dt, seed=c)


@pytest.mark.parametrize("form", ["both", "entry", "exit"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gates,gate_dt", [(0, "fp32"), (1, "fp32"), (6, "fp32"), (6, "fp16"),
                                           (96, "fp16"), (96, "fp32"), (1, "fp16"), (48, "fp32")])
def test_forms_and_gates(form, kind, gates, gate_dt):
    if form == "entry" and gates:
        pytest.skip("no gate without u")
    for c in (40, 333):
        _check(96, c, "fp16", kind, form, gates, gate_dt, seed=gates)


@pytest.mark.parametrize("form", ["both", "entry", "exit"])
@pytest.mark.parametrize("params", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 7, 1000])
def test_rows_and_missing_parameters(form, params, rows):
    _check(rows, 24, "bf16", "rms", form, 0, params=params, seed=rows)


def test_gradient_of_the_second_norm_alone():
    _check(50, 72, "fp16", with_g_y=False)


@pytest.mark.parametrize("rows,c,gates", [(70001, 16, 1), (20000, 64, 4), (3000, 512, 3),
                                          (40000, 20, 20000), (1500, 2048, 1)])
def test_many_rows(rows, c, gates):
    """Units of up to 128 rows for a thread, samples that end inside a unit."""
    _check(rows, c, "fp32", "layer", "both", gates, seed=rows)


@pytest.mark.parametrize("dt,spread", [("fp32", 2.0 ** 124 / 8), ("bf16", 2.0 ** 124 / 8),
                                       ("fp16", 8000.0), ("fp32", 2.0 ** 61)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("c", [40, 3000])
def test_rows_as_large_as_the_type(dt, spread, kind, c):
    """Squares past fp32: the entry form (a gradient of size 1 / spread leaves
    16-bit types, so g_y carries the backward)."""
    _check(9, c, dt, kind, "entry", params=False, spread=spread)


@pytest.mark.parametrize("spread", [2.0 ** -60, 2.0 ** -40, 2.0 ** -20])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("c", [40, 3000])
def test_small_rows_without_eps(spread, kind, c):
    _check(9, c, "fp32", kind, "entry", spread=spread, eps=0.0)


def test_rows_that_are_not_finite_stay_alone():
    rows, c = 40, 200
    for kind in ("layer", "rms"):
        op = ResidualNorm(rows, c, torch.float16, KIND[kind], EPS)
        x, u, p, gy, gh = _inputs(rows, c, "fp16", 0, "fp32", True)
        clean = op.fwd(x, u, **p)
        gclean = op.bwd(gy, gh, x=x, u=u, y=clean[0], **p)
        u2, x2 = u.clone(), x.clone()
        u2[3, 7], u2[11, 0], x2[20, 199] = float("inf"), float("nan"), float("-inf")
        y, h = op.fwd(x2, u2, **p)
        ok = torch.ones(rows, dtype=torch.bool)
        ok[[3, 11, 20]] = False
        assert torch.equal(y[ok], clean[0][ok]) and torch.equal(h[ok], clean[1][ok])
        assert y[[3, 11]].isnan().all() and h[[3, 11, 20]].isnan().all()
        got = op.bwd(gy, gh, x=x2, u=u2, y=y, **p)
        for k in ("g_x", "g_u"):
            assert torch.equal(got[k][ok], gclean[k][ok])
        assert got["g_u"][[3, 11]].isnan().all() and got["g_x"][[3, 11, 20]].isnan().all()


def test_in_place_and_bit_identical_runs():
    op, x, u, p, gy, gh, y, h, got = _check(333, 96, "fp16", gates=3)
    x2, u2 = x.clone(), u.clone()
    y2, h2 = op.fwd(x2, u2, y=x2, h=u2, **p)
    assert y2 is x2 and h2 is u2 and torch.equal(y2, y) and torch.equal(h2, h)
    u2, gy2 = u.clone(), gy.clone()
    again = op.bwd(gy2, gh, x=x, u=u2, y=y, out={"g_x": gy2, "g_u": u2}, **p)
    for k, v in got.items():
        assert torch.equal(again[k], v), k
    gh2 = gh.clone()
    again = op.bwd(gy, gh2, x=x, u=u, y=y, out={"g_u": gh2}, **p)
    assert torch.equal(again["g_u"], got["g_u"]) and torch.equal(again["g_x"], got["g_x"])


def test_outputs_end_with_the_rows():
    rows, c = 45, 20
    op = ResidualNorm(rows, c, torch.float16)
    x, u, p, gy, gh = _inputs(rows, c, "fp16", 0, "fp32", True)
    big = [torch.full((rows + 8, c), 7.0, dtype=torch.float16, device="cuda") for _ in range(4)]
    part = [t[:rows] for t in big]
    y, _ = op.fwd(x, u, y=part[0], h=part[1], **p)
    op.bwd(gy, gh, x=x, u=u, y=y, out={"g_x": part[2], "g_u": part[3]}, **p)
    for t in big:
        assert bool((t[rows:] == 7).all()) and not bool((t[:rows] == 7).all())


def test_other_stream_and_graph_replays():
    op, x, u, p, gy, gh, y, h, got = _check(700, 64, "bf16", gates=7)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    bufs = {k: torch.zeros_like(v) for k, v in got.items() if v is not None}
    y2, h2 = torch.zeros_like(x), torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    op2 = ResidualNorm(700, 64, torch.bfloat16)
    op2.fwd(x, u, y=y2, h=h2, stream=s.cuda_stream, **p)
    op2.bwd(gy, gh, x=x, u=u, y=y2, out=dict(bufs), stream=s.cuda_stream, **p)
    s.synchronize()
    assert torch.equal(y2, y) and torch.equal(h2, h)
    for k, v in bufs.items():
        assert torch.equal(v, got[k]), k
    with pytest.raises(ValueError):
        op2.fwd(x, u, stream=s.cuda_stream, **p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op2.fwd(x, u, y=y2, h=h2, **p)
        op2.bwd(gy, gh, x=x, u=u, y=y2, out=dict(bufs), **p)
    for turn in range(3):
        for t in [y2, h2] + list(bufs.values()):
            t.zero_()
        (x.float().sum() + turn).item()  # eager work of its own between replays
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and torch.equal(h2, h)
        for k, v in bufs.items():
            assert torch.equal(v, got[k]), (turn, k)


def test_wrapper_refusals():
    op = ResidualNorm(8, 16, torch.float16)
    x = torch.zeros(8, 16, dtype=torch.float16, device="cuda")
    w = torch.ones(16, device="cuda")
    for bad in (dict(x=None), dict(x=x.float()), dict(x=x[:7]), dict(x=x.t().contiguous().t()),
                dict(x=x.cpu()), dict(x=x, u=x[:, :8]), dict(x=x, u=x, post_w=w[:8]),
                dict(x=x, u=x, post_w=w.half()), dict(x=x, u=x, gate=torch.ones(3, 16, device="cuda")),
                dict(x=x, u=x, gate=torch.ones(2, 16, device="cuda").bfloat16()),
                dict(x=x, u=x, gate=torch.ones(16, device="cuda")), dict(x=x, pre=False),
                dict(x=x, y=x), dict(x=x, u=x, pre=False, h=x)):
        with pytest.raises((ValueError, B.FnoError)):
            op.fwd(**bad)
    for bad in (dict(g_y=x, post_w=w), dict(x=x, pre_w=w, g_y=x)):
        with pytest.raises((ValueError, B.FnoError)):
            op.fwd(x, **{k: v for k, v in bad.items() if k in ("post_w",)}) if "post_w" in bad else op.bwd(**bad)
    for bad in (dict(g_y=None), dict(g_y=x, g_h=x, u=x), dict(g_y=x, u=x, scale=w),
                dict(g_y=x), dict(g_y=x, u=x, out={"g_scale": w}), dict(g_y=x, u=x, out={"g_x": w}),
                dict(g_y=x, u=x, pre_w=w), dict(g_y=x, g_h=x, x=x, out={"g_u": x})):
        with pytest.raises((ValueError, B.FnoError)):
            op.bwd(**bad)
    for kw in (dict(rows=0, channels=4), dict(rows=4, channels=0), dict(rows=4, channels=16385),
               dict(rows=4, channels=4, eps=-1.0), dict(rows=4, channels=4, norm=2)):
        with pytest.raises(B.FnoError):
            ResidualNorm(**kw)
    with pytest.raises(ValueError):
        ResidualNorm(4, 4, torch.float64)


def test_one_row_with_a_gate():
    for c in (1, 5, 64, 300):
        for dt in ("fp32", "bf16"):
            _check(1, c, dt, gates=1, gate_dt=dt)


def test_rows_past_32_bits():
    """More than 2^31 values; the last rows against the same rows alone."""
    rows, c = (1 << 22) + 37, 520
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(rows, c, dtype=torch.float16, device="cuda").normal_(generator=g)
    u = torch.empty_like(x).normal_(generator=g)
    w = 1 + 0.2 * torch.randn(c, device="cuda", generator=g)
    y, h = ResidualNorm(rows, c).fwd(x, u, post_w=w, scale=w)
    got = ResidualNorm(rows, c).bwd(x, u, x=x, u=u, y=y, post_w=w, scale=w)
    n = 100
    last = [t[-n:].clone() for t in (x, u, y)]
    small = ResidualNorm(n, c)
    y2, h2 = small.fwd(last[0], last[1], post_w=w, scale=w)
    got2 = small.bwd(last[0], last[1], x=last[0], u=last[1], y=last[2], post_w=w, scale=w)
    assert torch.equal(y[-n:], y2) and torch.equal(h[-n:], h2)
    assert torch.equal(got["g_x"][-n:], got2["g_x"]) and torch.equal(got["g_u"][-n:], got2["g_u"])
    # the parameters' sums against torch's own, in pieces
    want = sum(((got["g_x"][i:i + (1 << 18)].double() / w.double()) * x[i:i + (1 << 18)].double()).sum(0)
               for i in range(0, rows, 1 << 18))
    size = sum(((got["g_x"][i:i + (1 << 18)].double() / w.double()) * x[i:i + (1 << 18)].double()).abs().sum(0)
               for i in range(0, rows, 1 << 18))
    # g_x is rounded to fp16 (2^-11 of each term, of either sign): far within 2^-11 of the sum of sizes
    assert bool(((got["g_scale"].double() - want).abs() <= 2.0 ** -11 * size).all())
