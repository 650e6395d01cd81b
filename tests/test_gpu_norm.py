"""Group norm with an activation on the GPU, through the layer wrapper and the
C ABI, against the float64 oracle.

Tolerances.  A stored result carries one rounding of its type: relative error
u = 2^-11 (fp16), 2^-8 (bf16), 2^-24 (fp32).  The fp32 arithmetic before it
works on terms of the size that the formula has (|z| for the output; the
oracle's `scale`, rstd gamma h, for gx, whose difference may cancel; the sum of
absolute terms for the parameter gradients), each with a few dozen roundings
of 2^-24, times |mean| / sigma <= 12 where x - mean cancels: 1e-5 of those
terms covers it.  Norms are taken over whole tensors and over the worst
(sample, channel) row.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from oracle import train_oracle as T  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.layer import GroupNormAct  # noqa: E402

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
ACT = {"none": B.FNO_NORM_ACT_NONE, "gelu": B.FNO_NORM_ACT_GELU, "silu": B.FNO_NORM_ACT_SILU}
EPS = 1e-5


def _close(name, got, ref, u, scale=None):
    """|got - ref| <= u |ref| + 1e-5 (|ref| + |scale|) in the 2-norm, over the
    whole tensor and over each row of its last axis."""
    got = np.asarray(got, np.float64)
    scale = ref if scale is None else scale
    for axis in (None, -1):
        n = [np.sqrt((np.asarray(t, np.float64) ** 2).sum(axis)) for t in (got - ref, ref, scale)]
        over = n[0] - (u * n[1] + 1e-5 * (n[1] + n[2]) + 1e-12)
        assert np.all(np.isfinite(n[0])) and np.all(over <= 0), (
            f"{name}: off by {np.max(n[0]):.3e}, norm {np.max(n[1]):.3e}")


def _rows(t, last):
    a = t.float().cpu().numpy().astype(np.float64)
    a = np.moveaxis(a, -1, 1) if last else a
    return a.reshape(a.shape[0], a.shape[1], -1)


def _inputs(seed, grid, batch, c, dt, last, offset=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    shape = (batch,) + (grid + (c,) if last else (c,) + grid)
    per = (c,) if last else (c,) + (1,) * len(grid)
    x = (r(*shape) * (0.5 + torch.rand(c, device="cuda", generator=g)).view(per)
         + offset * r(c).view(per)).to(DT[dt])
    return x, 1 + 0.2 * r(c), 0.3 * r(c), r(*shape).to(DT[dt]), r(*shape).to(DT[dt])


def _check(grid, batch, c, groups, dt, act, last, residual=False, offset=1.0, seed=0):
    say(f"norm grid={grid} B={batch} C={c} G={groups} {dt} {act} last={last} res={residual}")
    op = GroupNormAct(grid, batch, c, groups, DT[dt], ACT[act], last, EPS)
    x, ga, be, g, res = _inputs(seed, grid, batch, c, dt, last, offset)
    out, stats = op.fwd(x, ga, be, residual=res if residual else None)
    gx, gg, gb = op.bwd(x, g, stats, ga, be)
    torch.cuda.synchronize()
    xr, gr = _rows(x, last), _rows(g, last)
    gan, ben = (t.cpu().numpy().astype(np.float64) for t in (ga, be))
    ro, rs = T.group_norm_act_fwd(xr, gan, ben, groups, EPS, act,
                                  _rows(res, last) if residual else None)
    _close("out", _rows(out, last), ro, U[dt])
    # mean: the input's own size; rstd: 1e-5 of itself
    size = np.sqrt(np.mean(xr ** 2)) + np.abs(rs[..., 0])
    st = stats.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(st[..., 0] - rs[..., 0]) <= 1e-6 * size)
    assert np.all(np.abs(st[..., 1] - rs[..., 1]) <= 1e-5 * rs[..., 1])
    rx, rg, rb, scale, ag, ab = T.group_norm_act_bwd(xr, gan, ben, groups, EPS, act, gr)
    _close("gx", _rows(gx, last), rx, U[dt], scale)
    assert np.all(np.abs(gg.cpu().numpy() - rg) <= 1e-5 * ag + 1e-12), "g_gamma"
    assert np.all(np.abs(gb.cpu().numpy() - rb) <= 1e-5 * ab + 1e-12), "g_beta"
    return op, x, ga, be, g, out, stats, gx, gg, gb


SHAPES = [
    # (grid, batch, channels, groups)
    ((1,), 1, 1, 1),            # one value: the variance is zero
    ((1,), 3, 8, 2),            # one point
    ((1,), 2, 33, 33),          # one point per group
    ((2,), 2, 6, 3),
    ((7,), 2, 3, 1),
    ((63,), 3, 16, 4),
    ((64, 64), 2, 16, 4),       # the smallest workload
    ((15, 17), 3, 20, 4),       # rows of 40 bytes, odd planes
    ((9, 31), 2, 33, 11),       # odd channels
    ((35, 35), 4, 128, 32),
    ((257,), 2, 130, 13),
    ((5, 6, 7), 3, 48, 6),      # 3-D
    ((40, 40), 2, 64, 1),       # one group per sample
    ((24, 24), 2, 64, 64),      # one channel per group
    ((3,), 2, 2056, 257),       # more channels than a work-group has pieces
    ((5,), 1, 1025, 5),         # odd and many channels
    ((4099,), 3, 5, 1),
    ((128, 128), 5, 8, 2),      # long planes, few channels
    ((70000,), 1, 4, 2),        # several pieces of a plane
    ((1000,), 40, 12, 3),       # more samples than a chunk has
]


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_shapes(case, dt, last):
    grid, b, c, g = SHAPES[case]
    act = ("gelu", "silu", "none")[(case + len(dt) + last) % 3]
    _check(grid, b, c, g, dt, act, last, residual=case % 2 == 0, seed=case)


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("residual", [False, True])
def test_activations(act, residual, last):
    _check((37, 21), 3, 24, 6, "fp32", act, last, residual, seed=50)
    _check((37, 21), 3, 24, 6, "fp16", act, last, residual, seed=51)


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
def test_workload_sizes(last):
    """The Navier-Stokes workload's tensor (four samples of it), several
    chunks per sample and more groups of work than the chip holds."""
    _check((128, 128), 4, 64, 8, "fp16", "gelu", last, True, seed=60)
    _check((64, 64, 64), 1, 32, 1, "fp32", "silu", last, seed=61)
    _check((241, 241), 2, 20, 4, "fp16", "gelu", last, seed=62)


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
@pytest.mark.parametrize("dt", ["fp32", "fp16"])
def test_offset_and_outliers(dt, last):
    """A mean far from zero (sums of squares would cancel), and a first value
    far from all others (a shift by it would cancel)."""
    grid, b, c, groups = (61, 50), 2, 16, 4
    op = GroupNormAct(grid, b, c, groups, DT[dt], ACT["none"], last, EPS)
    x, ga, be, _, _ = _inputs(70, grid, b, c, dt, last, 0.0)
    for kind in ("offset", "outlier"):
        y = x.clone()
        if kind == "offset":
            y = (x.float() * 0.25 + 300.0).to(DT[dt])
        else:
            y.view(-1)[:3] = 3000.0
        out, stats = op.fwd(y, ga, be)
        ro, rs = T.group_norm_act_fwd(_rows(y, last), ga.cpu().numpy(), be.cpu().numpy(), groups,
                                      EPS, "none")
        st = stats.cpu().numpy()
        # the mean is stored in fp32: 2^-24 |mean| of error in x - mean
        ratio = np.max(np.abs(rs[..., 0]) * rs[..., 1])
        assert np.all(np.abs(st[..., 0] - rs[..., 0]) <= 2.0 ** -23 * np.abs(rs[..., 0]) + 1e-6)
        assert np.all(np.abs(st[..., 1] - rs[..., 1]) <= 2e-5 * rs[..., 1]), kind
        _close(kind, _rows(out, last), ro, U[dt] + 3 * ratio * 2.0 ** -24)


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
def test_constant_group_gives_beta(last):
    """Variance zero: xh is 0, the output act(beta), no infinities."""
    op = GroupNormAct((20, 20), 2, 8, 2, torch.float16, ACT["gelu"], last, EPS)
    x = torch.full(op.shape, 3.0, dtype=torch.float16, device="cuda")
    be = torch.linspace(-2, 2, 8, device="cuda")
    out, stats = op.fwd(x, None, be)
    ref = torch.nn.functional.gelu(be.double()).cpu().numpy()
    got = _rows(out, last)
    assert np.all(np.abs(got - ref[None, :, None]) <= 2.0 ** -11 * np.abs(ref)[None, :, None] + 1e-6)
    assert np.allclose(stats[..., 1].cpu().numpy(), 1 / np.sqrt(EPS), rtol=1e-6)
    gx, _, gb = op.bwd(x, torch.ones_like(x), stats, None, be)
    # within a group: gx = rstd (h - mean h), h = act'(beta), the same for every sample
    assert torch.isfinite(gx).all() and torch.isfinite(gb).all()


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_stays_in_its_group(bad, last):
    grid, b, c, groups = (33, 31), 3, 16, 4
    op = GroupNormAct(grid, b, c, groups, torch.float16, ACT["gelu"], last, EPS)
    x, ga, be, g, _ = _inputs(80, grid, b, c, "fp16", last)
    clean, st0 = op.fwd(x, ga, be)
    gx0, _, _ = op.bwd(x, g, st0, ga, be)
    if last:
        x[1, 5, 6, 9] = bad
    else:
        x[1, 9, 5, 6] = bad
    out, st = op.fwd(x, ga, be)
    gx, gg, gb = op.bwd(x, g, st, ga, be)
    for got, ref in ((out, clean), (gx, gx0)):
        got, ref = _rows(got, last), _rows(ref, last)
        assert np.isnan(got[1, 8:12]).all()
        got[1, 8:12] = ref[1, 8:12] = 0
        assert np.array_equal(got, ref)
    assert torch.isnan(gg[8:12]).all() and torch.isfinite(gg[:8]).all()
    assert torch.isfinite(gg[12:]).all() and torch.isfinite(gb[:8]).all()


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
def test_in_place_inference_and_reruns(last):
    """The same bits: run again, with out on x or on the residual, gx on g_out
    or on x, without statistics kept, into given buffers."""
    grid, b, c, groups = (50, 41), 4, 40, 5
    op = GroupNormAct(grid, b, c, groups, torch.float16, ACT["silu"], last, EPS)
    x, ga, be, g, res = _inputs(90, grid, b, c, "fp16", last)
    out, st = op.fwd(x, ga, be, residual=res)
    gx, gg, gb = op.bwd(x, g, st, ga, be)
    out2, none = op.fwd(x, ga, be, residual=res, keep_stats=False)
    assert none is None and torch.equal(out, out2)
    y = x.clone()
    op.fwd(y, ga, be, residual=res, out=y)
    assert torch.equal(y, out)
    y = res.clone()
    op.fwd(x, ga, be, residual=y, out=y)
    assert torch.equal(y, out)
    for alias in ("g", "x"):
        xx, gg2 = x.clone(), g.clone()
        r = op.bwd(xx, gg2, st, ga, be, gx=gg2 if alias == "g" else xx)
        assert torch.equal(r[0], gx) and torch.equal(r[1], gg) and torch.equal(r[2], gb)


def test_affine_optional():
    op = GroupNormAct((19, 8), 2, 12, 3, torch.float32, ACT["gelu"], True, EPS)
    x, _, _, g, _ = _inputs(91, (19, 8), 2, 12, "fp32", True)
    one, zero = torch.ones(12, device="cuda"), torch.zeros(12, device="cuda")
    a, st = op.fwd(x)
    b, _ = op.fwd(x, one, zero)
    assert torch.equal(a, b)
    for r, s in zip(op.bwd(x, g, st), op.bwd(x, g, st, one, zero)):
        assert torch.equal(r, s)


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
def test_gradient_against_differences(last):
    """Along a random direction of x, gamma and beta, the oracle's loss at the
    fp32 inputs moves by what the GPU's gradients say."""
    grid, b, c, groups = (11, 13), 2, 12, 4
    op = GroupNormAct(grid, b, c, groups, torch.float32, ACT["gelu"], last, EPS)
    x, ga, be, g, _ = _inputs(92, grid, b, c, "fp32", last)
    _, st = op.fwd(x, ga, be)
    gx, gg, gb = op.bwd(x, g, st, ga, be)
    xr, gr = _rows(x, last), _rows(g, last)
    par = [xr, ga.cpu().numpy().astype(np.float64), be.cpu().numpy().astype(np.float64)]
    grads = [_rows(gx, last), gg.cpu().numpy(), gb.cpu().numpy()]
    r, h = np.random.default_rng(1), 1e-5

    def loss(p):
        return (T.group_norm_act_fwd(p[0], p[1], p[2], groups, EPS, "gelu")[0] * gr).sum()

    for i in range(3):
        d = r.standard_normal(par[i].shape)
        up, dn = list(par), list(par)
        up[i], dn[i] = par[i] + h * d, par[i] - h * d
        num = (loss(up) - loss(dn)) / (2 * h)
        # differences: h^2 of the third derivative; the gradient: 1e-5 of its terms
        assert abs(num - (grads[i] * d).sum()) <= 1e-5 * np.sum(np.abs(grads[i] * d)) + 1e-6


def test_offsets_past_32_bits():
    """More than 2^32 elements in both layouts: the last sample as by itself."""
    b, c, n = 5, 64, 3700  # 5 x 64 x 3700^2 = 4.38e9
    for last in (False, True):
        say(f"  {b}x{c}x{n}x{n} last={last}")
        op = GroupNormAct((n, n), b, c, 8, torch.float16, ACT["gelu"], last, EPS)
        one = GroupNormAct((n, n), 1, c, 8, torch.float16, ACT["gelu"], last, EPS)
        x = torch.empty(op.shape, dtype=torch.float16, device="cuda")
        for i in range(b):
            x[i].normal_(0.1 * i, 1.0)
        out, st = op.fwd(x)
        ref, rst = one.fwd(x[-1:].contiguous())
        assert torch.allclose(st[-1:], rst, rtol=1e-5, atol=1e-7)
        assert float((out[-1:] - ref).abs().max()) <= 2.0 ** -9  # one fp16 step below 8
        gx, gg, gb = op.bwd(x, x, st)
        rx, _, _ = one.bwd(x[-1:].contiguous(), x[-1:].contiguous(), rst)
        assert float((gx[-1:].float() - rx.float()).abs().max()) <= 2.0 ** -7
        del x, out, ref, gx, rx
        torch.cuda.empty_cache()


@pytest.mark.parametrize("last", [False, True], ids=["first", "last"])
def test_graph_replays(last):
    """Captured forward and backward, replayed on other inputs with eager work
    between: every replay gives the eager result's bits."""
    grid, b, c, groups = (64, 48), 4, 32, 8
    op = GroupNormAct(grid, b, c, groups, torch.float16, ACT["gelu"], last, EPS)
    x, ga, be, g, _ = _inputs(93, grid, b, c, "fp16", last)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, st = op.fwd(x, ga, be)
        op.bwd(x, g, st, ga, be)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, st = op.fwd(x, ga, be)
        gx, gg, gb = op.bwd(x, g, st, ga, be)
    eager = GroupNormAct(grid, b, c, groups, torch.float16, ACT["gelu"], last, EPS)
    for k in range(4):
        nx, _, _, ng, _ = _inputs(94 + k, grid, b, c, "fp16", last)
        x.copy_(nx)
        g.copy_(ng)
        graph.replay()
        ro, rs = eager.fwd(nx, ga, be)
        rx, rg, rb = eager.bwd(nx, ng, rs, ga, be)
        torch.cuda.synchronize()
        for a, r in ((out, ro), (st, rs), (gx, rx), (gg, rg), (gb, rb)):
            assert torch.equal(a, r), k


def test_another_stream():
    """Given buffers on a stream of the caller's, ordered by it alone."""
    grid, b, c, groups = (128, 128), 8, 32, 4
    op = GroupNormAct(grid, b, c, groups, torch.float16, ACT["gelu"], True, EPS)
    x, ga, be, g, _ = _inputs(99, grid, b, c, "fp16", True)
    ref, rst = op.fwd(x, ga, be)
    out, st = torch.empty_like(ref), torch.empty_like(rst)
    y = torch.zeros_like(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y.copy_(x)
    op.fwd(y, ga, be, out=out, stats=st, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(out, ref) and torch.equal(st, rst)
    with pytest.raises(ValueError, match="required where a stream"):
        op.fwd(x, ga, be, stream=s.cuda_stream)


def test_refusals():
    op = GroupNormAct((8, 8), 2, 16, 4, torch.float16, ACT["gelu"], True, EPS)
    x, ga, be, g, _ = _inputs(100, (8, 8), 2, 16, "fp16", True)
    out, st = op.fwd(x, ga, be)
    with pytest.raises(ValueError, match="dtype"):
        op.fwd(x.float(), ga, be)
    with pytest.raises(ValueError, match="shape"):
        op.fwd(x[:1], ga, be)
    with pytest.raises(ValueError, match="contiguous"):
        op.fwd(x.transpose(1, 2), ga, be)
    with pytest.raises(ValueError, match="gamma"):
        op.fwd(x, ga.half(), be)
    with pytest.raises(ValueError, match="GPU"):
        op.fwd(x.cpu(), ga, be)
    with pytest.raises(ValueError, match="stats"):
        op.bwd(x, g, None, ga, be)
    with pytest.raises(ValueError, match="x is required"):
        op.fwd(None)
    flat = torch.zeros(x.numel() + 8, dtype=torch.float16, device="cuda")
    with pytest.raises(B.FnoError, match="INVALID_ARGUMENT"):  # not 16-byte aligned
        op.fwd(flat[1:1 + x.numel()].view(x.shape), ga, be)
    args = (op.desc, x.data_ptr(), 0, 0, 0, out.data_ptr(), 0)
    ws = torch.empty(op.ws_bytes[B.FNO_OP_FWD], dtype=torch.uint8, device="cuda")
    assert B.fno_group_norm_act_fwd(*args, ws.data_ptr(), ws.numel() - 1, 0,
                                    check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL
    assert B.fno_group_norm_act_fwd(*args, 0, ws.numel(), 0,
                                    check=False) == B.FNO_ERR_INVALID_ARGUMENT
