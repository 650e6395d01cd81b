"""Host-side checks of the C entry points of the operators over channels (no GPU
needed): sizes, and refusals before any device call."""
import pytest

B = pytest.importorskip("paper_2307_15034_amd.binding")

BAD = B.FNO_ERR_INVALID_ARGUMENT
A = 1 << 20  # an aligned address that is never reached


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=-1), dict(rows=(1 << 40) + 1), dict(channels=0), dict(channels=16385),
    dict(rows=1 << 40, channels=16), dict(gate_rows=-1), dict(gate_rows=7), dict(gate_rows=200),
    dict(dtype=3), dict(dtype=-1), dict(norm=2), dict(norm=-1), dict(gate_dtype=2),
    dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_residual_norm_descriptor_refused(kw):
    with pytest.raises(B.FnoError) as e:
        B.fno_residual_norm_workspace_size(B.make_residual_norm_desc(**{**dict(rows=100, channels=64), **kw}))
    assert e.value.status == BAD


def test_residual_norm_workspace_grows_with_what_is_summed():
    size = lambda **kw: B.fno_residual_norm_workspace_size(  # noqa: E731
        B.make_residual_norm_desc(**{**dict(rows=1 << 20, channels=64), **kw}))
    assert size() % 256 == 0 and size() >= 1024 * 5 * 64 * 4
    assert size(gate_rows=1) == size() // 5 * 6
    assert size(rows=1, channels=1) == 256
    assert size(gate_rows=1 << 20) == size()


def _p(**kw):
    return B.FnoResidualNormParams(**kw)


def test_residual_norm_call_refusals():
    d = B.make_residual_norm_desc(100, 64)
    dg = B.make_residual_norm_desc(100, 64, 4)
    fwd = dict(params=_p(post_w=A, pre_w=A), x=A, u=A, y=A, h=2 * A, stream=0)
    for desc, kw in ((d, dict(x=0)), (d, dict(x=A + 2)), (d, dict(u=A + 8)), (d, dict(y=0)),
                     (d, dict(y=A + 4)), (d, dict(h=A + 2)), (d, dict(u=0)), (d, dict(h=0)),
                     (d, dict(u=0, y=0)), (d, dict(u=0, y=0, h=0, params=_p())),
                     (d, dict(params=_p(gate=A))), (dg, {}), (d, dict(h=A)),
                     (d, dict(params=_p(post_w=A + 4))), (d, dict(params=_p(scale=A + 8))),
                     (d, dict(u=0, y=0, params=_p(scale=A))), (d, dict(h=0, params=_p(pre_b=A)))):
        assert B.fno_residual_norm_fwd(desc, **{**fwd, **kw}, check=False) == BAD, kw
    bwd = dict(params=_p(post_w=A, pre_w=A), x=A, u=A, y=A, g_y=A, g_h=A, g_x=A, g_u=2 * A,
               grads=_p(post_w=A, pre_w=A, scale=A), ws=A, ws_bytes=1 << 30, stream=0)
    for kw in (dict(g_x=0), dict(g_u=0), dict(g_u=A), dict(y=0), dict(x=0), dict(g_y=0, g_h=0),
               dict(g_h=0), dict(g_y=A + 2), dict(g_x=A + 4), dict(ws=0), dict(ws=A + 8),
               dict(grads=_p(gate=A)), dict(grads=_p(pre_w=A + 4)),
               dict(u=0, g_u=0), dict(u=0, g_u=0, y=0), dict(params=_p(gate=A))):
        assert B.fno_residual_norm_bwd(d, **{**bwd, **kw}, check=False) == BAD, kw
    assert B.fno_residual_norm_bwd(d, **{**bwd, "ws_bytes": 0},
                                   check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(cols=0), dict(rows=-5), dict(rows=1 << 31), dict(cols=1 << 31),
    dict(rows=1 << 30, cols=1 << 30), dict(dtype=3), dict(dtype=-1), dict(format=2), dict(format=-1),
    dict(scale_type=2), dict(blocks=2), dict(activation=3), dict(activation=-1)])
def test_quantize_descriptor_refused(kw):
    with pytest.raises(B.FnoError) as e:
        B.fno_fp8_quantize_workspace_size(B.make_fp8_quantize_desc(**{**dict(rows=10, cols=20), **kw}))
    assert e.value.status == BAD


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(cols=0), dict(inner=0), dict(rows=1 << 31), dict(inner=1 << 31),
    dict(rows=1 << 30, cols=1 << 30), dict(out_dtype=3), dict(format_a=2), dict(format_b=-1),
    dict(scale_type=2), dict(blocks_a=2), dict(blocks_b=-1), dict(activation=3)])
def test_matmul_descriptor_refused(kw):
    with pytest.raises(B.FnoError) as e:
        B.fno_fp8_matmul_workspace_size(B.make_fp8_matmul_desc(**{**dict(rows=10, cols=20, inner=30), **kw}))
    assert e.value.status == BAD


def test_pitch():
    assert [B.fno_fp8_pitch(n) for n in (-1, 0, 1, 16, 17, 128, (1 << 31) - 1)] == \
        [0, 0, 16, 16, 32, 128, 1 << 31]


def test_fp8_call_refusals():
    d = B.make_fp8_quantize_desc(10, 20)
    call = dict(x=A, codes=A, scale=A, codes_t=2 * A, scale_t=A, col_sums=A, ws=A, ws_bytes=1 << 20,
                stream=0)
    for kw in (dict(x=0), dict(x=A + 4), dict(codes=A + 4), dict(codes=0), dict(scale=0),
               dict(codes_t=0), dict(scale_t=0), dict(scale=A + 1), dict(codes_t=A), dict(ws=0),
               dict(ws=A + 4), dict(col_sums=A + 4),
               dict(codes=0, scale=0, codes_t=0, scale_t=0)):
        assert B.fno_fp8_quantize(d, **{**call, **kw}, check=False) == BAD, kw
    assert B.fno_fp8_quantize(d, **{**call, "ws_bytes": 255}, check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL
    d = B.make_fp8_matmul_desc(10, 20, 100000)
    call = dict(a=A, scale_a=A, b=A, scale_b=A, z=0, bias=A, out=A, ws=A, ws_bytes=1 << 30, stream=0)
    for kw in (dict(a=0), dict(b=0), dict(scale_a=0), dict(scale_b=0), dict(out=0), dict(a=A + 8),
               dict(scale_b=A + 4), dict(z=A), dict(bias=A + 4), dict(out=A + 2), dict(ws=0), dict(ws=A + 4)):
        assert B.fno_fp8_matmul(d, **{**call, **kw}, check=False) == BAD, kw
    assert B.fno_fp8_matmul(d, **{**call, "ws_bytes": 255}, check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL
    d = B.make_fp8_matmul_desc(10, 20, 30, activation=B.FNO_NORM_ACT_GELU)
    assert B.fno_fp8_matmul(d, **call, check=False) == BAD


def test_sizes_past_a_launch_are_refused():
    none = B.FNO_ERR_UNSUPPORTED
    d = B.make_fp8_quantize_desc(1 << 19, 1 << 19)
    for call in (lambda: B.fno_fp8_quantize_workspace_size(d),
                 lambda: B.fno_fp8_quantize(d, A, A, A, 0, 0, 0, A, 1 << 40, 0),
                 lambda: B.fno_fp8_matmul_workspace_size(B.make_fp8_matmul_desc((1 << 31) - 1, 2048, 64)),
                 lambda: B.fno_residual_norm_workspace_size(B.make_residual_norm_desc(1 << 24, 8, 1 << 23))):
        with pytest.raises(B.FnoError) as e:
            call()
        assert e.value.status == none
    assert B.fno_fp8_matmul_workspace_size(B.make_fp8_matmul_desc((1 << 31) - 1, 1, 64)) == 256
    assert B.fno_residual_norm_workspace_size(B.make_residual_norm_desc(1 << 24, 8, 1 << 24)) > 0
