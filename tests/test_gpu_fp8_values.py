"""Every 16-bit value, and values that are not finite, on their way through codes and
products."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests import test_gpu_fp8 as F  # noqa: E402
from tests.gpu_util import say  # noqa: E402


@pytest.mark.parametrize("dt", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
@pytest.mark.parametrize("tile", [False, True])
def test_every_16_bit_value_to_codes(dt, fmt, kind, tile):
    """All 65536 values of the type (bfloat16's in fp32), in their order (blocks of
    infinities and NaN alone, of subnormal numbers alone) and mixed (beside every
    size, signaling NaN among them): codes and scales bit for bit, both ways, from
    whole vectors and short ones."""
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    mixed = every[torch.randperm(1 << 16, generator=torch.Generator().manual_seed(4))]
    for name, bits, cols in (("ordered", every, 128), ("mixed", mixed, 64), ("mixed", mixed, 256),
                             ("ordered, odd", every[:65535], 255), ("ordered, short rows", every, 24)):
        rows = bits.numel() // cols
        say(name)
        x = bits[:rows * cols].reshape(rows, cols).cuda()
        x = (x.int() << 16).view(torch.float32) if dt == "fp32" else x.view(F.DT[dt])
        _, _, (q, t, _) = F._quantize(rows, cols, dt, fmt, kind, tile, x=x)
        v = F._f64(x)
        F._codes_are("rows", q, v, fmt, kind, tile)
        F._codes_are("columns", t, np.ascontiguousarray(v.T), fmt, kind, tile)


@pytest.mark.parametrize("dt", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("rows,k,n", [(40, 30, 50), (700, 60, 64), (3000, 200, 136)])
def test_a_gradient_that_is_not_finite_reaches_what_it_belongs_to(dt, kind, bad, rows, k, n):
    """One value of g that is not finite (a loss scale too large) makes its row of
    gx, its row of gW and its entry of gb not finite, and leaves the rest as it is
    with a zero there."""
    op, x, w, gy, bv, p, y, kept, *_ = F._linear(rows, k, n, dt, kind, seed=rows)
    r, c = rows - 3, n - 2
    gy[r, c] = 0
    clean = op.bwd(gy, p, kept)
    gy[r, c] = bad
    gx, gw, gb = op.bwd(gy, p, kept)
    at_r, at_c = (torch.arange(s, device="cuda") for s in (rows, n))
    assert not bool(gx[r].isfinite().any()) and torch.equal(gx[at_r != r], clean[0][at_r != r])
    assert not bool(gw[c].isfinite().any()) and torch.equal(gw[at_c != c], clean[1][at_c != c])
    assert not bool(gb[c].isfinite()) and torch.equal(gb[at_c != c], clean[2][at_c != c])


@pytest.mark.parametrize("dt", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("rows,k,n", [(40, 30, 50), (700, 60, 64), (3000, 200, 136)])
def test_an_input_that_is_not_finite_stays_in_its_row(dt, act, rows, k, n):
    op, x, w, gy, bv, p, y, kept, *_ = F._linear(rows, k, n, dt, "pow2", act, seed=rows)
    r = rows - 5
    x[r, 3] = 0
    clean = op.fwd(x, p, bv)[0]
    for bad in (float("inf"), float("nan")):
        x[r, 3] = bad
        got, codes = op.fwd(x, p, bv)
        keep = torch.arange(rows, device="cuda") != r
        assert bool(got[r].isnan().all()) and torch.equal(got[keep], clean[keep])
        assert bool(codes.codes.float()[3, r].isnan())
        assert int(codes.codes.float()[:, :rows].isnan().sum()) == 1
