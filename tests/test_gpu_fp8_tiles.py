"""Every tile of the 8-bit products against the float64 product, with the bounds of
test_gpu_fp8."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests import test_gpu_fp8 as F  # noqa: E402
from paper_2307_15034_amd.fp8 import Fp8Codes  # noqa: E402

FORMATS = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")]
EPILOGUES = [("none", False), ("silu", True), ("gelu", False)]


# 256 x 256, which needs 192 such tiles: ragged rows and columns, one block and more
@pytest.mark.parametrize("m,n,k", [(48897, 250, 64), (4000, 4100, 144), (4096, 4096, 400)])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("fa,fb", FORMATS)
def test_tiles_of_256(m, n, k, dt, fa, fb):
    for i, (act, bias) in enumerate(EPILOGUES):
        F._matmul(m, n, k, fa, fb, tb=i > 0, dt=dt, act=act, bias=bias, seed=20 + i)


# 256 x 64 of one stage: one block, up to 64 columns
@pytest.mark.parametrize("m,n,k", [(300, 64, 128), (1000, 20, 80), (257, 63, 17), (129, 1, 128), (5000, 36, 16)])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
def test_narrow_tiles(m, n, k, dt, kind):
    for fa, fb in FORMATS:
        for i, (act, bias) in enumerate(EPILOGUES):
            F._matmul(m, n, k, fa, fb, kind, tb=i > 0, dt=dt, act=act, bias=bias, seed=30 + i)


# 128 x 128 split along the inner axis, joined in the output's type with its epilogue
@pytest.mark.parametrize("m,n,k", [(130, 67, 3000), (200, 68, 5000)])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
def test_split_tiles(m, n, k, dt, kind):
    for fa, fb in FORMATS:
        for act, bias in EPILOGUES:
            F._matmul(m, n, k, fa, fb, kind, dt=dt, act=act, bias=bias, seed=40)


# few rows: one and four groups of 16
@pytest.mark.parametrize("m,n,k", [(12, 260, 2100), (40, 100, 700), (64, 33, 130)])
@pytest.mark.parametrize("dt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kind", ["pow2", "f32"])
def test_few_rows(m, n, k, dt, kind):
    for fa, fb in FORMATS:
        for i, (act, bias) in enumerate(EPILOGUES):
            F._matmul(m, n, k, fa, fb, kind, tb=i > 0, dt=dt, act=act, bias=bias, seed=50 + i)


@pytest.mark.parametrize("m,n,dt", [(300, 200, "fp32"), (4096, 3100, "fp32"), (4096, 3100, "fp16"), (300, 40, "bf16")])
def test_scales_and_codes_that_are_not_a_number_in_every_tile(m, n, dt):
    """Byte 255 of a row and of a column, and a NaN code, reach exactly their row and
    column of the result."""
    k = 100 if n <= 64 else 300
    op, a, b, _, _, out = F._matmul(m, n, k, dt=dt)
    sa, sb, cb = (t.view(torch.uint8).clone() for t in (a.scale, b.scale, b.codes))
    sa[-1, m - 2], sb[0, n - 1], cb[n - 3, 5] = 255, 255, 0x7F
    e8 = lambda s: s.view(torch.float8_e8m0fnu)  # noqa: E731
    got = op.run(Fp8Codes(a.codes, e8(sa)), Fp8Codes(cb.view(torch.float8_e4m3fn), e8(sb)))
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[m - 2] = True
    bad[:, [n - 1, n - 3]] = True
    assert bool(got[bad].isnan().all()) and torch.equal(got[~bad], out[~bad])


@pytest.mark.parametrize("m,n", [(8, 20), (200, 150), (300, 40), (4096, 3100)])
def test_scales_at_the_ends_of_their_range(m, n):
    """Products of a small value and a large one.  16-bit results: every pair of
    scales.  fp32 results: values (code times scale) of 2^-126 to fp32's largest."""
    k = 100
    e8 = lambda v, r: torch.full((1, r), v, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)  # noqa: E731
    for dt in ("fp32", "bf16"):
        op = F.Fp8Matmul(m, n, k, F.DT[dt])
        for byte_a, byte_b in ((1, 253), (0, 254), (254, 0), (3, 250), (246, 8), (120, 134), (60, 70)):
            for code, value in ((0x38, 1.0), (0x01, 2.0 ** -9), (0x7E, 448.0)):
                size = value * 2.0 ** (byte_a - 127)
                if dt == "fp32" and not 2.0 ** -126 <= size < 2.0 ** 128:
                    continue
                if dt == "fp32" and 2.0 ** (byte_b - 127) < 2.0 ** -126:
                    continue
                a = torch.zeros(m, 112, dtype=torch.uint8, device="cuda")
                b = torch.zeros(n, 112, dtype=torch.uint8, device="cuda")
                a[:, 5], b[:, 5] = code, 0x38
                f = lambda c, s: Fp8Codes(c.view(torch.float8_e4m3fn), s)  # noqa: E731
                got = op.run(f(a, e8(byte_a, m)), f(b, e8(byte_b, n)))
                want = torch.tensor(size * 2.0 ** (byte_b - 127), dtype=torch.float64).to(F.DT[dt])
                assert bool((got == want.cuda()).all()), (dt, byte_a, byte_b, code)
