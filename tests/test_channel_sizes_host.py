"""Sizes that the C entry points of the 8-bit codes accept (no GPU needed)."""
import pytest

B = pytest.importorskip("paper_2307_15034_amd.binding")

MOST = (1 << 31) - 1


@pytest.mark.parametrize("rows,cols", [(1 << 29, 8), (1 << 30, 1), (1 << 29, 20), (1 << 29, 64), (MOST, 1),
                                       (MOST, 16), (MOST, 127), (1, MOST), (127, MOST), (1, MOST - 300),
                                       ((1 << 19) - 1, 1 << 19)])
def test_codes_of_every_size_below_2_38(rows, cols):
    for blocks in (B.FNO_BLOCKS_ROW, B.FNO_BLOCKS_TILE):
        d = B.make_fp8_quantize_desc(rows, cols, blocks=blocks)
        assert B.fno_fp8_quantize_workspace_size(d) >= -(-rows // 128) * cols * 4


@pytest.mark.parametrize("rows,cols", [(1 << 19, 1 << 19), (129, MOST), (MOST, 129)])
def test_codes_of_2_38_values_are_refused(rows, cols):
    with pytest.raises(B.FnoError) as e:
        B.fno_fp8_quantize_workspace_size(B.make_fp8_quantize_desc(rows, cols))
    assert e.value.status == B.FNO_ERR_UNSUPPORTED


def test_linear_maps_over_large_grids():
    """Four grids of 512^3 points."""
    F = pytest.importorskip("paper_2307_15034_amd.fp8")
    for c_in, c_out in ((8, 32), (64, 64), (20, 80)):
        op = F.Fp8Linear(1 << 29, c_in, c_out)
        assert op.q_x.shape_t.codes == (c_in, 1 << 29)


@pytest.mark.parametrize("rows,c,each", [(1 << 20, 64, 2), (1 << 19, 64, 32), (8192, 4096, 2), (1 << 16, 4096, 8),
                                         (1 << 21, 64, 128), (1 << 22, 8, 2), (600000, 520, 3), (1 << 20, 64, 256)])
def test_partial_sums_of_gates_of_a_few_rows_stay_below_the_rows(rows, c, each):
    """The backward's workspace against one of its tensors, 16-bit."""
    d = B.make_residual_norm_desc(rows, c, rows // each)
    assert B.fno_residual_norm_workspace_size(d) < rows * c * 2 / 3


def test_backwards_of_the_residual_norm_that_one_launch_does_not_hold():
    size = lambda rows, c: B.fno_residual_norm_workspace_size(B.make_residual_norm_desc(rows, c))  # noqa: E731
    for rows, c in (((1 << 29) - 128, 4096), ((1 << 29) - 128, 8192), ((1 << 34), 1)):
        assert size(rows, c) > 0
    for rows, c in ((1 << 36, 1), (1 << 29, 8192)):
        with pytest.raises(B.FnoError) as e:
            size(rows, c)
        assert e.value.status == B.FNO_ERR_UNSUPPORTED
