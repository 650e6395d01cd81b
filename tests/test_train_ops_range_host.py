"""Refusals of the gradient norm past the range of what it stores (no GPU needed)."""
import pytest

B = pytest.importorskip("paper_2307_15034_amd.binding")

from tests.test_train_ops_host import A, BAD, OPT, _list  # noqa: E402


@pytest.mark.parametrize("inv", [3.5e38, 1e39, 1e308])
def test_loss_scale_past_fp32_refused(inv):
    """grad_scale is fp32: inf there would make every zero gradient NaN."""
    t = _list()
    n = B.fno_grad_norm_workspace_size(t, 1)
    # a workspace a byte too small, so that nothing is launched either way
    assert B.fno_grad_norm(OPT, t, 1, max_norm=1.0, inv_loss_scale=inv, control=A, ws=A,
                           ws_bytes=n - 1, stream=0, check=False) == BAD
    assert B.fno_grad_norm(OPT, t, 1, max_norm=1.0, inv_loss_scale=3.3e38, control=A, ws=A,
                           ws_bytes=n - 1, stream=0, check=False) == B.FNO_ERR_WORKSPACE_TOO_SMALL
