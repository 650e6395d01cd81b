"""Group norm with an activation on the GPU where its kernels' limits, ranges
and values that are not numbers lie: every element within a bound of its own."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests.norm_bounds import check_elements  # noqa: E402


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("points", [1, 2])
@pytest.mark.parametrize("channels, groups", [
    (6112, 1),    # the most channels whose sums a work-group's LDS holds
    (6120, 1),    # one piece more
    (8192, 1),    # the most that its registers hold
    (65536, 8),
])
def test_wide_groups_of_few_rows(channels, groups, points, dt):
    """Channels last, one or two rows to a sample: a layer norm over features."""
    check_elements((points,), 3, channels, groups, dt, "gelu", True, points == 2, seed=400)
