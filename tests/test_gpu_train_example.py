"""The normalised block's training example: it learns, with 8-bit states as
with 32-bit ones, and runs the same bits twice."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def test_normalised_block_learns():
    from train_norm_block import train
    runs = {bits: train(60, bits) for bits in (32, 8)}
    for bits, losses in runs.items():
        assert all(v == v for v in losses)
        assert losses[-1] < 0.5 * losses[0], (bits, losses[0], losses[-1])
    # the 8-bit states' noise: a tenth of what the loss fell by
    assert abs(runs[8][-1] - runs[32][-1]) <= 0.1 * (runs[32][0] - runs[32][-1])
    assert train(20, 8, say=None) == runs[8][:20]
