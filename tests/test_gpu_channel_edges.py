"""The operators over channels where calls meet: captured graphs beside eager calls
of other forms, and memory that others own."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd.layer import ResidualNorm  # noqa: E402


def test_replays_keep_to_their_workspace_when_a_later_call_needs_more():
    """The backward without a gate is captured, then one with many gate rows (more
    partial sums) runs on the same object.  Replays give the same gradients and
    leave memory that was taken since as it was."""
    rows, c = 4096, 64
    say(f"residual norm {rows}x{c}, capture and a larger workspace")
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, u, gy = (r(rows, c).bfloat16() for _ in range(3))
    w, gate = 1 + 0.2 * r(c), r(rows // 2, c)
    op = ResidualNorm(rows, c, torch.bfloat16)
    want = op.bwd(gy, x=x, u=u, post_w=w)
    out = {k: torch.zeros_like(v) for k, v in want.items() if v is not None}
    torch.cuda.synchronize()
    small = op._ws._t.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.bwd(gy, x=x, u=u, post_w=w, out=dict(out))
    gated = op.bwd(gy, x=x, u=u, post_w=w, gate=gate)
    assert op._ws._t.numel() > small
    others = [torch.full((small,), 77, dtype=torch.uint8, device="cuda") for _ in range(16)]
    for turn in range(3):
        for t in out.values():
            t.zero_()
        (x.float().sum() + turn).item()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, want[k]), (turn, k)
        assert all(bool((t == 77).all()) for t in others), turn
        again = op.bwd(gy, x=x, u=u, post_w=w, gate=gate)
        for k, v in gated.items():
            assert v is None or torch.equal(again[k], v), (turn, k)
