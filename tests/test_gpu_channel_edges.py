"""The operators over channels where calls meet: captured graphs beside eager calls
of other forms, and memory that others own."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.fp8 import Fp8Linear, Fp8Quantize  # noqa: E402
from paper_2307_15034_amd.layer import ResidualNorm  # noqa: E402


def test_replays_keep_to_their_workspace_when_a_later_call_needs_more():
    """The backward without a gate is captured, then one with a gate (a partial sum
    more) runs on the same object.  Replays give the same gradients and
    leave memory that was taken since as it was."""
    rows, c = 4096, 64
    say(f"residual norm {rows}x{c}, capture and a larger workspace")
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, u, gy = (r(rows, c).bfloat16() for _ in range(3))
    w, gate = 1 + 0.2 * r(c), r(1, c)
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


def _same_codes(name, got, want):
    for a, b in zip(got, want):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), name


@pytest.mark.parametrize("rows,cols", [((1 << 29) + 77, 8), (3, (1 << 31) - 1)])
def test_codes_of_the_tallest_and_widest_matrices(rows, cols):
    """Work-groups past a row of the grid, columns up to 2^31 - 1: the last blocks
    (and the first) against the same blocks alone, bit for bit."""
    say(f"quantize {rows}x{cols}, all outputs, then codes of rows alone")
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    op = Fp8Quantize(rows, cols, torch.bfloat16)
    q, t, sums = op.run(x, transpose=True, col_sums=True)
    tall = rows > cols
    n = (rows if tall else cols)
    last = (n - 1000) // 128 * 128
    for a, b in ((0, 1280), (last, n)):
        some = (x[a:b] if tall else x[:, a:b]).contiguous()
        q2, t2, sums2 = Fp8Quantize(*some.shape, torch.bfloat16).run(some, transpose=True, col_sums=True)
        r, c = some.shape
        rows_of = slice(a, b) if tall else slice(0, r)
        cols_of = slice(0, c) if tall else slice(a, b)
        _same_codes("rows", (q.codes[rows_of, cols_of], q.scale[:, a:b] if tall else q.scale[a // 128:][:len(q2.scale)]),
                    (q2.codes[:, :c], q2.scale))
        _same_codes("columns", (t.codes[cols_of, rows_of],
                                t.scale[a // 128:][:len(t2.scale)] if tall else t.scale[:, a:b]),
                    (t2.codes[:, :r], t2.scale))
        if not tall:
            assert torch.equal(sums[a:b], sums2)
    if tall:  # fp32 chains of 8 and a tree over 16 threads, then doubles: 16 2^-24 of the sizes
        want, size = 0.0, 0.0
        for i in range(0, rows, 1 << 26):
            v = x[i:i + (1 << 26)].double()
            want, size = want + v.sum(0), size + v.abs().sum(0)
        assert bool(((sums.double() - want).abs() <= 16 * 2.0 ** -24 * size + 2.0 ** -24 * want.abs()).all())
    only, _, _ = op.run(x)
    _same_codes("rows alone", only, q)


def test_a_buffer_for_two_gradients_is_refused():
    op = Fp8Linear(48, 32, 48, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(9)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, w, gy = r(48, 32), r(48, 32), r(48, 48)
    p = op.pack(w)
    _, kept = op.fwd(x, p)
    want = op.bwd(gy, p, kept)
    both = torch.zeros(48, 32, device="cuda")
    with pytest.raises(ValueError, match="twice"):
        op.bwd(gy, p, kept, gx=both, gw=both)
    assert not bool(both.any())
    assert all(torch.equal(a, b) for a, b in zip(op.bwd(gy, p, kept, gx=both), want))
    norm = ResidualNorm(48, 32, torch.float32)
    one = torch.zeros(32, device="cuda")
    with pytest.raises(B.FnoError):
        norm.bwd(x, x, x=x, u=x, y=x, post_w=r(32), pre_w=r(32), out={"g_post_w": one, "g_pre_w": one})
    assert not bool(one.any())
