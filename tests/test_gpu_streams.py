"""The training operators' own memory on a stream of the caller's: taken from
that stream's memory, filled before its first use, and handed to nobody else
before its last.  The caller's stream is kept busy by a bounded wait, so that
the order of the calls, not their speed, decides."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.layer import GroupNormAct  # noqa: E402
from paper_2307_15034_amd.optim import AdamW  # noqa: E402

WAIT = 20_000_000  # cycles


def _busy(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(WAIT)


def _norm():
    op = GroupNormAct((64, 48), 4, 32, 8, torch.float16, B.FNO_NORM_ACT_GELU, True)
    x = torch.randn(op.shape, device="cuda").half()
    return op, x


def test_norm_workspace_is_of_the_calls_stream():
    """The current stream still works on a block that it has given back, of the
    size of the workspace: the first call on another stream leaves it alone."""
    ref_op, x = _norm()
    ref, rst = ref_op.fwd(x)
    out, st = torch.empty_like(ref), torch.empty_like(rst)
    op = _norm()[0]
    n = max(op.ws_bytes.values())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    block = torch.empty(n, dtype=torch.uint8, device="cuda")
    at = block.data_ptr()
    torch.cuda._sleep(WAIT)
    block.fill_(255)
    del block
    op.fwd(x, out=out, stats=st, stream=s.cuda_stream)
    assert op._ws.data_ptr() != at
    again = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert again.data_ptr() == at  # the current stream's own may have it
    s.synchronize()
    assert torch.equal(out, ref) and torch.equal(st, rst)
    torch.cuda.synchronize()


def test_norm_workspace_outlives_its_object():
    """The object goes while a second stream's call is still queued: the
    workspace is not handed out before that call ends."""
    op, x = _norm()
    ref, rst = op.fwd(x)
    out, st = torch.empty_like(ref), torch.empty_like(rst)
    n, at = op._ws.numel(), op._ws.data_ptr()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(s)
    op.fwd(x, out=out, stats=st, stream=s.cuda_stream)
    del op
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not s.query()
    assert at not in [t.data_ptr() for t in others]
    for t in others:
        t.fill_(255)
    s.synchronize()
    assert torch.equal(out, ref) and torch.equal(st, rst)


def test_norm_on_the_default_stream_from_another():
    """stream 0 given while another stream is current."""
    op, x = _norm()
    ref, rst = _norm()[0].fwd(x)
    out, st = torch.empty_like(ref), torch.empty_like(rst)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        op.fwd(x, out=out, stats=st, stream=torch.cuda.default_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(st, rst)


def test_norm_first_call_inside_a_capture():
    op, x = _norm()
    ref, rst = _norm()[0].fwd(x)
    out, st = torch.empty_like(ref), torch.empty_like(rst)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.fwd(x, out=out, stats=st)
    for _ in range(3):
        out.zero_()
        junk = torch.full((op._ws.numel(),), 255, dtype=torch.uint8, device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(st, rst)
        del junk


N = 300001


def _params():
    g = torch.Generator(device="cuda").manual_seed(7)
    return [torch.randn(N, device="cuda", generator=g) for _ in range(2)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("control", [False, True])
def test_adamw_first_step_on_another_stream(bits, control):
    """The constructor's own tensors are filled behind a busy current stream,
    in blocks that held other values; the first step on another stream finds
    them filled."""
    p, g = _params()
    ref = p.clone()
    AdamW([ref], [g], state_bits=bits).step()
    q = p.clone()
    torch.cuda.synchronize()
    junk = [torch.full((N,), 3.0, device="cuda") for _ in range(4)]
    junk += [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (N, N, 64, 512, 8192)]
    torch.cuda._sleep(WAIT)
    del junk
    opt = AdamW([q], [g], state_bits=bits, device_control=control)
    s = torch.cuda.Stream()
    if control:
        opt.clip_grads(stream=s.cuda_stream)
    opt.step(stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(q, ref)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_states_outlive_their_object(bits):
    """The object goes while another stream's step is still queued."""
    p, g = _params()
    ref = p.clone()
    opt = AdamW([ref], [g], state_bits=bits, device_control=True)
    opt.clip_grads()
    opt.step()
    q = p.clone()
    opt = AdamW([q], [g], state_bits=bits, device_control=True)
    made = {t.data_ptr(): (t.numel(), t.dtype) for t in opt._made}
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(s)
    opt.clip_grads(stream=s.cuda_stream)
    opt.step(stream=s.cuda_stream)
    del opt
    others = [torch.full((n,), 1, dtype=dt, device="cuda") for n, dt in made.values()
              for _ in range(3)]
    assert not s.query()
    assert not made.keys() & {t.data_ptr() for t in others}
    s.synchronize()
    assert torch.equal(q, ref)
