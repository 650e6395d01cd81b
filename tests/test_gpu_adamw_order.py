"""The order of an AdamW object's calls, and what it counts."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2307_15034_amd.optim import AdamW  # noqa: E402


def _opt(**kw):
    g = torch.Generator(device="cuda").manual_seed(3)
    p, d = (torch.randn(5000, device="cuda", generator=g) for _ in range(2))
    return p, d, AdamW([p], [d], weight_decay=0.1, **kw)


def test_a_step_follows_a_clip():
    """Refused before the first clip_grads and after its step; nothing changes."""
    p, _, opt = _opt(device_control=True)
    before = p.clone()
    with pytest.raises(ValueError, match="clip_grads"):
        opt.step()
    opt.clip_grads(1.0)
    opt.clip_grads(1.0)  # the later one counts
    opt.step()
    after = p.clone()
    assert not torch.equal(before, after)
    for lr in (None, 5.0):
        with pytest.raises(ValueError, match="clip_grads"):
            opt.step(lr=lr)
    assert torch.equal(p, after) and opt.desc.lr != 5.0
    opt.clip_grads(1.0)
    opt.step()
    assert not torch.equal(p, after)


@pytest.mark.parametrize("given", [False, True])
def test_a_captured_clip_serves_every_step_behind_its_replays(given):
    p, d, opt = _opt(device_control=True)
    q, _, ref = _opt(device_control=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.clip_grads(1.0, stream=torch.cuda.current_stream().cuda_stream if given else None)
    for k in range(3):
        d.normal_(0, 1.0 + k)
        ref.grads[0].copy_(d)
        graph.replay()
        opt.step()
        ref.clip_grads(1.0)
        ref.step()
        torch.cuda.synchronize()
        assert torch.equal(p, q) and opt.read_control() == ref.read_control()


def test_steps_counts_in_both_ways():
    """What a checkpoint keeps and a new object starts from."""
    _, _, host = _opt(step=4)
    _, d, dev = _opt(step=4, device_control=True)
    assert (host.steps, dev.steps) == (4, 4)
    for k in range(3):
        host.step()
        if k == 1:  # one that is left out
            keep = d[7].clone()
            d[7] = float("inf")
            dev.clip_grads()
            dev.step()
            d[7] = keep
        dev.clip_grads()
        dev.step()
    assert (host.steps, dev.steps) == (7, 7)
    assert torch.equal(host.params[0], dev.params[0])
