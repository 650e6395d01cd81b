"""The group norm and the optimizer at the sizes where their kernels change:
groups at the end of what one work-group holds, rows aligned or not, groups
that cross vectors, channels past a work-group, sums joined by a launch of
their own; gradient lists on both sides of one launch and of one join, and
parameter lists on both sides of two pieces to a work-group.

The norm's tolerances are those of tests/test_gpu_norm.py; the step is compared
bit for bit; the gradient norm, a double sum rounded to fp32 once, within 2^-23
of numpy's."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_adamw import HYP, _expect, _host, _model, _same  # noqa: E402
from tests.test_gpu_norm import _check  # noqa: E402
from paper_2307_15034_amd.optim import AdamW  # noqa: E402

NORM = [
    # (points, batch, channels, groups, type, channels last)
    (16384, 2, 4, 4, "fp16", False),    # one plane of 16384: the last held by a work-group
    (16385, 2, 4, 4, "fp16", False),    # the first that is not, odd
    (4096, 2, 8, 2, "fp32", False),     # four planes of 4096
    (4104, 2, 8, 2, "fp32", False),
    (1024, 3, 32, 2, "bf16", False),    # sixteen planes, a wave each
    (64, 2, 512, 2, "fp16", False),     # more planes than waves
    (2048, 2, 16, 2, "fp16", True),     # 8 channels by 2048 rows
    (2049, 2, 16, 2, "fp16", True),
    (4096, 2, 8, 2, "fp16", True),      # 4 channels of 8-element vectors
    (4097, 2, 8, 2, "bf16", True),
    (2730, 2, 9, 3, "fp32", True),      # channels one by one
    (2731, 2, 9, 3, "fp32", True),
    (300, 2, 1032, 1, "fp16", True),    # a row longer than a work-group's pieces
    (6000, 2, 24, 6, "fp16", True),     # aligned rows, groups of half a vector
    (5999, 3, 12, 1, "fp16", True),     # rows of 24 bytes, the sample's end inside one
    (700, 2, 4096, 2, "fp16", True),    # channels past a work-group
    (333, 2, 4100, 4, "fp32", True),
    (99, 2, 2051, 7, "bf16", True),     # and odd
    (40, 2, 4096, 256, "fp32", True),   # many groups of a sample
    (9000, 1, 64, 64, "fp16", True),    # one channel to a group, several chunks
    (140000, 1, 48, 48, "bf16", True),  # sums joined by a launch of their own
    (300, 2, 1600, 2, "fp32", False),   # 800 planes to a group, the same
    (9000, 2, 6, 2, "fp16", False),     # planes for a wave / for a work-group
    (8200, 2, 6, 2, "bf16", False),
    (8192, 3, 10, 2, "fp16", False),
]


@pytest.mark.parametrize("case", range(len(NORM)))
def test_norm_sizes(case):
    points, b, c, g, dt, last = NORM[case]
    act = ("silu", "gelu", "none")[case % 3]
    _check((points,), b, c, g, dt, act, last, residual=case % 2 == 1, seed=200 + case)


@pytest.mark.parametrize("points, channels, dt", [(300001, 48, "fp16"), (5000001, 4, "fp16"),
                                                  (2500001, 4, "fp32")])
def test_norm_of_many_segments(points, channels, dt):
    """Channels first, one group: up to the segments that the second pass joins
    itself, and more."""
    _check((points,), 1, channels, 1, dt, "gelu", False, residual=True, seed=300)


def _norm_of(grads):
    return np.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


@pytest.mark.parametrize("count, size", [
    (1, 8192 * 512),       # the most chunks that the same launch joins
    (1, 8192 * 512 + 1),   # one more
    (128, 100),            # the most tensors of a launch
    (129, 100),            # two launches
    (300, 8193),           # several launches, two chunks each
    (700, 5),
])
def test_gradient_norm_lists(count, size):
    say(f"norm of {count} gradients of {size}")
    g = torch.Generator(device="cuda").manual_seed(count + size)
    big = torch.randn(count * (size + 3), device="cuda", generator=g)
    # aligned and separate, a few of them far larger
    grads = [(big[i * (size + 3):][:size] * (100.0 if i % 50 == 7 else 1.0)).clone()
             for i in range(count)]
    params = [torch.zeros(size, device="cuda") for _ in range(count)]
    opt = AdamW(params, grads, device_control=True, **HYP)
    want = _norm_of(grads)
    for _ in range(2):  # the second pass finds the first's workspace
        got = float(opt.clip_grads(0.5))
        assert abs(got - want) <= 2.0 ** -23 * want
    # a value that is no number, in the last tensor's last place
    grads[-1][-1] = float("nan")
    opt.clip_grads(0.5)
    opt.step()
    c = opt.read_control()
    assert c["skip"] != 0 and c["skipped"] == 1
    assert all(not p.any() for p in params[-3:])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", [("fp32", "fp32", False), ("fp16", "fp16", True),
                                  ("bf16", "fp32", True), ("fp16", "fp32", False)])
def test_long_lists_bit_for_bit(kind, bits):
    """Lists just below and past 2^22 elements, tensors that end in and between
    the pieces of a work-group."""
    for total in ((1 << 22) - 4096, (1 << 22) + 4096):
        sizes = [2047, 2048, 2049, 1023, 1025, 1, 256, 3000]
        sizes.append(total - sum(sizes))
        params, grads, masters, states = _model(total % 97, sizes, *kind, bits)
        host = _host(params, grads, masters, states)
        opt = AdamW(params, grads, masters=masters, states=states, weight_decay=0.02,
                    state_bits=bits, step=3, **HYP)
        opt.step()
        _expect(host, 4, 0.02)
        _same(host, params, masters, opt.states, f"{total}")


def test_moments_given_lists():
    """The read-out into the caller's lists, with states of both widths, and what
    it refuses."""
    sizes = [300, 5000, 1, 70000]
    params, grads, _, _ = _model(5, sizes, "fp32", "fp32", False, 32)
    opt = AdamW(params, grads, state_bits=[8, 32, 8, 8], **HYP)
    opt.step()
    want = opt.moments()
    outs = [[torch.full((n,), 7.0, device="cuda") for n in sizes] for _ in range(2)]
    got = opt.moments(*outs)
    for w, g in zip(want, got):
        for i in (0, 2, 3):
            assert torch.equal(w[i], g[i])
        assert (g[1] == 7).all()  # 32-bit states stay where they are
    for bad in ("float", None, torch.zeros(300), torch.zeros(300, device="cuda", dtype=torch.float16),
                torch.zeros(301, device="cuda"), torch.zeros(600, device="cuda")[::2]):
        lists = [list(o) for o in outs]
        lists[1][0] = bad
        with pytest.raises(ValueError):
            opt.moments(*lists)
    with pytest.raises(ValueError):
        opt.moments(outs[0][:-1], outs[1])
