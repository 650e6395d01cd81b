"""Pins of the float64 oracle of the training operators: torch's own float64
norm, activations, automatic differentiation and AdamW, finite differences,
and the properties that the 8-bit states promise."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import train_oracle as T  # noqa: E402


def _case(seed, b=3, c=12, p=17):
    r = np.random.default_rng(seed)
    return (r.standard_normal((b, c, p)) * 1.5 + r.standard_normal((1, c, 1)),
            1 + 0.2 * r.standard_normal(c), 0.3 * r.standard_normal(c),
            r.standard_normal((b, c, p)))


@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
@pytest.mark.parametrize("groups", [1, 4, 12])
def test_norm_matches_torch_in_float64(kind, groups):
    x, ga, be, g = _case(1)
    F = torch.nn.functional
    xt, gt, bt = (torch.tensor(a, requires_grad=True) for a in (x, ga, be))
    fn = {"none": lambda v: v, "gelu": F.gelu, "silu": F.silu}[kind]
    y = fn(F.group_norm(xt, groups, gt, bt, 1e-5)) + torch.tensor(g)
    out, stats = T.group_norm_act_fwd(x, ga, be, groups, 1e-5, kind, residual=g)
    np.testing.assert_allclose(out, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    v = x.reshape(3, groups, -1)
    np.testing.assert_allclose(stats[..., 0], v.mean(2), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(stats[..., 1], 1 / np.sqrt(v.var(2) + 1e-5), rtol=1e-12)
    ref = torch.autograd.grad(y, (xt, gt, bt), torch.tensor(g))
    for a, b in zip(T.group_norm_act_bwd(x, ga, be, groups, 1e-5, kind, g)[:3], ref):
        np.testing.assert_allclose(a, b.numpy(), rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
def test_norm_gradient_against_differences(kind):
    x, ga, be, g = _case(2, 2, 6, 5)
    gx, gg, gb = T.group_norm_act_bwd(x, ga, be, 3, 1e-5, kind, g)[:3]

    def loss(x, ga, be):
        return (T.group_norm_act_fwd(x, ga, be, 3, 1e-5, kind)[0] * g).sum()

    r, h = np.random.default_rng(3), 1e-6
    for i, (v, gr) in enumerate(((x, gx), (ga, gg), (be, gb))):
        d = r.standard_normal(v.shape)
        args = [x, ga, be]
        up, dn = list(args), list(args)
        up[i], dn[i] = v + h * d, v - h * d
        num = (loss(*up) - loss(*dn)) / (2 * h)
        assert abs(num - (gr * d).sum()) <= 1e-7 * (1 + abs(num))


def test_adamw_matches_torch_in_float64():
    r = np.random.default_rng(4)
    p0 = r.standard_normal(50)
    pt = torch.tensor(p0, requires_grad=True)
    opt = torch.optim.AdamW([pt], lr=3e-3, betas=(0.8, 0.95), eps=1e-7, weight_decay=0.1)
    p, m, v = p0, np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = r.standard_normal(50)
        pt.grad = torch.tensor(g)
        opt.step()
        p, m, v = T.adamw_step(p, g, m, v, t, 3e-3, 0.8, 0.95, 1e-7, 0.1)
        np.testing.assert_allclose(p, pt.detach().numpy(), rtol=1e-12, atol=1e-13)


def test_adamw_float32_order_is_near_float64():
    """Nine rounded operations: the update within 16 x 2^-24 of its own size,
    the parameter within that and 3 x 2^-24 of itself."""
    r = np.random.default_rng(5)
    p, g, m = (r.standard_normal(4096).astype(np.float32) for _ in range(3))
    v = (r.standard_normal(4096) ** 2).astype(np.float32)
    a = T.adamw_step32(p, g, m, v, 7, 1e-3, 0.9, 0.999, 1e-8, 0.01, 0.5)
    b = T.adamw_step(p, g, m, v, 7, 1e-3, 0.9, 0.999, 1e-8, 0.01, 0.5)
    u = 2.0 ** -24
    m_terms = np.abs(m) * 0.9 + np.abs(g) * 0.05
    assert np.all(np.abs(a[1] - b[1]) <= 6 * u * m_terms)
    assert np.all(np.abs(a[2] - b[2]) <= 8 * u * b[2])
    upd = 1e-3 * m_terms / (1 - 0.9 ** 7) / np.sqrt(b[2] / (1 - 0.999 ** 7))
    assert np.all(np.abs(a[0] - b[0]) <= u * (3 * np.abs(p) + 16 * upd))


def test_eight_bit_states_round_to_the_nearest_code():
    """In the square root of the value the error is at most half a step of
    the block's range; a second moment that is not zero stays so; zeros stay."""
    r = np.random.default_rng(6)
    m = (r.standard_normal(1000) * 10 ** r.uniform(-6, 0, 1000)).astype(np.float32)
    w = np.abs(r.standard_normal(1000) * 10 ** r.uniform(-9, 0, 1000)).astype(np.float32)
    m[:7] = 0
    w[:7] = 0
    m[300:512] = 0
    w[512:768] = 0
    qm, qv, a, b = T.encode8(m, w)
    dm, dv = T.decode8(qm, qv, a, b)
    A, B = np.repeat(a, 256)[:1000], np.repeat(b, 256)[:1000]
    e = np.abs(np.sqrt(np.abs(dm)) - np.sqrt(np.abs(m)))
    assert np.all(e <= np.sqrt(A) * (0.5 / 127) * 1.0001)
    assert np.all((dm == 0) | (np.sign(dm) == np.sign(m)))
    e = np.abs(np.sqrt(np.sqrt(dv)) - np.sqrt(w))
    assert np.all(e <= np.sqrt(B) * np.where(qv == 1, 1.0, 0.5) / 255 * 1.0001)
    assert np.array_equal(dv > 0, w > 0)
    assert np.all(dm[:7] == 0) and np.all(dv[512:768] == 0)


def test_eight_bit_training_follows_32_bit():
    """A noisy quadratic: 400 steps with 8-bit states end as near to the
    optimum as with 32-bit ones (within a quarter of the distance left)."""
    r = np.random.default_rng(7)
    n = 512
    target = r.standard_normal(n)
    curv = 10 ** r.uniform(-1, 1, n)
    ends = []
    for bits in (32, 8):
        rr = np.random.default_rng(8)
        p, m, v = (np.zeros(n, np.float32) for _ in range(3))
        q = T.encode8(m, v)
        for t in range(1, 401):
            g = (curv * (p - target) + 0.1 * rr.standard_normal(n)).astype(np.float32)
            if bits == 8:
                m, v = T.decode8(*q)
            p, m, v, w = T.adamw_step32(p, g, m, v, t, 1e-2, 0.9, 0.999, 1e-8, 0.0)
            if bits == 8:
                q = T.encode8(m, w)
        ends.append(np.sqrt(((p - target) ** 2).mean()))
    assert ends[0] < 0.2 and abs(ends[1] - ends[0]) <= 0.25 * ends[0], ends


def test_grad_norm_clips_and_sees_non_finite_values():
    a = [np.array([3.0, 0.0]), np.array([4.0])]
    assert T.grad_norm(a, 1.0, 0.5) == (2.5, 0.5 / 2.5, True)
    assert T.grad_norm(a, 10.0, 0.5) == (2.5, 0.5, True)
    assert T.grad_norm([np.zeros(3)], 1.0, 1.0) == (0.0, 1.0, True)
    assert not T.grad_norm([np.array([np.inf])], 1.0, 1.0)[2]
    assert not T.grad_norm([np.array([np.nan])], 1.0, 1.0)[2]
