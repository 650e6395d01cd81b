"""The AdamW step, the gradient norm and the 8-bit moments on the GPU.

The step's order of rounded operations is stated, so results are compared bit
for bit with numpy's float32 in that order (its sums, products, quotients and
square roots are correctly rounded, as the device's are); the float64 oracle's
distance to that order is pinned on the CPU.  The gradient norm is a double
sum: within 2^-23 of the oracle's after its rounding to fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from oracle import train_oracle as T  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.optim import AdamW  # noqa: E402

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HYP = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-8)
SIZES = [1, 3, 255, 256, 257, 1000, 2047, 2048, 2049, 5000, 0, 8191, 4, 70001]


def _np(t):
    return t.detach().float().cpu().numpy().reshape(-1)


def _model(seed, sizes, param, grad, master, bits):
    r = np.random.default_rng(seed)
    f = lambda n, s: torch.tensor(r.standard_normal(n) * s, dtype=torch.float32)  # noqa: E731
    params = [f(n, 0.5).to(DT[param]).cuda() for n in sizes]
    grads = [f(n, 10.0 ** r.uniform(-3, 1)).to(DT[grad]).cuda() for n in sizes]
    masters = None
    if master:  # values between those the 16-bit type has
        masters = [(p.float() * (1 + 2.0 ** -12)).contiguous() for p in params]
    states = []
    for n in sizes:
        m, v = r.standard_normal(n).astype(np.float32), (r.standard_normal(n) ** 2).astype(np.float32)
        m *= np.float32(0.1)
        if bits == 32:
            states.append({"exp_avg": torch.tensor(m).cuda(), "exp_avg_sq": torch.tensor(v).cuda()})
        else:
            q = T.encode8(m, np.sqrt(v))
            states.append({k: torch.tensor(a).cuda() for k, a in zip(
                ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"), q)})
    return params, grads, masters, states


def _host(params, grads, masters, states):
    cp = lambda t: None if t is None else t.detach().cpu().numpy().copy().reshape(-1)  # noqa: E731
    return ([_np(p).copy() for p in params], [_np(g).copy() for g in grads],
            [cp(m) for m in masters] if masters else None,
            [{k: cp(v) for k, v in s.items()} for s in states])


def _expect(host, t, wd, scale=1.0):
    """The step in float32 on the host's copies, in place."""
    params, grads, masters, states = host
    for i, g in enumerate(grads):
        s = states[i]
        if "exp_avg_scale" in s:
            m, v = T.decode8(s["exp_avg"], s["exp_avg_sq"], s["exp_avg_scale"],
                             s["exp_avg_sq_scale"])
        else:
            m, v = s["exp_avg"], s["exp_avg_sq"]
        src = masters if masters else params
        w = wd[i] if isinstance(wd, list) else wd
        p, m, v, root = T.adamw_step32(src[i], g, m, v, t, HYP["lr"], *HYP["betas"], HYP["eps"],
                                       np.float32(w).astype(np.float64), scale)
        if "exp_avg_scale" in s:
            (s["exp_avg"], s["exp_avg_sq"], s["exp_avg_scale"],
             s["exp_avg_sq_scale"]) = T.encode8(m, root)
        else:
            s["exp_avg"], s["exp_avg_sq"] = m, v
        src[i] = p
        if masters:
            params[i] = p


def _same(host, params, masters, states, what=""):
    for i, p in enumerate(params):
        want = torch.tensor(host[0][i]).to(p.dtype).float().numpy()
        assert np.array_equal(_np(p), want), f"{what} param {i} (n = {p.numel()})"
        if not host[2]:
            host[0][i] = want
        else:
            assert np.array_equal(_np(masters[i]), host[2][i]), f"{what} master {i}"
        for k, v in states[i].items():
            assert np.array_equal(v.cpu().numpy(), host[3][i][k]), f"{what} {k} {i}"


KINDS = [("fp32", "fp32", False), ("fp16", "fp32", True), ("bf16", "fp32", True),
         ("fp16", "fp16", True), ("bf16", "bf16", True), ("fp16", "fp32", False),
         ("bf16", "bf16", False)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_step_bit_for_bit(kind, bits):
    param, grad, master = KINDS[kind]
    say(f"adamw {param} grad {grad} master {master} {bits} bits")
    params, grads, masters, states = _model(kind, SIZES, param, grad, master, bits)
    host = _host(params, grads, masters, states)
    opt = AdamW(params, grads, masters=masters, states=states, weight_decay=0.05, state_bits=bits,
                step=9, **HYP)
    for t in (10, 11, 12):
        opt.step()
        _expect(host, t, 0.05)
        _same(host, params, masters, opt.states, f"step {t}")
    assert opt.steps == 12


def test_many_mixed_tensors():
    """More tensors than a launch takes, types and state widths mixed, a decay
    of its own for each."""
    r = np.random.default_rng(3)
    params, grads, masters, states, bits, decay = [], [], [], [], [], []
    for i in range(3 * 40 + 7):
        k, b = KINDS[i % len(KINDS)], (32, 8, 8)[i % 3]
        p, g, m, s = _model(100 + i, [int(r.integers(1, 5000))], *k, b)
        params += p
        grads += g
        masters += m if m else [None]
        states += s
        bits.append(b)
        decay.append(0.01 * (i % 4))
    host = _host(params, grads, None, states)
    own = [None if m is None else m.cpu().numpy().copy() for m in masters]
    opt = AdamW(params, grads, masters=masters, states=states, weight_decay=decay, state_bits=bits,
                **HYP)
    opt.step()
    for i in range(len(params)):
        one = ([host[0][i]], [host[1][i]], [own[i]] if own[i] is not None else None, [host[3][i]])
        _expect(one, 1, decay[i])
        _same(one, params[i:i + 1], masters[i:i + 1], opt.states[i:i + 1], f"tensor {i}")


@pytest.mark.parametrize("bits", [32, 8])
def test_fresh_states_and_new_grads(bits):
    """Moments from zero, other gradients each step, an all-zero gradient."""
    params, grads, masters, _ = _model(5, [700, 33], "fp16", "fp32", True, bits)
    opt = AdamW(params, grads, masters=masters, state_bits=bits, weight_decay=0.0, **HYP)
    host = _host(params, grads, masters, opt.states)
    for t in (1, 2, 3):
        new = [g * t if t < 3 else torch.zeros_like(g) for g in grads]
        opt.step(new)
        host[1][:] = [_np(g) for g in new]
        _expect(host, t, 0.0)
        _same(host, params, masters, opt.states, f"step {t}")


def test_extreme_blocks():
    """Blocks of zeros, of one large value among tiny ones, and of values near
    the ends of fp32."""
    n = 6 * 256
    g = torch.zeros(n)
    g[256] = 1e3
    g[257:512] = 1e-9
    g[512:768] = 1e-18
    g[768:1024] = 1e15
    g[1024:1280] = torch.linspace(-1, 1, 256)
    g[1280:] = 1e-30  # squares below the smallest fp32
    params, grads = [torch.ones(n, device="cuda")], [g.cuda()]
    opt = AdamW(params, grads, state_bits=8, weight_decay=0.1, **HYP)
    host = _host(params, grads, None, opt.states)
    for t in (1, 2):
        opt.step()
        _expect(host, t, 0.1)
        _same(host, params, None, opt.states, f"step {t}")
    assert torch.isfinite(params[0]).all()


def test_moments_read_out():
    params, grads, _, states = _model(6, SIZES, "fp32", "fp32", False, 8)
    opt = AdamW(params, grads, states=states, state_bits=8, **HYP)
    for dt in ("fp32", "fp16", "bf16"):
        m, v = opt.moments(dtype=DT[dt])
        for i, s in enumerate(states):
            rm, rv = T.decode8(*[s[k].cpu().numpy() for k in (
                "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")])
            for got, ref in ((m[i], rm), (v[i], rv)):
                assert np.array_equal(_np(got), torch.tensor(ref).to(DT[dt]).float().numpy())
    # 32-bit states are their own values; a mixed list keeps its places
    mixed = AdamW([p.clone() for p in params], grads, state_bits=[32, 8] * 7, **HYP)
    mixed.step()
    m, v = mixed.moments()
    assert m[0] is mixed.states[0]["exp_avg"] and v[2] is mixed.states[2]["exp_avg_sq"]
    # from zero, the new first moment is 0.1 g: a code's distance from it
    assert float((m[1] - 0.1 * grads[1]).abs().max()) <= 0.01 * float(grads[1].abs().max())


def test_non_finite_gradient_without_control():
    """32-bit states: the element alone; 8-bit: its block, from the next step on."""
    for bits in (32, 8):
        params, grads, _, states = _model(7, [1024], "fp32", "fp32", False, bits)
        grads[0][300] = float("nan")
        opt = AdamW(params, grads, states=states, state_bits=bits, **HYP)
        opt.step()
        bad = torch.isnan(params[0])
        assert int(bad.sum()) == 1 and bool(bad[300])
        m, v = opt.moments()
        bad = torch.isnan(m[0]) | torch.isnan(v[0])
        want = torch.zeros(1024, dtype=torch.bool, device="cuda")
        want[300 if bits == 32 else slice(256, 512)] = True
        assert torch.equal(bad, want)


@pytest.mark.parametrize("kind", [0, 1, 4])
def test_control_clip_scale_and_skip(kind):
    """The norm within 2^-23, the clipped step bit for bit with that scale, a
    skipped step that changes nothing, the counts."""
    param, grad, master = KINDS[kind]
    params, grads, masters, states = _model(20 + kind, SIZES, param, grad, master, 32)
    host = _host(params, grads, masters, states)
    opt = AdamW(params, grads, masters=masters, states=states, step=4, device_control=True,
                weight_decay=0.02, **HYP)
    for t, (max_norm, loss_scale) in enumerate([(1.0, 64.0), (float("inf"), 2.0), (1e6, 1.0)], 5):
        norm = opt.clip_grads(max_norm, loss_scale)
        opt.step()
        c = opt.read_control()
        rn, rs, _ = T.grad_norm(host[1], max_norm, 1.0 / loss_scale)
        assert abs(float(norm) - rn) <= 2.0 ** -23 * rn
        assert abs(c["grad_scale"] - rs) <= 2.0 ** -23 * rs
        assert (c["step"], c["skip"], c["skipped"]) == (t, 0, 0)
        _expect(host, t, 0.02, np.float32(c["grad_scale"]))
        _same(host, params, masters, opt.states, f"step {t}")
    for k, bad in enumerate((float("inf"), float("nan"), -float("inf")), 1):
        keep = grads[5][77].clone()
        grads[5][77] = bad
        opt.clip_grads(1.0)
        opt.step()
        grads[5][77] = keep
        c = opt.read_control()
        assert (c["step"], c["skip"], c["skipped"]) == (7, 1, k)
        _same(host, params, masters, opt.states, "skipped")
    opt.set_lr_factor(0.0)
    opt.clip_grads(1.0)
    before = [p.clone() for p in params]
    opt.step()
    assert opt.read_control()["step"] == 8
    assert all(torch.equal(a, b) for a, b in zip(params, before))


def test_norm_of_large_gradients():
    """fp32 gradients whose squares overflow fp32 have a finite norm."""
    params = [torch.zeros(5000, device="cuda")]
    grads = [torch.full((5000,), 1e25, device="cuda")]
    opt = AdamW(params, grads, device_control=True, **HYP)
    norm = float(opt.clip_grads(1.0))
    assert abs(norm - 1e25 * np.sqrt(5000)) <= 1e-6 * norm
    opt.step()
    assert opt.read_control()["skip"] == 0 and torch.isfinite(params[0]).all()


def test_control_equals_host_steps():
    """With no clip, no loss scale and a finite gradient both ways give the same bits."""
    a = _model(30, SIZES, "fp16", "fp32", True, 8)
    b = [[None if t is None else ({k: v.clone() for k, v in t.items()} if isinstance(t, dict)
                                  else t.clone()) for t in col] for col in a]
    x = AdamW(a[0], a[1], masters=a[2], states=a[3], state_bits=8, step=99, **HYP)
    y = AdamW(b[0], b[1], masters=b[2], states=b[3], state_bits=8, step=99, device_control=True,
              **HYP)
    for _ in range(3):
        x.step()
        y.clip_grads()
        y.step()
    for p, q in zip(a[0] + a[2], b[0] + b[2]):
        assert torch.equal(p, q)
    for s, t in zip(x.states, y.states):
        assert all(torch.equal(s[k], t[k]) for k in s)


@pytest.mark.parametrize("bits", [32, 8])
def test_graph_replays(bits):
    """Norm and step captured once, replayed with other gradients, a skipped
    one and a changed learning rate among them: as eager calls give."""
    a = _model(40, [5000, 3, 70001], "fp16", "fp32", True, bits)
    b = [[None if t is None else ({k: v.clone() for k, v in t.items()} if isinstance(t, dict)
                                  else t.clone()) for t in col] for col in a]
    x = AdamW(a[0], a[1], masters=a[2], states=a[3], state_bits=bits, device_control=True, **HYP)
    y = AdamW(b[0], b[1], masters=b[2], states=b[3], state_bits=bits, device_control=True, **HYP)
    for o in (x, y):
        o.clip_grads(1.0)
        o.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.clip_grads(1.0)
        x.step()
    for k in range(5):
        for g, h in zip(a[1], b[1]):
            g.normal_(0, 1.0 + k)
            if k == 2:
                g[0] = float("inf")
            h.copy_(g)
        for o in (x, y):
            o.set_lr_factor(0.5 ** k)
        graph.replay()
        y.clip_grads(1.0)
        y.step()
        torch.cuda.synchronize()
        assert x.read_control() == y.read_control()
        for p, q in zip(a[0] + a[2], b[0] + b[2]):
            assert torch.equal(p, q), k
        for s, t in zip(x.states, y.states):
            assert all(torch.equal(s[j], t[j]) for j in s), k
    assert x.read_control()["skipped"] == 1


def test_another_stream():
    params, grads, masters, states = _model(45, [70001, 5], "fp16", "fp32", True, 32)
    host = _host(params, grads, masters, states)
    late = [torch.zeros_like(g) for g in grads]
    opt = AdamW(params, late, masters=masters, states=states, weight_decay=0.0, **HYP)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for a, b in zip(late, grads):
            a.copy_(b)
    opt.step(stream=s.cuda_stream)
    s.synchronize()
    _expect(host, 1, 0.0)
    _same(host, params, masters, opt.states)


@pytest.mark.parametrize("bits", [32, 8])
def test_offsets_past_32_bits(bits):
    """A tensor of more than 2^32 elements: its head and its tail as short
    tensors of the same values."""
    n = (1 << 32) + 1000
    p = torch.ones(n, dtype=torch.float16, device="cuda")
    g = torch.empty(n, dtype=torch.float16, device="cuda").fill_(0.25)
    tail = (1 << 20) + 1000 - (1 << 20) % 256
    at = n - tail
    assert at % 256 == 0
    g[at:].normal_(0, 1)
    sp, sg = p[at:].clone(), g[at:].clone()
    big = AdamW([p], [g], state_bits=bits, weight_decay=0.1, device_control=True, **HYP)
    small = AdamW([sp], [sg], state_bits=bits, weight_decay=0.1, **HYP)
    norm = float(big.clip_grads())
    rn = np.sqrt(at * 0.0625 + float((sg.double() ** 2).sum()))
    assert abs(norm - rn) <= 1e-6 * rn
    big.step()
    small.step()
    assert torch.equal(p[at:], sp)
    m = big.states[0]["exp_avg"]
    assert torch.equal(m[at:], small.states[0]["exp_avg"])
    assert torch.equal(p[:1 << 20], p[:1].expand(1 << 20)) and float(p[0]) < 1
    if bits == 8:
        out = [torch.empty(n, dtype=torch.float16, device="cuda") for _ in range(2)]
        big.moments([out[0]], [out[1]])
        ref = small.moments(dtype=torch.float16)
        assert torch.equal(out[0][at:], ref[0][0]) and torch.equal(out[1][at:], ref[1][0])


def test_storage_outlives_its_tensor():
    """The object keeps what it writes to: a gradient tensor that goes away
    leaves its memory in place until other gradients are given."""
    params, grads, _, states = _model(46, [5000], "fp32", "fp32", False, 32)
    host = _host(params, grads, None, states)
    opt = AdamW(params, [grads[0]], states=states, weight_decay=0.0, **HYP)
    opt.grads = None
    del grads
    junk = [torch.full((5000,), float("nan"), device="cuda") for _ in range(8)]
    opt.step()
    _expect(host, 1, 0.0)
    _same(host, params, None, opt.states)
    del junk


def test_refusals():
    p, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    h = p.half()
    cases = [
        (dict(params=[], grads=[]), "empty"),
        (dict(params=[p], grads=[]), "entries"),
        (dict(params=[p], grads=[None]), "required"),
        (dict(params=[p], grads=[g[:32]]), "shape"),
        (dict(params=[p], grads=[h]), "dtype"),
        (dict(params=[h], grads=[g.bfloat16()]), "dtype"),
        (dict(params=[p.double()], grads=[g]), "dtype"),
        (dict(params=[p], grads=[g], masters=[p.clone()]), "has none"),
        (dict(params=[p, p], grads=[g, g]), "twice"),
        (dict(params=[p], grads=[g], state_bits=16), "state_bits"),
        (dict(params=[p], grads=[g], step=-1), "step"),
        (dict(params=[p], grads=[g], states=[{"exp_avg": g}]), "states"),
        (dict(params=[p.cpu()], grads=[g]), "GPU"),
        (dict(params=[torch.zeros(64, 2, device="cuda")[:, 0]], grads=[g]), "contiguous"),
    ]
    for kw, match in cases:
        with pytest.raises(ValueError, match=match):
            AdamW(kw.pop("params"), kw.pop("grads"), **kw)
    opt = AdamW([p], [g])
    with pytest.raises(ValueError, match="device_control"):
        opt.clip_grads(1.0)
    for lr in (-1.0, float("nan"), float("inf")):
        with pytest.raises(B.FnoError, match="INVALID_ARGUMENT"):
            opt.step(lr=lr)
    ctl = AdamW([p], [g], device_control=True)
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(B.FnoError, match="INVALID_ARGUMENT"):
            ctl.clip_grads(bad)
        with pytest.raises(ValueError, match="loss_scale"):
            ctl.clip_grads(1.0, loss_scale=bad)
    with pytest.raises(ValueError, match="set_grads"):
        ctl.step([g])
    off = torch.zeros(65, device="cuda")
    with pytest.raises(B.FnoError, match="INVALID_ARGUMENT"):  # not 16-byte aligned
        AdamW([off[1:]], [g]).step()
