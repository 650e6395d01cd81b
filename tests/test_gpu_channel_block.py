"""The operators over channels together, as a block uses them: norm, a linear map
to four times the channels, GELU and the way back, norm with gate and residual
scale and the next block's norm; forward, backward and the optimizer's step."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from oracle import channel_oracle as C  # noqa: E402
from tests import rownorm_bounds as RB  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.fp8 import Fp8Linear  # noqa: E402
from paper_2307_15034_amd.layer import ResidualNorm  # noqa: E402
from paper_2307_15034_amd.optim import AdamW  # noqa: E402

BATCH, POINTS, CH = 4, 300, 40
ROWS = BATCH * POINTS


class Block:
    def __init__(self, seed, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.norm = ResidualNorm(ROWS, CH, dtype)
        self.up = Fp8Linear(ROWS, CH, 4 * CH, dtype)
        self.down = Fp8Linear(ROWS, 4 * CH, CH, dtype, B.FNO_NORM_ACT_GELU)
        self.p = {"in_w": 1 + 0.1 * r(CH), "in_b": 0.1 * r(CH), "w1": r(4 * CH, CH) / CH ** 0.5,
                  "b1": 0.1 * r(4 * CH), "w2": r(CH, 4 * CH) / (2 * CH ** 0.5), "b2": 0.1 * r(CH),
                  "post_w": 1 + 0.1 * r(CH), "gate": 0.5 + 0.2 * r(BATCH, CH), "scale": 1 + 0.1 * r(CH),
                  "pre_w": 1 + 0.1 * r(CH)}
        self.x = r(ROWS, CH).to(dtype)
        self.g_y, self.g_h = (0.1 * r(ROWS, CH)).to(dtype), (0.1 * r(ROWS, CH)).to(dtype)
        self.dtype = dtype

    def step(self):
        p = self.p
        w1, w2 = self.up.pack(p["w1"].to(self.dtype)), self.down.pack(p["w2"].to(self.dtype))
        _, h0 = self.norm.fwd(self.x, pre_w=p["in_w"], pre_b=p["in_b"])
        z, k1 = self.up.fwd(h0, w1, p["b1"])
        u, k2 = self.down.fwd(z, w2, p["b2"])
        join = dict(post_w=p["post_w"], gate=p["gate"], scale=p["scale"], pre_w=p["pre_w"])
        y, h = self.norm.fwd(self.x, u, **join)
        n = self.norm.bwd(self.g_y, self.g_h, x=self.x, u=u, y=y, **join)
        g_z, g_w2, g_b2 = self.down.bwd(n["g_u"], w2, k2, z)
        g_h0, g_w1, g_b1 = self.up.bwd(g_z, w1, k1)
        e = self.norm.bwd(n["g_x"], g_h0, x=self.x, pre_w=p["in_w"], pre_b=p["in_b"])
        grads = {"in_w": e["g_pre_w"], "in_b": e["g_pre_b"], "w1": g_w1, "b1": g_b1, "w2": g_w2,
                 "b2": g_b2, "post_w": n["g_post_w"], "gate": n["g_gate"], "scale": n["g_scale"],
                 "pre_w": n["g_pre_w"]}
        return dict(h0=h0, z=z, u=u, y=y, h=h, g_u=n["g_u"], g_z=g_z, g_h0=g_h0, g_x=e["g_x"], **
                    {"d_" + k: v for k, v in grads.items()})


def _f64(t):
    return t.double().cpu().numpy()


def test_each_stage_against_the_oracle():
    """Norms within their elements' bounds, products within the 2-norm's: a stored
    bfloat16 result is off by 2^-8 of itself, the eights' joins by 7 2^-13 of the
    sum of sizes, codes behind GELU by a neighbour now and then (2e-7 of values
    next to a tie, 2^-3 of each)."""
    say("block, stages")
    b = Block(1)
    o = b.step()
    p = {k: _f64(v) for k, v in b.p.items()}
    x = _f64(b.x)
    RB.close("h0", _f64(o["h0"]), *RB.forward(x, None, {"pre_w": p["in_w"], "pre_b": p["in_b"]}, "layer", 1e-5, "bf16")["h"])
    q = {k: p[k] for k in ("post_w", "gate", "scale", "pre_w")}
    want = RB.forward(x, _f64(o["u"]), q, "layer", 1e-5, "bf16")
    for k in ("y", "h"):
        RB.close(k, _f64(o[k]), *want[k])
    want = RB.backward(x, _f64(o["u"]), _f64(o["y"]), q, "layer", 1e-5, _f64(b.g_y), _f64(b.g_h), "bf16")
    RB.close("g_u", _f64(o["g_u"]), *want["g_u"])
    for k in ("post_w", "gate", "scale", "pre_w"):
        RB.close(k, _f64(o["d_" + k]), *want["g_" + k])

    def near(name, got, a, c, bias, u):
        want, size = a @ c.T + bias, np.abs(a) @ np.abs(c).T
        off = np.linalg.norm(_f64(got) - want)
        assert off <= u * np.linalg.norm(want) + 7 * 2.0 ** -13 * np.linalg.norm(size), name

    def codes(v, fmt="e4m3", tile=False):
        return C.values(*C.quantize(np.ascontiguousarray(v), fmt, "pow2", tile), tile)

    def gelu(v):
        from scipy.special import erf
        return v * 0.5 * (1 + erf(v / np.sqrt(2)))

    w1, w2 = (codes(_f64(b.p[k].bfloat16()), tile=True) for k in ("w1", "w2"))
    h0, z, g_u, g_z = (_f64(o[k]) for k in ("h0", "z", "g_u", "g_z"))
    near("z", o["z"], codes(h0), w1, p["b1"], 2.0 ** -8)
    near("u", o["u"], codes(gelu(z)), w2, p["b2"], 2.0 ** -8)
    near("g_h0", o["g_h0"], codes(g_z, "e5m2"), w1.T, 0.0, 2.0 ** -8)
    near("d_w1", o["d_w1"], codes(g_z.T, "e5m2"), codes(h0.T), 0.0, 1e-6)
    near("d_w2", o["d_w2"], codes(g_u.T, "e5m2"), codes(gelu(z).T), 0.0, 1e-6)
    assert np.allclose(_f64(o["d_b1"]), g_z.sum(0), rtol=0, atol=16 * 2.0 ** -24 * np.abs(g_z).sum(0).max())


def test_two_blocks_at_once_and_captured():
    """Two blocks on two streams, and one captured with the optimizer's step behind
    it and replayed, give what one alone gives."""
    say("block, streams and capture")
    first, second = Block(2), Block(3)
    want = [first.step(), second.step()]
    torch.cuda.synchronize()
    blocks, streams, got = [Block(2), Block(3)], [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = blocks[i].step()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for k in a:
            assert torch.equal(a[k], b[k]), k

    def train(steps, captured):
        b = Block(4)
        names = list(b.p)
        grads = {k: torch.zeros_like(v) for k, v in b.p.items()}
        opt = AdamW([b.p[k] for k in names], [grads[k] for k in names], lr=1e-2, device_control=True)

        def one():
            o = b.step()
            for k in names:
                grads[k].copy_(o["d_" + k])
            opt.clip_grads(1.0)
            opt.step()

        if not captured:
            for _ in range(steps):
                one()
            return b.p
        one()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one()
        for _ in range(steps - 1):
            graph.replay()
            b.x.float().sum().item()
        return b.p

    eager, replayed = train(5, False), train(5, True)
    for k in eager:
        assert torch.equal(eager[k], replayed[k]), k
