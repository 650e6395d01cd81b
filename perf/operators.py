"""Group norm with an activation, and the optimizer step, as timed cases.

"norm_fwd"  group norm + activation (+ residual) of a tensor, the statistics
            kept for the backward
"norm_bwd"  its backward: the input's and the affine parameters' gradients
"adamw"     one AdamW step over all the tensors of an operator model (blocks of
            spectral weights, skip, bias and norm parameters): states in 32
            bits, behind the global gradient norm with clip, loss scale and
            non-finite check ("clip"), or in 8 bits

With `own` false a pass computes the plain form in elementary torch operations
(32 bits, rounded once at the end); with `own` true it makes the calls of this
package.  `listed()` are the fixed cases, `draw()` gives others of the same
ranges, `exact()` the same results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _norm(name, do, n, batch, channels, groups, dtype="fp16", act="gelu", last=True,
          residual=False):
    """Grids are written as text ("128x128") so that a case is plain values."""
    c = {"do": do, "n": n, "batch": batch, "channels": channels, "groups": groups,
         "dtype": dtype, "act": act, "last": last, "residual": residual}
    if name:
        c["name"] = name
    return c


def _adamw(name, layers, channels, modes, weight="dense", rank="", param="fp16", bits=32,
           clip=True):
    """param "fp16" / "bf16": 16-bit parameters beside an fp32 master."""
    c = {"do": "adamw", "layers": layers, "channels": channels, "modes": modes,
         "weight": weight, "rank": rank, "param": param, "bits": bits, "clip": clip}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The norm behind one block of the smallest workload (64 x 64, two
        # samples of 16 channels): latency.
        _norm("norm-fwd-64", "norm_fwd", "64x64", 2, 16, 4),
        # Behind a block of the Navier-Stokes workload, channels last, as a
        # pointwise network around the spectral layer keeps its tensors.
        _norm("norm-fwd-last-128", "norm_fwd", "128x128", 32, 64, 8),
        _norm("norm-bwd-last-128", "norm_bwd", "128x128", 32, 64, 8),
        # The largest: the 1024 x 1024 workload in the spectral layer's own
        # layout, the block's residual added behind the activation.
        _norm("norm-fwd-first-1024", "norm_fwd", "1024x1024", 8, 64, 8, last=False,
              residual=True),
        # The Tucker workload's 128 channels in 32 groups, SiLU, bfloat16.
        _norm("norm-bwd-first-256", "norm_bwd", "256x256", 16, 128, 32, "bf16", "silu",
              last=False),
        # An odd grid (data on node grids) with 20 channels: rows of 40 bytes,
        # groups of five channels.
        _norm("norm-bwd-last-odd", "norm_bwd", "241x241", 16, 20, 4),
        # The 3-D workload in full precision, one group (all channels of a
        # sample normalised together).
        _norm("norm-fwd-last-3d", "norm_fwd", "64x64x64", 4, 32, 1, "fp32", "silu"),
        # The optimizer of the smallest workload's operator: latency.
        _adamw("adamw-64", 4, 16, "8x8"),
        # Navier-Stokes operator, mixed precision: fp16 weights and fp32
        # masters, behind the clipped gradient norm.
        _adamw("adamw-128", 4, 64, "32x32"),
        # The Tucker-factorised operator: many small tensors, full precision.
        _adamw("adamw-tucker", 8, 128, "32x32", "tucker", "13,13,6,3", param="fp32"),
        # The Navier-Stokes operator with its states in 8 bits.
        _adamw("adamw8-128", 4, 64, "32x32", bits=8, clip=False),
        # The 1024 x 1024 workload's weights, fp32, states in 8 bits.
        _adamw("adamw8-1024", 4, 64, "64x64", param="fp32", bits=8, clip=False),
    ]


# ---------------------------------------------------------------------------
# Other cases of the same ranges
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["norm_fwd", "norm_bwd", "norm_fwd", "norm_bwd", "adamw", "adamw"])
    if do == "adamw":
        bits = rng.choice([32, 8])
        weight = rng.choice(["dense", "dense", "dense", "tucker", "cp"])
        channels = rng.choice([16, 20, 32, 33, 48, 64, 128])
        # as many modes as keep a layer within 2^24 complex weights
        most = max(8, min(64, int(math.sqrt((1 << 24) / (2 * channels * channels)))))
        modes = "%dx%d" % (_log(rng, 4, most), _log(rng, 4, most))
        rank = {"dense": "", "cp": str(_log(rng, 4, 40)),
                "tucker": ",".join(str(rng.randint(3, 16)) for _ in range(4))}[weight]
        return _adamw(None, rng.randint(1, 4) if weight == "dense" else rng.randint(1, 12),
                      channels, modes, weight, rank, rng.choice(["fp32", "fp16", "bf16"]), bits,
                      bits == 32 and rng.random() < 0.6)
    d = rng.choice([1, 2, 2, 2, 3])
    top = {1: 65536, 2: 1024, 3: 96}[d]
    n = []
    for _ in range(d):
        v = _log(rng, {1: 64, 2: 16, 3: 8}[d], top)
        how = rng.random()
        even = 1 << max(3, round(math.log2(v)))
        n.append(even if how < 0.4 else v // 8 * 8 if how < 0.6 and d > 1 else v | 1)
    channels = rng.choice([16, 20, 32, 48, 64, 64, 128, rng.randint(3, 160)])
    groups = rng.choice([g for g in range(1, channels + 1) if channels % g == 0])
    batch = _log(rng, 1, max(1, min(32, (1 << 27) // (math.prod(n) * channels))))
    return _norm(None, do, "x".join(map(str, n)), batch, channels, groups,
                 rng.choice(["fp16", "fp16", "bf16", "fp32"]), rng.choice(["gelu", "silu", "none"]),
                 rng.random() < 0.6, do == "norm_fwd" and rng.random() < 0.4)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _grid(case):
    return tuple(int(v) for v in case["n"].split("x"))


def _shape(case):
    n, c = _grid(case), case["channels"]
    return (case["batch"],) + (n + (c,) if case["last"] else (c,) + n)


def _rows(t, last):
    """[batch, channels, points] view of a tensor of either layout."""
    return t.flatten(1, -2).transpose(1, 2) if last else t.flatten(2)


EPS = 1e-5


def _prepare_norm(case, seed):
    """Activations with an offset and a spread of their own in each channel,
    affine parameters near (1, 0), white output gradients."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    f32 = dict(device="cuda", generator=g)
    c, dt, shape = case["channels"], DTYPES[case["dtype"]], _shape(case)
    per = (1,) * (len(shape) - 1) + (c,) if case["last"] else (1, c) + (1,) * (len(shape) - 2)
    spread = torch.rand((c,), **f32) + 0.5
    offset = torch.randn((c,), **f32)

    def noise():
        out = torch.empty(shape, dtype=dt, device="cuda")
        for b in range(shape[0]):
            out[b] = torch.randn(shape[1:], **f32).to(dt)
        return out

    x = noise()
    for b in range(shape[0]):
        x[b] = (x[b].float() * spread.view(per[1:]) + offset.view(per[1:])).to(dt)
    s = {"case": case, "x": x, "gamma": 1 + 0.1 * torch.randn((c,), **f32),
         "beta": 0.1 * torch.randn((c,), **f32)}
    if case["residual"]:
        s["residual"] = noise()
    if case["do"] == "norm_bwd":
        s["g_out"] = noise()
        stats = torch.empty((case["batch"], case["groups"], 2), device="cuda")
        for b in range(shape[0]):  # what the forward keeps: mean and 1 / deviation
            v = _rows(x[b:b + 1], case["last"]).reshape(case["groups"], -1).double()
            m = v.mean(1)
            stats[b, :, 0] = m.float()
            stats[b, :, 1] = (v.var(1, unbiased=False) + EPS).rsqrt().float()
        s["stats"] = stats
    return s


LR, BETAS, OPT_EPS, DECAY, STEPS = 1e-3, (0.9, 0.999), 1e-8, 1e-2, 1000
LOSS_SCALE, MAX_NORM = 1024.0, 1.0
ALIGN = 1024  # elements: the start of each tensor in the flat buffers


def _sizes(case):
    """Elements (reals; complex weights count twice) of the model's tensors:
    per block the spectral weight or its factors, skip, bias and the norm's
    parameters, and the lifting and projection maps around the blocks."""
    c = case["channels"]
    m = [int(v) for v in case["modes"].split("x")]
    k = [2 * v for v in m[:-1]] + m[-1:]
    r = [int(v) for v in case["rank"].split(",")] if case["rank"] else []
    if case["weight"] == "dense":
        spectral = [c * c * math.prod(k)]
    elif case["weight"] == "tucker":
        spectral = [math.prod(r), c * r[0], c * r[1]] + [a * b for a, b in zip(k, r[2:])]
    else:
        spectral = [r[0], c * r[0], c * r[0]] + [a * r[0] for a in k]
    block = [2 * v for v in spectral] + [c * c, c, c, c]
    return [3 * c, c] + block * case["layers"] + [c, 1]


def _encode(m, w):
    """8-bit states of blocks of 256: codes and scales of m and of
    w = sqrt(v), see _decode."""
    a, b = m.abs().amax(1, keepdim=True), w.amax(1, keepdim=True)
    qm = (torch.sqrt(m.abs() / torch.where(a > 0, a, 1.0)) * 127.0).round() * m.sign()
    qv = (torch.sqrt(w / torch.where(b > 0, b, 1.0)) * 255.0).round()
    qv = torch.where((w > 0) & (qv < 1), 1.0, qv)
    return qm.to(torch.int8), qv.to(torch.uint8), a, b


def _decode(qm, qv, a, b):
    """m = (A / 127^2) q |q|, v = ((B / 255^2) q^2)^2."""
    q = qm.float()
    m = (a * (1.0 / 16129.0)) * (q * q.abs())
    q = qv.float()
    s = (b * (1.0 / 65025.0)) * (q * q)
    return m, s * s


def _prepare_adamw(case, seed):
    """The model's tensors as views of flat buffers; gradients of a loss scaled
    by LOSS_SCALE (with clip), each tensor of a size of its own; moments as
    they are after many steps on such gradients."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    sizes = _sizes(case)
    at, total = [], 0
    for v in sizes:
        at.append(total)
        total += -(-v // ALIGN) * ALIGN
    flat = {k: torch.zeros(total, device="cuda") for k in ("p", "g", "m", "v")}
    scale = LOSS_SCALE if case["clip"] else 1.0
    std = 10.0 ** (torch.rand((len(sizes),), generator=g, device="cuda") * 2 - 4).cpu()
    for o, v, sd in zip(at, sizes, std.tolist()):
        flat["p"][o:o + v].normal_(0, 1 / case["channels"], generator=g)
        flat["g"][o:o + v].normal_(0, sd * scale, generator=g)
        flat["m"][o:o + v].normal_(0, 0.2 * sd, generator=g)
        flat["v"][o:o + v].normal_(0, sd, generator=g)
        flat["v"][o:o + v].square_().add_(0.05 * sd * sd)
    s = {"case": case, "at": at, "sizes": sizes, "grad": flat["g"], "step": STEPS}
    if case["param"] == "fp32":
        s["param"] = flat["p"]
    else:
        s["param"], s["master"] = flat["p"].to(DTYPES[case["param"]]), flat["p"]
    if case["bits"] == 8:
        q = _encode(flat["m"].view(-1, 256), flat["v"].sqrt().view(-1, 256))
        s["exp_avg"], s["exp_avg_sq"] = q[0].view(-1), q[1].view(-1)
        s["exp_avg_scale"], s["exp_avg_sq_scale"] = q[2].view(-1), q[3].view(-1)
    else:
        s["exp_avg"], s["exp_avg_sq"] = flat["m"], flat["v"]
    return s


def prepare(case, seed):
    return (_prepare_adamw if case["do"] == "adamw" else _prepare_norm)(case, seed)


# ---------------------------------------------------------------------------
# One pass: the plain forms
# ---------------------------------------------------------------------------
def _phi(z):
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


def _plain_fwd(s):
    case = s["case"]
    b, c, g = case["batch"], case["channels"], case["groups"]
    x = _rows(s["x"].float(), case["last"])
    v = x.reshape(b, g, -1)
    mean = v.mean(2, keepdim=True)
    rstd = torch.rsqrt((v - mean).square().mean(2, keepdim=True) + EPS)
    z = ((v - mean) * rstd).view(b, c, -1) * s["gamma"].view(1, c, 1) + s["beta"].view(1, c, 1)
    out = {"gelu": lambda: z * _phi(z), "silu": lambda: z * torch.sigmoid(z),
           "none": lambda: z}[case["act"]]()
    if case["residual"]:
        out = out + _rows(s["residual"].float(), case["last"])
    out = out.transpose(1, 2) if case["last"] else out
    out = out.to(s["x"].dtype).reshape(s["x"].shape)
    return {"out": out, "stats": torch.cat([mean, rstd], 2)}


def _plain_bwd(s):
    case = s["case"]
    b, c, g = case["batch"], case["channels"], case["groups"]
    mean, rstd = s["stats"][:, :, :1], s["stats"][:, :, 1:]
    x = _rows(s["x"].float(), case["last"]).reshape(b, g, -1)
    xh = ((x - mean) * rstd).view(b, c, -1)
    gamma = s["gamma"].view(1, c, 1)
    z = xh * gamma + s["beta"].view(1, c, 1)
    h = _rows(s["g_out"].float(), case["last"])
    if case["act"] == "gelu":
        h = h * (_phi(z) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)))
    elif case["act"] == "silu":
        sg = torch.sigmoid(z)
        h = h * (sg * (1 + z * (1 - sg)))
    g_gamma, g_beta = (h * xh).sum((0, 2)), h.sum((0, 2))
    h = (h * gamma).reshape(b, g, -1)
    xh = xh.reshape(b, g, -1)
    gx = rstd * (h - h.mean(2, keepdim=True) - xh * (h * xh).mean(2, keepdim=True))
    gx = gx.view(b, c, -1)
    gx = gx.transpose(1, 2) if case["last"] else gx
    gx = gx.to(s["x"].dtype).reshape(s["x"].shape)
    return {"gx": gx, "g_gamma": g_gamma, "g_beta": g_beta}


def _plain_adamw(s):
    """The step over the flat buffers, in place (between the tensors they hold
    zeros, which it leaves zero)."""
    case = s["case"]
    s["step"] += 1
    b1, b2 = BETAS
    size = LR / (1 - b1 ** s["step"])
    root = 1 / math.sqrt(1 - b2 ** s["step"])
    out, g = {}, s["grad"]
    if case["clip"]:
        norm = torch.sqrt(g.square().sum()) * (1 / LOSS_SCALE)
        g = g * (torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0) * (1 / LOSS_SCALE))
        out["norm"] = norm
    p = s["param"] if case["param"] == "fp32" else s["master"]
    m, v = s["exp_avg"], s["exp_avg_sq"]
    if case["bits"] == 8:
        m, v = _decode(m.view(-1, 256), v.view(-1, 256), s["exp_avg_scale"].view(-1, 1),
                       s["exp_avg_sq_scale"].view(-1, 1))
        m, v = m.view(-1), v.view(-1)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    w = torch.sqrt(v)
    p.copy_(p * (1 - LR * DECAY) - (m * size) / (w * root + OPT_EPS))
    if case["bits"] == 8:
        q = _encode(m.view(-1, 256), w.view(-1, 256))
        for k, t in zip(("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"), q):
            s[k].copy_(t.view(-1))
        m, v = _decode(*q)
        # states of eight bits come back as the values that they stand for
        out["exp_avg"], out["exp_avg_sq"] = m.view(-1).bfloat16(), v.view(-1).bfloat16()
    else:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
        out["exp_avg"], out["exp_avg_sq"] = s["exp_avg"], s["exp_avg_sq"]
    if case["param"] != "fp32":
        s["param"].copy_(p)
        out["master"] = p
    out["param"] = s["param"]
    return out


# ---------------------------------------------------------------------------
# One pass: this package's calls
# ---------------------------------------------------------------------------
def _own_norm(s):
    """The handle a program keeps for a shape."""
    from paper_2307_15034_amd import binding as B
    from paper_2307_15034_amd.layer import GroupNormAct
    case = s["case"]
    act = {"none": B.FNO_NORM_ACT_NONE, "gelu": B.FNO_NORM_ACT_GELU,
           "silu": B.FNO_NORM_ACT_SILU}[case["act"]]
    return GroupNormAct(_grid(case), case["batch"], case["channels"], case["groups"],
                        dtype=s["x"].dtype, activation=act, channels_last=case["last"], eps=EPS)


def _own_adamw(s):
    """The optimizer a program keeps for its model, taking up its states."""
    from paper_2307_15034_amd.optim import AdamW
    case = s["case"]

    def views(t, per=1):
        return [t[o // per:o // per - (-v // per)] for o, v in zip(s["at"], s["sizes"])]

    keys = {"exp_avg": 1, "exp_avg_sq": 1}
    if case["bits"] == 8:
        keys.update(exp_avg_scale=256, exp_avg_sq_scale=256)
        for k in ("exp_avg", "exp_avg_sq"):  # where the states' values are read to
            s[k + "_out"] = torch.zeros(s[k].numel(), dtype=torch.bfloat16, device="cuda")
        s["moments_out"] = (views(s["exp_avg_out"]), views(s["exp_avg_sq_out"]))
    cols = {k: views(s[k], per) for k, per in keys.items()}
    states = [{k: cols[k][i] for k in keys} for i in range(len(s["at"]))]
    return AdamW(views(s["param"]), views(s["grad"]),
                 masters=None if case["param"] == "fp32" else views(s["master"]),
                 states=states, lr=LR, betas=BETAS, eps=OPT_EPS, weight_decay=DECAY,
                 state_bits=case["bits"], step=s["step"], device_control=case["clip"])


def _own_pass(s):
    case = s["case"]
    if "op" not in s:
        s["op"] = _own_adamw(s) if case["do"] == "adamw" else _own_norm(s)
    op = s["op"]
    if case["do"] == "norm_fwd":
        out, stats = op.fwd(s["x"], s["gamma"], s["beta"], residual=s.get("residual"))
        return {"out": out, "stats": stats}
    if case["do"] == "norm_bwd":
        gx, g_gamma, g_beta = op.bwd(s["x"], s["g_out"], s["stats"], s["gamma"], s["beta"])
        return {"gx": gx, "g_gamma": g_gamma, "g_beta": g_beta}
    out = {"param": s["param"]}
    if case["clip"]:
        out["norm"] = op.clip_grads(MAX_NORM, loss_scale=LOSS_SCALE)
    op.step()
    if case["bits"] == 8:
        op.moments(*s["moments_out"])
        out["exp_avg"], out["exp_avg_sq"] = s["exp_avg_out"], s["exp_avg_sq_out"]
    else:
        out["exp_avg"], out["exp_avg_sq"] = s["exp_avg"], s["exp_avg_sq"]
    if case["param"] != "fp32":
        out["master"] = s["master"]
    return out


def run(state):
    if own:
        return _own_pass(state)
    return {"norm_fwd": _plain_fwd, "norm_bwd": _plain_bwd,
            "adamw": _plain_adamw}[state["case"]["do"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Bytes: each input read once, each output written once.  The norm's
    forward reads x (and the residual) and writes out; its backward reads x
    and g_out and writes gx.  The step reads the gradient, the fp32 parameter
    (or master) and both moments and writes parameter, master and moments;
    8-bit states carry two scales per 256 elements and are read out as two
    16-bit values.  Operations: about what the formulas count per element."""
    if case["do"] == "adamw":
        n = sum(_sizes(case))
        each = 4 + 8 + (0 if case["param"] == "fp32" else 2)
        each += 4 + 4 + 16 / 256.0 if case["bits"] == 8 else 16
        return {"bytes": n * each, "flops": n * (16.0 + 2 * case["clip"])}
    es = 4 if case["dtype"] == "fp32" else 2
    c = case["channels"]
    n = case["batch"] * math.prod(_grid(case)) * c
    tensors = 3 if case["do"] == "norm_bwd" or case["residual"] else 2
    small = 16 * c + 8 * case["batch"] * case["groups"]
    act = {"none": 0, "gelu": 12, "silu": 6}[case["act"]]
    return {"bytes": n * es * tensors + small,
            "flops": n * (16.0 + act) if case["do"] == "norm_bwd" else n * (8.0 + act)}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _exact_norm(case, s):
    """torch's own norm and activations in float64, one sample at a time;
    the gradients by automatic differentiation (the statistics are functions
    of x)."""
    F = torch.nn.functional
    act = {"gelu": F.gelu, "silu": F.silu, "none": lambda v: v}[case["act"]]
    last, bwd = case["last"], case["do"] == "norm_bwd"
    gamma = s["gamma"].double().requires_grad_(bwd)
    beta = s["beta"].double().requires_grad_(bwd)
    outs, stats, gg, gb = [], [], 0, 0
    for b in range(case["batch"]):
        x = s["x"][b:b + 1].double()
        x = x.movedim(-1, 1) if last else x
        x = x.contiguous().requires_grad_(bwd)
        y = act(F.group_norm(x, case["groups"], gamma, beta, EPS))
        if bwd:
            g = s["g_out"][b:b + 1].double()
            r = torch.autograd.grad(y, (x, gamma, beta), g.movedim(-1, 1) if last else g)
            y, gg, gb = r[0], gg + r[1], gb + r[2]
        else:
            v = x.reshape(1, case["groups"], -1)
            var, mean = torch.var_mean(v, 2, unbiased=False)
            stats.append(torch.stack([mean, 1 / torch.sqrt(var + EPS)], 2))
        y = y.movedim(1, -1) if last else y
        outs.append(y + s["residual"][b:b + 1].double() if case["residual"] else y)
    if bwd:
        return {"gx": torch.cat(outs), "g_gamma": gg, "g_beta": gb}
    return {"out": torch.cat(outs), "stats": torch.cat(stats)}


def _exact_adamw(case, s):
    d = torch.float64
    t = s["step"] + 1
    g, out = s["grad"].to(d), {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g) / LOSS_SCALE
        g = g / LOSS_SCALE * torch.clamp(MAX_NORM / norm, max=1)
        out["norm"] = norm
    p = (s["param"] if case["param"] == "fp32" else s["master"]).to(d)
    m, v = s["exp_avg"].to(d), s["exp_avg_sq"].to(d)
    if case["bits"] == 8:
        def spread(k):
            return s[k].to(d).repeat_interleave(256)
        m = spread("exp_avg_scale") * m.sign() * (m / 127) ** 2
        v = (spread("exp_avg_sq_scale") * (v / 255) ** 2) ** 2
    b1, b2 = BETAS
    m.mul_(b1).add_(g, alpha=1 - b1)
    v.mul_(b2).addcmul_(g, g, value=1 - b2)
    del g
    p *= 1 - LR * DECAY
    p -= LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + OPT_EPS)
    if case["bits"] == 8:
        def code(x, levels):
            top = x.view(-1, 256).amax(1).clamp_min(1e-300).repeat_interleave(256)
            return torch.round(levels * torch.sqrt(x / top)), top
        q, top = code(m.abs(), 127)
        m = m.sign() * top * (q / 127) ** 2
        q, top = code(v.sqrt(), 255)
        v = (top * (torch.where(v > 0, q.clamp_min(1), q) / 255) ** 2) ** 2
    out.update(exp_avg=m, exp_avg_sq=v, param=p)
    if case["param"] != "fp32":
        out["master"] = p
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.set_grad_enabled(case["do"] == "norm_bwd"):
        return (_exact_adamw if case["do"] == "adamw" else _exact_norm)(case, s)
