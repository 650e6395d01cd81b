"""Channel mixing in 8-bit floating point, and the norms around a block, as
timed cases.

"mix_fwd"   a linear map over channels, y = Q(act(x)) Q(W)^T + bias: x rounded to
            8-bit codes with one scale for each 128 consecutive channels of a
            row, W to codes with one scale for each 128 x 128 tile; for training
            the codes of act(x)^T (scales along the rows) are kept
"mix_bwd"   its backward: g rounded in both directions, gx = Q(g) Q(W) (times
            act'(x)), gW = Q(g^T) Q(act(x)^T)^T and the bias's gradient
"mix_pack"  the weights' codes and scales, in both orders, as after each step of
            the optimizer
"norm_fwd"  between two blocks: y = scale x + gate norm(u), h = norm(y); u the
            block's output, x the residual stream, h the next block's input
            (also "entry", h = norm(x), and "exit", y alone)
"norm_bwd"  its backward: the gradients of u, x and of every parameter

Codes are e4m3 (e5m2 for gradients).  A block's scale is the least power of two
that brings its largest size within the format's, or that size over the
format's as an fp32 number ("f32").

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
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
BLOCK = 128
EPS = 1e-5


def _mix(name, do, rows, c_in, c_out, dtype="fp16", scale="pow2", act="none", bias=True,
         keep=False):
    c = {"do": do, "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "scale": scale,
         "act": act, "bias": bias, "keep": keep}
    if name:
        c["name"] = name
    return c


def _norm(name, do, batch, points, channels, dtype="fp16", kind="layer", form="both",
          gate="none", scale=False, bias=True):
    """gate: "none", "shared" [1, C], "sample" [batch, C] or "row" (a tensor)."""
    c = {"do": do, "batch": batch, "points": points, "channels": channels, "dtype": dtype,
         "kind": kind, "form": form, "gate": gate, "scale": scale, "bias": bias}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One row through a wide map: latency, and the weights' bytes.
        _mix("mix-fwd-1", "mix_fwd", 1, 4096, 4096, "bf16"),
        # The pointwise network behind the Navier-Stokes block: 64 channels to
        # four times as many, all points of 32 samples of 128 x 128, training.
        _mix("mix-fwd-128", "mix_fwd", 32 * 128 * 128, 64, 256, keep=True),
        # The way back of such a network, GELU before it, fp32 scales, ragged.
        _mix("mix-fwd-gelu", "mix_fwd", 10007, 1000, 520, "bf16", "f32", "gelu"),
        # The largest: the matrix cores' rate.
        _mix("mix-fwd-4096", "mix_fwd", 16384, 4096, 4096, "bf16", bias=False),
        # An odd grid (data on node grids) with 20 channels: rows of 40 bytes,
        # blocks that end inside a row.
        _mix("mix-bwd-odd", "mix_bwd", 16 * 241 * 241, 20, 80),
        # A training step of a wide network.
        _mix("mix-bwd-4096", "mix_bwd", 8192, 4096, 4096, "bf16", act="silu"),
        # The weights of one wide map behind the optimizer's step.
        _mix("mix-pack", "mix_pack", 1, 4096, 16384, "bf16"),
        # One row between two blocks: latency.
        _norm("norm-fwd-1", "norm_fwd", 1, 1, 4096, "bf16", "rms", gate="shared", bias=False),
        # Between two blocks of the Navier-Stokes operator, gates by sample
        # (conditioning), a learned scale on the residual.
        _norm("norm-fwd-128", "norm_fwd", 32, 128 * 128, 64, gate="sample", scale=True),
        _norm("norm-bwd-128", "norm_bwd", 32, 128 * 128, 64, gate="sample", scale=True),
        # Wide rows, RMS, one learned gate.
        _norm("norm-bwd-wide", "norm_bwd", 4, 2048, 4096, "bf16", "rms", gate="shared", bias=False),
        # The odd grid in full precision, rows of 80 bytes.
        _norm("norm-bwd-odd", "norm_bwd", 16, 241 * 241, 20, "fp32"),
    ]


# ---------------------------------------------------------------------------
# Other cases of the same ranges
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["mix_fwd", "mix_fwd", "mix_bwd", "mix_bwd", "mix_pack", "norm_fwd",
                     "norm_fwd", "norm_bwd", "norm_bwd"])
    dtype = rng.choice(["fp16", "bf16", "bf16", "fp32"])
    if do.startswith("mix"):
        def width():
            v = _log(rng, 8, 4096)
            how = rng.random()
            return max(8, v // 64 * 64) if how < 0.5 else v // 8 * 8 if how < 0.75 else v
        c_in, c_out = width(), width()
        most = min(1 << 20, (16384 << 24) // (2 * c_in * c_out), (1 << 27) // (c_in + c_out))
        rows = 1 if do == "mix_pack" else _log(rng, 1, max(1, most))
        if rng.random() < 0.4:
            rows = max(1, rows // 128 * 128)
        # fp32 results behind an activation would hang on codes next to a border
        act = "none" if dtype == "fp32" or do == "mix_pack" else rng.choice(["none", "gelu", "silu"])
        return _mix(None, do, rows, c_in, c_out, dtype, rng.choice(["pow2", "pow2", "f32"]), act,
                    do != "mix_pack" and rng.random() < 0.5,
                    do == "mix_fwd" and rng.random() < 0.5)
    channels = _log(rng, 8, 8192)
    if rng.random() < 0.5:
        channels = max(16, channels // 16 * 16)
    total = _log(rng, channels, 1 << 25) // channels
    batch = _log(rng, 1, max(1, min(32, total)))
    form = rng.choice(["both", "both", "both", "entry", "exit"])
    return _norm(None, do, batch, max(1, total // batch), channels, dtype,
                 rng.choice(["layer", "rms"]), form,
                 "none" if form == "entry" else rng.choice(["none", "shared", "sample", "row"]),
                 form != "entry" and rng.random() < 0.4, rng.random() < 0.6)


# ---------------------------------------------------------------------------
# 8-bit codes, in 32 bits
# ---------------------------------------------------------------------------
def _top(fmt):
    return 448.0 if fmt == E4M3 else 57344.0


def _two32(e):
    """2^e of whole numbers e, -126 to 127, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _act32(x, act):
    if act == "gelu":
        return x * (0.5 * (1 + torch.erf(x * math.sqrt(0.5))))
    return x * torch.sigmoid(x) if act == "silu" else x


def _act_grad32(x, act):
    if act == "gelu":
        return (0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
                + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi)))
    s = torch.sigmoid(x)
    return s * (1 + x * (1 - s))


def _blocks(v, tile):
    """v [R, C] padded with zeros to whole blocks: [R', C'/128, 128] (rows), or
    [R'/128, 128, C'/128, 128] (tiles)."""
    r, c = v.shape
    v = torch.nn.functional.pad(v, (0, -c % BLOCK, 0, -r % BLOCK if tile else 0))
    return v.view(-1, BLOCK, v.shape[1] // BLOCK, BLOCK) if tile else v.view(r, -1, BLOCK)


def _codes(v, fmt, scale, tile=False):
    """Codes [R, C rounded up to 16] (zeros behind C) and scales [C / 128, R]
    ([C / 128, R / 128] by tiles) of v [R, C] fp32."""
    r, c = v.shape
    b = _blocks(v, tile)
    a = b.abs().amax((1, 3) if tile else 2)
    if scale == "pow2":
        m, e = torch.frexp(a)  # top = 0.875 2^9 (e4m3), 0.875 2^16 (e5m2)
        e = (e - (9 if fmt == E4M3 else 16) + (m > 0.875)).clamp(-126, 127)
        s = torch.where(a > 0, _two32(e), 1.0)
    else:
        s = torch.where(a > 0, (a / _top(fmt)).clamp_min(2.0 ** -126), 1.0)
    inv = 1 / s
    b = b * (inv[:, None, :, None] if tile else inv[:, :, None])
    q = b.view(-1, s.shape[1] * BLOCK)[:r, :c]
    q = torch.nn.functional.pad(q, (0, -c % 16)).to(fmt)
    s = s.t().contiguous()
    return q, s.to(E8M0) if scale == "pow2" else s


def _values(q, s, c, tile=False):
    """What codes and scales stand for: [R, C] fp32."""
    r = q.shape[0]
    s = s.float().t()
    if tile:
        s = s.repeat_interleave(BLOCK, 0)[:r]
    return q.float()[:, :c] * s.repeat_interleave(BLOCK, 1)[:, :c]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _prepare_mix(case, seed):
    """Activations whose channels have spreads of their own and some values far
    out; output gradients of rows of sizes far apart, a few rows masked (zero);
    the weights as the program keeps them, in codes."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = dict(device="cuda", generator=g)
    m, k, n, dt = case["rows"], case["c_in"], case["c_out"], DTYPES[case["dtype"]]
    w = torch.randn((n, k), **rand) * (torch.rand((n, 1), **rand) + 0.5) / math.sqrt(k)
    s = {"case": case}
    if case["do"] == "mix_pack":
        s["w"] = w.to(dt)
        return s
    x = torch.randn((m, k), **rand) * (torch.rand((k,), **rand) * 2 + 0.1)
    x = torch.where(torch.rand((m, k), **rand) < 1e-3, x * 20, x).to(dt)
    s["w"] = _codes(w, E4M3, case["scale"], True)
    if case["do"] == "mix_fwd":
        s["x"] = x
        s["bias"] = torch.randn((n,), **rand) if case["bias"] else None
        return s
    s["wt"] = _codes(w.t().contiguous(), E4M3, case["scale"], True)
    s["kept"] = _codes(_act32(x.float(), case["act"]).t().contiguous(), E4M3, case["scale"])
    s["x"] = x if case["act"] != "none" else None
    size = torch.exp(torch.randn((m, 1), **rand)) * 1e-2
    size = torch.where(torch.rand((m, 1), **rand) < 0.05, 0.0, size)
    s["g"] = (torch.randn((m, n), **rand) * size).to(dt)
    return s


def _prepare_norm(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = dict(device="cuda", generator=g)
    b, c, dt = case["batch"], case["channels"], DTYPES[case["dtype"]]
    rows = b * case["points"]
    spread, offset = torch.rand((c,), **rand) + 0.5, torch.randn((c,), **rand)

    def noise():
        return torch.randn((rows, c), **rand)

    def param():
        return 1 + 0.2 * torch.randn((c,), **rand), (
            0.2 * torch.randn((c,), **rand) if case["bias"] else None)

    s = {"case": case, "x": (noise() + offset).to(dt)}
    if case["form"] != "entry":
        s["u"] = (noise() * spread + offset).to(dt)
        s["post_w"], s["post_b"] = param()
        s["scale"] = 1 + 0.1 * torch.randn((c,), **rand) if case["scale"] else None
        many = {"none": 0, "shared": 1, "sample": b, "row": rows}[case["gate"]]
        s["gate"] = 0.5 + 0.5 * torch.randn((many, c), **rand) if many else None
        if case["gate"] == "row":
            s["gate"] = s["gate"].to(dt)
    if case["form"] != "exit":
        s["pre_w"], s["pre_b"] = param()
    if case["do"] == "norm_bwd":
        if case["form"] == "both":  # the stream as the forward left it
            s["y"] = _stream(s)[0].to(dt)
        s["g_y"] = (noise() * 0.1).to(dt)
        if case["form"] != "exit":
            s["g_h"] = (noise() * (torch.rand((rows, 1), **rand) < 0.95)).to(dt)
    return s


def prepare(case, seed):
    return (_prepare_mix if case["do"].startswith("mix") else _prepare_norm)(case, seed)


# ---------------------------------------------------------------------------
# One pass: the plain forms
# ---------------------------------------------------------------------------
def _plain_mix(s):
    case = s["case"]
    k, n, scale = case["c_in"], case["c_out"], case["scale"]
    if case["do"] == "mix_pack":
        w = s["w"].float()
        q, a = _codes(w, E4M3, scale, True)
        qt, at = _codes(w.t(), E4M3, scale, True)
        return {"codes": q, "scale": a, "codes_t": qt, "scale_t": at}
    if case["do"] == "mix_fwd":
        x = _act32(s["x"].float(), case["act"])
        y = _values(*_codes(x, E4M3, scale), k) @ _values(*s["w"], k, True).t()
        if s["bias"] is not None:
            y = y + s["bias"]
        out = {"y": y.to(s["x"].dtype)}
        if case["keep"]:
            out["codes"], out["scale"] = _codes(x.t(), E4M3, scale)
        return out
    g, m = s["g"].float(), case["rows"]
    gx = _values(*_codes(g, E5M2, scale), n) @ _values(*s["wt"], n, True).t()
    if case["act"] != "none":
        gx = gx * _act_grad32(s["x"].float(), case["act"])
    gw = _values(*_codes(g.t(), E5M2, scale), m) @ _values(*s["kept"], m).t()
    out = {"gx": gx.to(s["g"].dtype), "gw": gw}
    if case["bias"]:
        out["gb"] = g.sum(0)
    return out


def _unit(v, kind):
    """(v - mean) / deviation by rows, and 1 / deviation."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * r, r


def _affine(v, w, b):
    return v * w if b is None else v * w + b


def _gate(s):
    """The gate of every row, [rows, C] or broadcast."""
    g, case = s["gate"], s["case"]
    if case["gate"] != "sample":
        return g.float()
    return g.repeat_interleave(case["points"], 0)


def _stream(s):
    """y in 32 bits, norm(u) and the normalised u with its 1 / deviation."""
    xh, r = _unit(s["u"].float(), s["case"]["kind"])
    n = _affine(xh, s["post_w"], s["post_b"])
    x = s["x"].float()
    y = (x if s["scale"] is None else x * s["scale"]) + (n if s["gate"] is None else n * _gate(s))
    return y, n, xh, r


def _plain_norm_fwd(s):
    case, dt, out = s["case"], s["x"].dtype, {}
    y = s["x"].float()
    if case["form"] != "entry":
        y = _stream(s)[0]
        out["y"] = y.to(dt)
    if case["form"] != "exit":
        out["h"] = _affine(_unit(y, case["kind"])[0], s["pre_w"], s["pre_b"]).to(dt)
    return out


def _unit_bwd(h, xh, r, kind):
    """The gradient of a row from that of its normalised values, h."""
    v = h - xh * (h * xh).mean(1, keepdim=True)
    if kind == "layer":
        v = v - h.mean(1, keepdim=True)
    return v * r


def _plain_norm_bwd(s):
    case, dt, out = s["case"], s["x"].dtype, {}
    kind = case["kind"]
    g = s["g_y"].float()
    if case["form"] != "exit":
        gh = s["g_h"].float()
        xh, r = _unit((s["y"] if case["form"] == "both" else s["x"]).float(), kind)
        out["g_pre_w"] = (gh * xh).sum(0)
        if case["bias"]:
            out["g_pre_b"] = gh.sum(0)
        g = g + _unit_bwd(gh * s["pre_w"], xh, r, kind)
    if case["form"] == "entry":
        out["g_x"] = g.to(dt)
        return out
    xh, r = _unit(s["u"].float(), kind)
    if case["scale"]:
        out["g_scale"] = (g * s["x"].float()).sum(0)
    out["g_x"] = (g * s["scale"] if case["scale"] else g).to(dt)
    if s["gate"] is not None:
        d = g * _affine(xh, s["post_w"], s["post_b"])
        if case["gate"] == "row":
            out["g_gate"] = d.to(dt)
        else:
            out["g_gate"] = d.view(s["gate"].shape[0], -1, case["channels"]).sum(1)
        g = g * _gate(s)
    out["g_post_w"] = (g * xh).sum(0)
    if case["bias"]:
        out["g_post_b"] = g.sum(0)
    out["g_u"] = _unit_bwd(g * s["post_w"], xh, r, kind).to(dt)
    return out


# ---------------------------------------------------------------------------
# One pass: this package's calls
# ---------------------------------------------------------------------------
def _own_mix(s):
    from paper_2307_15034_amd import binding as B
    from paper_2307_15034_amd.fp8 import Fp8Codes, Fp8Linear, Fp8Weights
    case = s["case"]
    if "op" not in s:
        act = {"none": B.FNO_NORM_ACT_NONE, "gelu": B.FNO_NORM_ACT_GELU,
               "silu": B.FNO_NORM_ACT_SILU}[case["act"]]
        s["op"] = Fp8Linear(case["rows"], case["c_in"], case["c_out"], DTYPES[case["dtype"]],
                            activation=act, pow2_scales=case["scale"] == "pow2")
        if case["do"] != "mix_pack":
            s["weights"] = Fp8Weights(*s["w"], *s.get("wt", (None, None)))
        if case["do"] == "mix_bwd":
            s["codes"] = Fp8Codes(*s["kept"])
    op = s["op"]
    if case["do"] == "mix_pack":
        return op.pack(s["w"])._asdict()
    if case["do"] == "mix_fwd":
        y, kept = op.fwd(s["x"], s["weights"], s["bias"], keep=case["keep"])
        return {"y": y, "codes": kept.codes, "scale": kept.scale} if case["keep"] else {"y": y}
    gx, gw, gb = op.bwd(s["g"], s["weights"], s["codes"], s["x"], bias=case["bias"])
    return {"gx": gx, "gw": gw, "gb": gb} if case["bias"] else {"gx": gx, "gw": gw}


def _own_norm(s):
    from paper_2307_15034_amd import binding as B
    from paper_2307_15034_amd.layer import ResidualNorm
    case = s["case"]
    if "op" not in s:
        s["op"] = ResidualNorm(case["batch"] * case["points"], case["channels"],
                               DTYPES[case["dtype"]],
                               B.FNO_ROW_NORM_LAYER if case["kind"] == "layer"
                               else B.FNO_ROW_NORM_RMS, eps=EPS)
    op = s["op"]
    par = {k: s.get(k) for k in ("post_w", "post_b", "gate", "scale", "pre_w", "pre_b")}
    if case["do"] == "norm_fwd":
        y, h = op.fwd(s["x"], s.get("u"), pre=case["form"] != "exit", **par)
        return {k: v for k, v in (("y", y), ("h", h)) if v is not None and (k, case["form"]) != ("y", "entry")}
    got = op.bwd(s.get("g_y"), s.get("g_h"), x=s["x"], u=s.get("u"), y=s.get("y"), **par)
    return {k: v for k, v in got.items() if v is not None}


def run(state):
    do = state["case"]["do"]
    if own:
        return (_own_mix if do.startswith("mix") else _own_norm)(state)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd}.get(do, _plain_mix)(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Bytes: each input read once, each output written once; codes take one
    byte, their scales one or four for 128 codes.  Operations: the products',
    and about what the formulas count per element."""
    es = 4 if case["dtype"] == "fp32" else 2
    if case["do"].startswith("mix"):
        m, k, n = case["rows"], case["c_in"], case["c_out"]
        one = 1 + (1 if case["scale"] == "pow2" else 4) / 128.0  # a code with its share of a scale
        if case["do"] == "mix_pack":
            return {"bytes": n * k * (es + 2.0), "flops": n * k * 4.0}
        if case["do"] == "mix_fwd":
            size = es * m * (k + n) + n * k + (one * m * k if case["keep"] else 0)
            return {"bytes": size + 4 * n * case["bias"], "flops": 2.0 * m * n * k}
        size = es * m * (n + k * (1 if case["act"] == "none" else 2)) + n * k + one * m * k
        return {"bytes": size + 4 * n * k + 4 * n * case["bias"], "flops": 4.0 * m * n * k}
    c, rows = case["channels"], case["batch"] * case["points"]
    bwd, both, row = case["do"] == "norm_bwd", case["form"] == "both", case["gate"] == "row"
    if case["form"] == "entry":
        tensors = 4 if bwd else 2      # x, g_y, g_h, g_x; x, h
    elif bwd:                          # u, g_y, g_u, g_x, and y, g_h, x, the gate and its gradient
        tensors = 4 + 2 * both + bool(case["scale"]) + 2 * row
    else:                              # u, x, y, and h, the gate
        tensors = 3 + both + row
    many = {"none": 0, "shared": 1, "sample": case["batch"], "row": 0}[case["gate"]]
    params = (2 if bwd else 1) * (many + (1 + case["bias"]) * (1 + both) + bool(case["scale"]))
    return {"bytes": es * tensors * rows * c + 4.0 * params * c,
            "flops": rows * c * (16.0 if bwd else 8.0) * (1 + both)}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _two64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round8(v, fmt):
    """v rounded to the nearest value of the format, ties to even."""
    bits, low = (3, -6) if fmt == E4M3 else (2, -14)
    e = torch.frexp(v)[1].clamp_min(low + 1) - 1 - bits
    unit = _two64(e)
    return torch.round(v / unit) * unit


def _exact_codes(v, fmt, scale, tile=False):
    """Codes' values and scales of v [R, C] (float64), one block column at a
    time.  fp32 scales, their reciprocals and the products with them are fp32
    numbers by definition."""
    r, c = v.shape
    q, scales = torch.zeros((r, c + -c % 16), dtype=torch.float64, device=v.device), []
    for j in range(0, c, BLOCK):
        b = v[:, j:j + BLOCK]
        a = b.abs().amax(1)
        if tile:
            a = torch.stack([p.amax() for p in a.split(BLOCK)])
        if scale == "pow2":
            s = _two64(torch.ceil(torch.log2(a / _top(fmt))).clamp(-1000, 1000))
            s = torch.where(a / s > _top(fmt), s * 2, s)
            s = torch.where(a / s <= _top(fmt) / 2, s / 2, s).clamp_min(2.0 ** -126)
        else:
            s = (a / _top(fmt)).float().double().clamp_min(2.0 ** -126)
        s = torch.where(a > 0, s, 1.0)
        scales.append(s)
        s = s.repeat_interleave(BLOCK)[:r] if tile else s
        t = b / s[:, None] if scale == "pow2" else (b * (1 / s).float().double()[:, None])
        q[:, j:j + b.shape[1]] = _round8(t if scale == "pow2" else t.float().double(), fmt)
    return q, torch.stack(scales)


def _exact_values(q, s, c, tile=False):
    """The same as float64 values, from codes of either kind."""
    out = q.double()[:, :c].clone()
    for j in range(0, c, BLOCK):
        f = s[j // BLOCK].double()
        out[:, j:j + BLOCK] *= (f.repeat_interleave(BLOCK)[:q.shape[0]] if tile else f)[:, None]
    return out


def _act64(x, act):
    return {"none": lambda v: v, "gelu": torch.nn.functional.gelu,
            "silu": torch.nn.functional.silu}[act](x)


def _exact_mix(case, s):
    k, n, m, scale = case["c_in"], case["c_out"], case["rows"], case["scale"]
    if case["do"] == "mix_pack":
        w = s["w"].double()
        q, a = _exact_codes(w, E4M3, scale, True)
        qt, at = _exact_codes(w.t(), E4M3, scale, True)
        return {"codes": q, "scale": a, "codes_t": qt, "scale_t": at}
    if case["do"] == "mix_fwd":
        x = _act64(s["x"].double(), case["act"])
        y = torch.nn.functional.linear(_exact_values(*_exact_codes(x, E4M3, scale), k),
                                       _exact_values(*s["w"], k, True))
        out = {"y": y if s["bias"] is None else y + s["bias"].double()}
        if case["keep"]:
            out["codes"], out["scale"] = _exact_codes(x.t(), E4M3, scale)
        return out
    g = s["g"].double()
    gx = torch.nn.functional.linear(_exact_values(*_exact_codes(g, E5M2, scale), n),
                                    _exact_values(*s["wt"], n, True))
    if case["act"] != "none":
        x = s["x"].double().requires_grad_()
        with torch.enable_grad():
            gx = gx * torch.autograd.grad(_act64(x, case["act"]).sum(), x)[0]
    gw = torch.nn.functional.linear(_exact_values(*_exact_codes(g.t(), E5M2, scale), m),
                                    _exact_values(*s["kept"], m))
    out = {"gx": gx, "gw": gw}
    if case["bias"]:
        out["gb"] = g.sum(0)
    return out


def _exact_norm(case, s):
    """Automatic differentiation of the definition; the second norm's backward
    at the stored y."""
    bwd = case["do"] == "norm_bwd"
    d = {k: v.double().requires_grad_(bwd) for k, v in s.items() if isinstance(v, torch.Tensor)}
    c = case["channels"]

    def norm(v, w, b):
        if case["kind"] == "layer":
            return torch.nn.functional.layer_norm(v, (c,), w, b, EPS)
        v = v / torch.sqrt(v.pow(2).mean(1, keepdim=True) + EPS) * w
        return v if b is None else v + b

    out, y = {}, d["x"]
    if case["form"] != "entry":
        n = norm(d["u"], d["post_w"], d.get("post_b"))
        if "gate" in d:
            n = (n.view(d["gate"].shape[0], -1, c) * d["gate"][:, None]).view(-1, c)
        y = out["y"] = (y * d["scale"] if "scale" in d else y) + n
    if not bwd:
        if case["form"] != "exit":
            out["h"] = norm(y, d["pre_w"], d.get("pre_b"))
        return out
    g, got = d["g_y"].detach(), {}
    if case["form"] != "exit":
        at = d["y"] if case["form"] == "both" else d["x"]
        names = ["pre_w"] + ["pre_b"] * ("pre_b" in d)
        r = torch.autograd.grad(norm(at, d["pre_w"], d.get("pre_b")), [at] + [d[p] for p in names],
                                d["g_h"].detach())
        g = g + r[0]
        got.update({"g_" + p: v for p, v in zip(names, r[1:])})
    if case["form"] == "entry":
        return {"g_x": g, **got}
    names = [p for p in ("x", "u", "post_w", "post_b", "gate", "scale") if p in d]
    r = torch.autograd.grad(y, [d[p] for p in names], g)
    return {**got, **{"g_" + p: v for p, v in zip(names, r)}}


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"].startswith("mix"):
        with torch.no_grad():
            return _exact_mix(case, s)
    with torch.set_grad_enabled(case["do"] == "norm_bwd"):
        return _exact_norm(case, s)
