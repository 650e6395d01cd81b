"""Trains one normalised FNO block on the GPU with this library's kernels alone:

    out = gelu( group_norm( W_skip x + b + K x ) ) + x

K the spectral convolution (fp16 weights beside fp32 masters), the skip path,
the norm with its activation and the residual, their backward, the global
gradient norm with clip and loss scale, and AdamW with its states in 32 or in
8 bits.  torch holds the memory and forms the loss.  The block learns a block
of the same shape with other weights on smooth random fields (synthetic data).

    python3 examples/train_norm_block.py --steps 100 --state-bits 8
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import synth  # noqa: E402
from paper_2307_15034_amd import binding as B  # noqa: E402
from paper_2307_15034_amd.layer import BlockEpilogue, GroupNormAct, SpectralConv  # noqa: E402
from paper_2307_15034_amd.optim import AdamW  # noqa: E402


class NormBlock:
    """One block with its parameters: "w" (dense spectral weights, fp16 pairs),
    "skip", "bias" (fp16), "gamma", "beta" (fp32)."""

    def __init__(self, wl, batch, groups, seed):
        self.layer = SpectralConv(wl.n, wl.modes, batch, wl.c_in, wl.c_out)
        self.epi = BlockEpilogue(wl.n, batch, wl.c_in, wl.c_out, activation=B.FNO_EPI_ACT_NONE)
        self.norm = GroupNormAct(wl.n, batch, wl.c_out, groups, activation=B.FNO_NORM_ACT_GELU)
        self.x_hat = self.layer.spectrum_buffer(0)
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        c = wl.c_in
        self.params = {
            "w": (r(wl.c_in, wl.c_out, *self.layer.kdims, 2) / c).half(),
            "skip": (r(wl.c_out, wl.c_in) / c ** 0.5).half(),
            "bias": torch.zeros(wl.c_out, dtype=torch.float16, device="cuda"),
            "gamma": torch.ones(wl.c_out, device="cuda"),
            "beta": 0.2 * r(wl.c_out),
        }

    def forward(self, x):
        p = self.params
        y = self.layer.fwd(x, p["w"], x_hat=self.x_hat)
        z, _ = self.epi.fwd(x, y, p["skip"], p["bias"])
        out, stats = self.norm.fwd(z, p["gamma"], p["beta"], residual=x)
        return out, (x, z, stats)

    def backward(self, kept, g_out):
        """The parameters' gradients (fp32) and the input's."""
        x, z, stats = kept
        p = self.params
        g_z, g_gamma, g_beta = self.norm.bwd(z, g_out, stats, p["gamma"], p["beta"])
        _, g_skip, g_bias = self.epi.bwd_weight(x, None, g_z)
        g_spec, g_w = self.layer.bwd(x, p["w"], g_z, x_hat=self.x_hat)
        g_x = self.epi.bwd_data(g_z, p["skip"], g_spec, gx=g_spec)
        grads = {"w": g_w, "skip": g_skip, "bias": g_bias, "gamma": g_gamma, "beta": g_beta}
        return grads, g_x + g_out  # the residual's share


def train(steps=100, state_bits=8, batch=8, lr=2e-2, loss_scale=256.0, max_norm=100.0, seed=0,
          say=print):
    """The losses (mean squared error) of `steps` steps, one float each; the
    gradient is the squared error's, summed over a sample and averaged over
    the batch."""
    wl = synth.WORKLOADS[1]  # 64 x 64, 16 channels
    x = torch.from_numpy(synth.make_x(wl, np.float16, batch)).cuda()
    target, _ = NormBlock(wl, batch, 4, seed + 100).forward(x)
    net = NormBlock(wl, batch, 4, seed)
    names = list(net.params)
    params = [net.params[k] for k in names]
    opt = None
    losses = []
    for step in range(steps):
        out, kept = net.forward(x)
        diff = out.float() - target.float()
        losses.append(diff.square().mean())
        g_out = (diff * (2.0 * loss_scale / batch)).half()
        grads, _ = net.backward(kept, g_out)
        grads = [grads[k] for k in names]
        if opt is None:  # weights decay, biases and norm parameters do not; few elements: 32 bits
            opt = AdamW(params, grads, masters=AdamW.make_masters(params), lr=lr,
                        weight_decay=[1e-4 if k in ("w", "skip") else 0.0 for k in names],
                        state_bits=[state_bits if k in ("w", "skip") else 32 for k in names],
                        device_control=True)
        else:
            opt.set_grads(grads)
        opt.clip_grads(max_norm, loss_scale)
        opt.step()
        if say and (step % 20 == 0 or step == steps - 1):
            say(f"step {step:4d}  loss {float(losses[-1]):.5f}  "
                f"gradient norm {opt.read_control()['grad_norm']:.4f}")
    return torch.stack(losses).cpu().tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--state-bits", type=int, choices=[8, 32], default=8)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--lr", type=float, default=2e-2)
    a = ap.parse_args()
    train(a.steps, a.state_bits, a.batch, a.lr)
