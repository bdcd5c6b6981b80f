"""A transformer over the patches of a latent as the denoiser, from the library's operators.

    python examples/latent_transformer.py [--steps 150]

The model predicts the noise in a latent cut into patches: layer norms modulated by the timestep,
rotary positions over height and width, two-sided attention, the gated feed-forward product and dropout
with the residual's addition come from the library, the other matrix products from torch.  The program
trains it on toy latents (waves of a random direction) and samples a batch with the sequential chain and
with ParaDiGMS, where every point of a window has its own timestep, and so its own modulation.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2305_16317_amd as pd  # noqa: E402
from trajectory_transformer import Attend, sample  # noqa: E402


# ------------------------------------------------------------------ the operators under autograd
class Norm(torch.autograd.Function):
    """Layer norm of x [batch, token, width] times weight plus bias, [batch, width] each."""

    @staticmethod
    def forward(ctx, x, weight, bias):
        x = x.contiguous()
        y = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[:-1], device=x.device) for _ in range(2))
        pd.pd_layernorm_forward(x, y, weight=weight, bias=bias, mean=mean, rstd=rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx = torch.empty_like(x)
        dw, db = (torch.empty(weight.shape, device=x.device) for _ in range(2))
        pd.pd_layernorm_backward(dy.contiguous(), x, mean, rstd, dx, weight=weight, dweight=dw, dbias=db)
        return dx, dw, db


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, table, sections):
        ctx.save_for_backward(positions, table)
        ctx.sections = sections
        qo, ko = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        pd.pd_rotary_axes_apply(q, k, positions, table, sections, qo, ko)
        return qo, ko

    @staticmethod
    def backward(ctx, dq, dk):
        positions, table = ctx.saved_tensors
        dq, dk = dq.contiguous(), dk.contiguous()       # (not to be written: they may be another consumer's too)
        to_q, to_k = torch.empty_like(dq), torch.empty_like(dk)
        pd.pd_rotary_axes_apply(dq, dk, positions, table, ctx.sections, to_q, to_k, backward=True)
        return to_q, to_k, None, None, None


class Add(torch.autograd.Function):
    """residual + dropout(x); the gradient draws the mask again."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, site, step):
        ctx.how = (p, seed, site)
        ctx.save_for_backward(step.clone())            # (the caller's may be counted up before the gradient)
        y = torch.empty_like(residual)
        pd.pd_dropout_apply(x.contiguous(), y, p, seed, rng_stream=site, step_more=step, residual=residual.contiguous())
        return y

    @staticmethod
    def backward(ctx, dy):
        (p, seed, site), (step,) = ctx.how, ctx.saved_tensors
        dy = dy.contiguous()
        dx = torch.empty_like(dy)
        pd.pd_dropout_apply(dy, dx, p, seed, rng_stream=site, step_more=step)
        return dx, dy, None, None, None, None


class Gated(torch.autograd.Function):
    """act(x w_gate) * (x w_up); the product itself is formed again where its gradient needs it."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up):
        x = x.contiguous()
        h, gate, up = (torch.empty((*x.shape[:-1], w_gate.shape[1]), dtype=x.dtype, device=x.device) for _ in range(3))
        pd.pd_gated_forward(x, w_gate, w_up, h, gate=gate, up=up)
        ctx.save_for_backward(x, w_gate, w_up, gate, up)
        return h

    @staticmethod
    def backward(ctx, dh):
        x, w_gate, w_up, gate, up = ctx.saved_tensors
        dx, dg, du = (torch.empty_like(t) for t in (x, w_gate, w_up))
        pd.pd_gated_backward(dh.contiguous(), x, w_gate, w_up, gate, up, dx=dx, dw_gate=dg, dw_up=du)
        return dx, dg, du


# ------------------------------------------------------------------ the model
class Model(torch.nn.Module):
    def __init__(self, grid=(6, 8), patch=8, width=128, layers=2, heads=4, dtype=torch.bfloat16, dropout=0.1, seed=0):
        super().__init__()
        self.width, self.heads, self.dim, self.dtype, self.p, self.seed = width, heads, width // heads, dtype, dropout, seed + 1
        g = torch.Generator().manual_seed(seed)

        def matrix(fan_in, fan_out, gain=1.0):
            return torch.nn.Parameter((torch.randn(fan_in, fan_out, generator=g) * gain / math.sqrt(fan_in)).cuda())
        self.enter, self.leave, self.time = matrix(patch, width), matrix(width, patch, 0.1), matrix(width, width)
        self.blocks = torch.nn.ModuleList()
        hidden = 8 * (width // 3)
        for _ in range(layers):
            b = torch.nn.Module()
            b.qkv, b.out = matrix(width, 3 * width), matrix(width, width, 0.5)
            b.gate, b.up, b.down = matrix(width, hidden), matrix(width, hidden), matrix(hidden, width, 0.5)
            b.modulation = matrix(width, 4 * width, 0.2)
            self.blocks.append(b)
        self.modulation = matrix(width, 2 * width, 0.2)
        # height turns the first half of a head's pairs, width the others
        self.sections = [self.dim // 4, self.dim // 4]
        self.register_buffer("table", torch.empty((max(grid), self.dim // 2, 2), device="cuda"))
        pd.pd_rotary_axes_table(self.table, self.sections, base=100.0)
        at = torch.meshgrid(*[torch.arange(n, device="cuda", dtype=torch.int32) for n in grid], indexing="ij")
        self.register_buffer("positions", torch.stack([a.flatten() for a in at], 1))
        self.register_buffer("step", torch.zeros(1, device="cuda", dtype=torch.int32))

    def _times(self, n):
        f = torch.exp(-math.log(10000.0) * torch.arange(self.width // 2, device="cuda") / (self.width // 2))
        a = n[:, None].float() * f
        return torch.nn.functional.silu(torch.cat([a.sin(), a.cos()], 1) @ self.time)

    def _product(self, x, w):
        return x @ w.to(self.dtype)

    def _add(self, x, h, site):
        return Add.apply(x, h, self.p if self.training else 0.0, self.seed, site, self.step)

    def forward(self, x, n):
        """The noise in x [batch, patch, value] at the timesteps n [batch]."""
        t = self._times(n)
        h = self._product(x.to(self.dtype), self.enter)
        for i, b in enumerate(self.blocks):
            scale1, shift1, scale2, shift2 = (t @ b.modulation).chunk(4, 1)
            y = Norm.apply(h, 1 + scale1, shift1)
            q, k, v = self._product(y, b.qkv).unflatten(2, (3 * self.heads, self.dim)).split(self.heads, 2)
            q, k = Rotary.apply(q, k, self.positions, self.table, self.sections)
            a = Attend.apply(q, k, v, False, 0, 0)
            h = self._add(self._product(a.flatten(2), b.out), h, 2 * i)
            y = Norm.apply(h, 1 + scale2, shift2)
            f = Gated.apply(y, b.gate.to(self.dtype), b.up.to(self.dtype))
            h = self._add(self._product(f, b.down), h, 2 * i + 1)
        scale, shift = (t @ self.modulation).chunk(2, 1)
        return self._product(Norm.apply(h, 1 + scale, shift), self.leave).float()


# ------------------------------------------------------------------ training
def latents(batch, grid, patch, g):
    """Waves of a random direction and phase over the grid of patches."""
    y, x = torch.meshgrid(*[torch.linspace(0, 1, n, device="cuda") for n in grid], indexing="ij")
    r = torch.rand(batch, 1, 3, device="cuda", generator=g) * 2 * math.pi
    wave = torch.cos(r[..., 0]) * y.flatten() + torch.sin(r[..., 0]) * x.flatten()
    c = torch.arange(patch, device="cuda") / patch
    return torch.sin(2 * math.pi * (wave[..., None] + c) + r[..., 1:2])


def train(model, sched, steps, grid=(6, 8), patch=8, batch=32, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    beta = torch.linspace(1e-4, 0.02, sched.T_train, device="cuda", dtype=torch.float64)
    abar = (1 - beta).cumprod(0).float()
    opt = torch.optim.Adam(model.parameters(), lr=1e-3)
    losses = []
    model.train()
    for _ in range(steps):
        x0 = latents(batch, grid, patch, g)
        n = torch.randint(0, sched.T_train, (batch,), device="cuda", generator=g)
        eps = torch.randn(x0.shape, device="cuda", generator=g)
        a = abar[n][:, None, None]
        loss = ((model(a.sqrt() * x0 + (1 - a).sqrt() * eps, n) - eps) ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        model.step += 1                            # the next step's masks
        losses.append(loss.detach())
    model.eval()
    return torch.stack(losses).cpu()


def main(steps=150, batch=4, dtype=torch.bfloat16):
    sched = pd.pd_init_schedule(pd.PD_DDIM, 100, 25)
    model = Model(dtype=dtype)
    losses = train(model, sched, steps)
    seq, rounds = sample(model, sched, (batch, 48, 8))
    par, windows = sample(model, sched, (batch, 48, 8), p=16, tau=0.02)
    return {"loss_first": float(losses[:10].mean()), "loss_last": float(losses[-10:].mean()), "sequential_rounds": rounds,
            "picard_rounds": windows, "picard_vs_sequential": float((par - seq).norm() / seq.norm())}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    a = ap.parse_args()
    for name, value in main(a.steps).items():
        print(f"{name}: {value:.4g}")
