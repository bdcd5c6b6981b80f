"""A transformer over an action sequence as the denoiser, from the library's operators.

    python examples/trajectory_transformer.py [--steps 200] [--eight-bits]

The model predicts the noise in a sequence of actions: RMS norm with the residual's addition, rotary
positions and grouped attention from the library, matrix products from torch.  The program

  1. trains it on a toy set of trajectories (the operators' backward passes),
  2. samples a batch with the sequential chain and with ParaDiGMS (Algorithm 1), where all points of a
     window go through the network as one batch, with pd_init_schedule's tables, and
  3. runs the causal form over a long history, at once and token by token over a cache with a
     sliding window and sinks.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2305_16317_amd as pd  # noqa: E402


# ------------------------------------------------------------------ the operators under autograd
class Norm(torch.autograd.Function):
    """(x + residual, its norm times weight)."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        x, residual = x.contiguous(), residual.contiguous()
        total, y = torch.empty_like(x), torch.empty_like(x)
        rstd = torch.empty(x.numel() // x.shape[-1], device=x.device)
        pd.pd_rmsnorm_forward(x, weight, y, residual=residual, sum_out=total, rstd=rstd)
        ctx.save_for_backward(total, weight, rstd)
        return total, y

    @staticmethod
    def backward(ctx, dtotal, dy):
        total, weight, rstd = ctx.saved_tensors
        dx, dweight = torch.empty_like(total), torch.empty_like(weight)
        pd.pd_rmsnorm_backward(dy.contiguous(), total, weight, rstd, dx, dweight, dsum=dtotal.contiguous())
        return dx, dx, dweight


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, table):
        ctx.save_for_backward(positions, table)
        qo, ko = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        pd.pd_rotary_apply(q, k, positions, table, qo, ko)
        return qo, ko

    @staticmethod
    def backward(ctx, dq, dk):
        positions, table = ctx.saved_tensors
        dq, dk = dq.contiguous(), dk.contiguous()
        pd.pd_rotary_apply(dq, dk, positions, table, dq, dk, backward=True)
        return dq, dk, None, None


class Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, window, sinks):
        out = torch.empty_like(q)
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), device=q.device)
        pd.pd_attention_forward(q, k, v, out, lse=lse, causal=causal, window=window, sinks=sinks)
        ctx.save_for_backward(q, k, v, out, lse)
        ctx.how = dict(causal=causal, window=window, sinks=sinks)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        pd.pd_attention_backward(q, k, v, out, lse, dout.contiguous(), dq, dk, dv, **ctx.how)
        return dq, dk, dv, None, None, None


# ------------------------------------------------------------------ the model
class Model(torch.nn.Module):
    def __init__(self, actions=10, width=256, layers=2, heads=8, kv_heads=2, dtype=torch.bfloat16, seed=0,
                 causal=False, window=0, sinks=0, positions=4096):
        super().__init__()
        self.width, self.heads, self.kv, self.dim = width, heads, kv_heads, width // heads
        self.causal, self.window, self.sinks, self.dtype = causal, window, sinks, dtype
        g = torch.Generator().manual_seed(seed)

        def matrix(fan_in, fan_out, gain=1.0):
            return torch.nn.Parameter((torch.randn(fan_in, fan_out, generator=g) * gain / math.sqrt(fan_in)).cuda())
        self.enter, self.leave = matrix(actions, width), matrix(width, actions, 0.1)
        self.blocks = torch.nn.ModuleList()
        for _ in range(layers):
            b = torch.nn.Module()
            b.qkv = matrix(width, (heads + 2 * kv_heads) * self.dim)
            b.out, b.up, b.down = matrix(width, width, 0.5), matrix(width, 4 * width), matrix(4 * width, width, 0.5)
            b.norm1, b.norm2 = (torch.nn.Parameter(torch.ones(width, device="cuda")) for _ in range(2))
            self.blocks.append(b)
        self.norm = torch.nn.Parameter(torch.ones(width, device="cuda"))
        self.register_buffer("table", torch.empty((positions, self.dim // 2, 2), device="cuda"))
        pd.pd_rotary_table(self.table)

    def _times(self, n):
        f = torch.exp(-math.log(10000.0) * torch.arange(self.width // 2, device="cuda") / (self.width // 2))
        a = n[:, None].float() * f
        return torch.cat([a.sin(), a.cos()], 1)[:, None]

    def _product(self, x, w):
        return x @ w.to(self.dtype)

    def forward(self, x, n=None):
        """The noise in x [batch, token, action] at the timesteps n [batch] (None: no diffusion)."""
        B, L = x.shape[:2]
        h = self._product(x.to(self.dtype), self.enter)
        if n is not None:
            h = h + self._times(n).to(self.dtype)
        more = torch.zeros_like(h)
        pos = torch.arange(L, device="cuda", dtype=torch.int32)
        sizes = [self.heads, self.kv, self.kv]
        for b in self.blocks:
            h, y = Norm.apply(more, h, b.norm1)
            q, k, v = self._product(y, b.qkv).unflatten(2, (sum(sizes), self.dim)).split(sizes, 2)
            q, k = Rotary.apply(q, k, pos, self.table)
            a = Attend.apply(q, k, v, self.causal, self.window, self.sinks)
            h, y = Norm.apply(self._product(a.flatten(2), b.out), h, b.norm2)
            more = self._product(torch.nn.functional.gelu(self._product(y, b.up)), b.down)
        return self._product(Norm.apply(more, h, self.norm)[1], self.leave).float()


# ------------------------------------------------------------------ 1: training
def trajectories(batch, length, actions, g):
    """Sums of two slow waves with a random phase for each action."""
    t = torch.linspace(0, 1, length, device="cuda")[None, :, None]
    ph = torch.rand(batch, 1, actions, device="cuda", generator=g) * 2 * math.pi
    return torch.sin(2 * math.pi * t + ph) + 0.3 * torch.sin(6 * math.pi * t + 2 * ph)


def train(model, sched, steps, batch=64, length=16, actions=10, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    beta = torch.linspace(1e-4, 0.02, sched.T_train, device="cuda", dtype=torch.float64)
    abar = (1 - beta).cumprod(0).float()
    opt = torch.optim.Adam(model.parameters(), lr=1e-3)
    losses = []
    for _ in range(steps):
        x0 = trajectories(batch, length, actions, g)
        n = torch.randint(0, sched.T_train, (batch,), device="cuda", generator=g)
        eps = torch.randn(x0.shape, device="cuda", generator=g)
        a = abar[n][:, None, None]
        loss = ((model(a.sqrt() * x0 + (1 - a).sqrt() * eps, n) - eps) ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    return torch.stack(losses).cpu()


# ------------------------------------------------------------------ 2: sampling
@torch.no_grad()
def sample(model, sched, shape, seed=0, p=0, tau=0.1):
    """One batch of samples [batch, length, actions]: the sequential chain, or with p > 0 ParaDiGMS with
    window p.  Returns (sample, rounds of the network)."""
    tb = {k: torch.from_numpy(v).cuda() for k, v in sched.tables().items()}
    T, B = sched.T, shape[0]
    x = torch.empty(shape, device="cuda")
    noise = torch.empty((T, *shape), device="cuda")
    pd.pd_normals(seed, 0, x)
    pd.pd_normals(seed, 1, noise)
    z = noise * tb["noise_std"][:, None, None, None]

    def drift(points, i):                          # points [m, batch, length, actions] at the steps i [m]
        m = i.numel()
        eps = model(points.flatten(0, 1), tb["model_t"][i].repeat_interleave(B)).reshape(points.shape)
        c = lambda v: v[i].reshape(m, 1, 1, 1)     # noqa: E731
        return c(tb["A"]) * points + c(tb["B"]) * eps
    if not p:
        for i in range(T):
            x = x + drift(x[None], torch.tensor([i], device="cuda"))[0] + z[i]
        return x, T
    X = x[None].repeat(T + 1, 1, 1, 1)
    t = f = rounds = 0
    while t < T:                                   # Algorithm 1
        pe = min(p, T - t)
        i = torch.arange(t, t + pe, device="cuda")
        old = X[i.clamp(max=f)]
        new = X[t] + (drift(old, i) + z[t:t + pe]).cumsum(0)
        err = ((new[:-1] - old[1:]) ** 2).mean((2, 3))
        bad = (err > tau**2 * tb["tol_var"][i[1:]][:, None]).any(1).nonzero()
        X[t + 1:t + pe + 1] = new
        f, t, rounds = t + pe, t + (int(bad[0]) + 1 if bad.numel() else pe), rounds + 1
    return X[T], rounds


# ------------------------------------------------------------------ 3: token by token
class Decoder:
    """The causal model one token at a time: the keys and values of each layer stay in a cache.  With
    eight_bits the norms give e4m3 and a scale a row, for products in 8 bits."""

    def __init__(self, model, batch, length, eight_bits=False):
        self.m, self.n, self.eight = model, 0, eight_bits
        shape = (batch, model.kv, length, model.dim)
        self.cache = [tuple(torch.zeros(shape, device="cuda", dtype=model.dtype) for _ in "kv") for _ in model.blocks]
        self.lens = torch.zeros(batch, device="cuda", dtype=torch.int32)
        if eight_bits:                             # weights [out, in] in e4m3 with a scale for each output
            self.w8 = {}
            for b in model.blocks:
                for name in ("qkv", "up"):
                    w = getattr(b, name).detach().float().t().contiguous()
                    s = w.abs().amax(1, keepdim=True) / 448
                    self.w8[id(b), name] = ((w / s).to(torch.float8_e4m3fn), s)

    def _normed_product(self, x, residual, weight, block, name):
        """(x + residual, its norm times the block's matrix)."""
        total = torch.empty_like(x)
        if not self.eight:
            y = torch.empty_like(x)
            pd.pd_rmsnorm_forward(x, weight, y, residual=residual, sum_out=total)
            return total, y @ getattr(block, name).to(self.m.dtype)
        y = torch.empty(x.shape, device="cuda", dtype=torch.float8_e4m3fn)
        scale = torch.empty((x.shape[0], 1), device="cuda")
        pd.pd_rmsnorm_forward(x, weight, y, residual=residual, sum_out=total, scale=scale)
        w, ws = self.w8[id(block), name]
        return total, torch._scaled_mm(y, w.t(), scale_a=scale, scale_b=ws.t().contiguous(), out_dtype=self.m.dtype)

    @torch.no_grad()
    def step(self, x):
        """The outputs for the next token x [batch, action] of every sequence."""
        m, B = self.m, x.shape[0]
        h = x.to(m.dtype) @ m.enter.to(m.dtype)
        more = torch.zeros_like(h)
        pos = self.lens.view(B, 1).clone()
        self.lens += 1
        sizes = [m.heads, m.kv, m.kv]
        for b, (kc, vc) in zip(m.blocks, self.cache):
            h, qkv = self._normed_product(more, h, b.norm1, b, "qkv")
            q, k, v = qkv.view(B, 1, sum(sizes), m.dim).split(sizes, 2)
            at = slice(self.n, self.n + 1)
            vc[:, :, at].copy_(v.transpose(1, 2))
            pd.pd_rotary_apply(q, k, pos, m.table, q, kc[:, :, at].transpose(1, 2))   # the turned key into the cache
            a = torch.empty((B, 1, m.heads, m.dim), device="cuda", dtype=m.dtype)
            pd.pd_attention_forward(q, kc.transpose(1, 2), vc.transpose(1, 2), a, causal=True, window=m.window,
                                    sinks=m.sinks, kv_lens=self.lens)
            h, up = self._normed_product(a.view(B, -1) @ b.out.to(m.dtype), h, b.norm2, b, "up")
            more = torch.nn.functional.gelu(up) @ b.down.to(m.dtype)
        y = torch.empty_like(h)
        pd.pd_rmsnorm_forward(more, m.norm, y, residual=h)
        self.n += 1
        return (y @ m.leave.to(m.dtype)).float()


def main(steps=200, batch=8, history=96, eight_bits=False, dtype=torch.bfloat16):
    sched = pd.pd_init_schedule(pd.PD_DDIM, 100, 25)
    model = Model(dtype=dtype)
    losses = train(model, sched, steps)
    seq, rounds = sample(model, sched, (batch, 16, 10))
    par, windows = sample(model, sched, (batch, 16, 10), p=16, tau=0.02)
    causal = Model(dtype=dtype, causal=True, window=32, sinks=4, seed=5)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = trajectories(batch, history, 10, g)
    with torch.no_grad():
        whole = causal(x)
    dec = Decoder(causal, batch, history, eight_bits)
    one = torch.stack([dec.step(x[:, i]) for i in range(history)], 1)
    rel = lambda a, b: float((a - b).norm() / b.norm())      # noqa: E731
    return {"loss_first": float(losses[:10].mean()), "loss_last": float(losses[-10:].mean()), "sequential_rounds": rounds,
            "picard_rounds": windows, "picard_vs_sequential": rel(par, seq), "tokens_vs_whole": rel(one, whole)}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--eight-bits", action="store_true")
    a = ap.parse_args()
    for name, value in main(a.steps, eight_bits=a.eight_bits).items():
        print(f"{name}: {value:.4g}")
