"""A small hybrid stack, trained and then served with libm3.

Two blocks, each a mixer and a gated feed-forward block: the first mixes with
the Mamba-3 scan, the second with the gated linear recurrence.  Training runs
their forwards and backwards and AdamW with 8-bit states; serving runs the
same stack token by token from the states that the prompt left, and has to give
what the whole sequence gives.

The task is synthetic: tell the moving average of a noisy signal, which takes a
memory.  Projections and the loss are plain torch.

    python examples/hybrid_stack.py [--steps 60]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_15569_amd import m3  # noqa: E402

HEADS, P, N, CHUNK = 2, 64, 128, 64    # the scan: rank 1, its state N x P a head
D, FF = HEADS * P, 352                 # width, feed-forward width


class Scan(torch.autograd.Function):
    """m3_scan_fwd / m3_scan_bwd: x [B,L,H,1,P], B and C [B,L,H,1,N]."""

    @staticmethod
    def forward(ctx, x, Bm, Cm, dt, A, lam, theta, skip):
        args = [t.contiguous() for t in (x, Bm, Cm, dt, A, lam, theta, skip)]
        ctx.save_for_backward(*args)
        return m3.scan_fwd(*args, chunk=CHUNK)[0]

    @staticmethod
    def backward(ctx, dy):
        g = m3.scan_bwd(*ctx.saved_tensors, dy.contiguous(), chunk=CHUNK)
        return tuple(g[k] for k in ("dx", "dB", "dC", "ddt", "dA", "dlam", "dtheta", "dD"))


class Recurrence(torch.autograd.Function):
    """m3_glr_fwd / m3_glr_bwd on the slices of one projection: xriz [B,L,4D]."""

    @staticmethod
    def forward(ctx, xriz, A):
        x, r, i, z = xriz.split(D, dim=-1)
        y, _, states = m3.glr_fwd(x, r, i, A, z=z, save_states=True)
        ctx.save_for_backward(xriz, A, states)
        return y

    @staticmethod
    def backward(ctx, dy):
        xriz, A, states = ctx.saved_tensors
        x, r, i, z = xriz.split(D, dim=-1)
        g = m3.glr_bwd(x, r, i, A, states, dy.contiguous(), z=z)
        return torch.cat([g[k] for k in ("dx", "dr", "di", "dz")], -1), g["dA"]


class FeedForward(torch.autograd.Function):
    """m3_ffn_fwd / m3_ffn_bwd."""

    @staticmethod
    def forward(ctx, x, Wg, Wu, Wd):
        ctx.save_for_backward(x, Wg, Wu, Wd)
        return m3.ffn_fwd(x, Wg, Wu, Wd)

    @staticmethod
    def backward(ctx, dy):
        g = m3.ffn_bwd(*ctx.saved_tensors, dy.contiguous())
        return g["dx"], g["dWg"], g["dWu"], g["dWd"]


def make_params(gen, dev):
    """fp32 parameters by name; matrices are used through bf16 copies."""
    def w(*shape):
        return torch.randn(shape, device=dev, generator=gen) * shape[-1] ** -0.5
    p = dict(embed=torch.randn((D, 1), device=dev, generator=gen), head=w(1, D))
    p.update(s_x=w(D, D), s_b=w(HEADS * N, D), s_c=w(HEADS * N, D), s_out=w(D, D),
             s_dt=w(2 * HEADS, D), s_theta=w(HEADS * N // 2, D) * 0.1, s_skip=torch.ones(HEADS, device=dev),
             s_logA=torch.linspace(-3.0, 0.0, HEADS, device=dev))
    p.update(r_in=w(4 * D, D), r_out=w(D, D), r_logA=torch.linspace(math.log(0.005), 0.0, D, device=dev))
    for b in "12":
        p["f_gate" + b], p["f_up" + b], p["f_down" + b] = w(FF, D), w(FF, D), w(D, FF) * 0.5
    return p


def norm(h):
    return (h.float() * torch.rsqrt(h.float().square().mean(-1, keepdim=True) + 1e-6)).to(h.dtype)


def scan_inputs(p, low, h):
    lead = h.shape[:-1]
    x = F.linear(h, low["s_x"]).view(*lead, HEADS, 1, P)
    Bm = norm(F.linear(h, low["s_b"]).view(*lead, HEADS, 1, N))
    Cm = norm(F.linear(h, low["s_c"]).view(*lead, HEADS, 1, N)) * N ** -0.5
    dt, lam = F.linear(h, low["s_dt"]).float().split(HEADS, -1)
    dt, lam = F.softplus(dt - 2.0), torch.sigmoid(lam)
    theta = dt[..., None] * F.linear(h, low["s_theta"]).float().view(*lead, HEADS, N // 2)
    return x, Bm, Cm, dt, -torch.exp(p["s_logA"]), lam, theta, p["s_skip"]


def stack(p, low, u, state=None):
    """The stack over u [B,L] (training, or a prompt), or with `state` over one token
    u [B]; returns what it predicts and, for a token, advances the states in place."""
    h = (u[..., None] * low["embed"].view(-1)).to(torch.bfloat16)
    t = norm(h)
    args = scan_inputs(p, low, t)
    if state is None:
        y = Scan.apply(*args)
    else:
        x, Bm, Cm, dt, A, lam, theta, skip = (a.contiguous() for a in args)
        y = m3.step(state["scan"], state["carry"], x, Bm, Cm, dt, A, lam, theta, skip)
    h = h + F.linear(y.reshape(*h.shape[:-1], D), low["s_out"])
    h = h + FeedForward.apply(norm(h), low["f_gate1"], low["f_up1"], low["f_down1"])
    xriz, A = F.linear(norm(h), low["r_in"]), -torch.exp(p["r_logA"])
    if state is None:
        y = Recurrence.apply(xriz, A)
    else:
        x, r, i, z = xriz.split(D, dim=-1)
        y = m3.glr_step(state["recurrence"], x, r, i, A, z=z)
    h = h + F.linear(y, low["r_out"])
    h = h + FeedForward.apply(norm(h), low["f_gate2"], low["f_up2"], low["f_down2"])
    return F.linear(norm(h), low["head"]).float().squeeze(-1)


def zero_state(batch, dev):
    bf = dict(dtype=torch.bfloat16, device=dev)
    return dict(scan=torch.zeros(batch, HEADS, N, P, device=dev), recurrence=torch.zeros(batch, D, device=dev),
                carry=(torch.zeros(batch, HEADS, 1, N, **bf), torch.zeros(batch, HEADS, 1, P, **bf)))


def batch_of(gen, dev, B, L):
    """A noisy signal and its exponential moving average, what the stack has to tell."""
    u = torch.randn((B, L), device=dev, generator=gen)
    avg, out = torch.zeros(B, device=dev), []
    for t in range(L):
        avg = 0.95 * avg + 0.31 * u[:, t]
        out.append(avg)
    return u, torch.stack(out, 1)


def train(steps=60, B=32, L=256, seed=0, lr=1e-3, dev="cuda:0", tell=print):
    gen = torch.Generator(dev).manual_seed(seed)
    p = make_params(gen, dev)
    names = list(p)
    low = {k: v.to(torch.bfloat16) for k, v in p.items()}
    leaves = {k: low[k].requires_grad_() for k in names}
    # what the scan and the recurrence take in fp32 learns from its own gradients
    f32 = {k: p[k].requires_grad_() for k in ("s_logA", "s_skip", "r_logA")}
    grads = {k: torch.zeros_like(p[k], dtype=torch.bfloat16) for k in names}
    state8 = [[torch.zeros_like(p[k], dtype=torch.float8_e4m3fn) for k in names] for _ in range(2)]
    scales = [torch.zeros(-(-p[k].numel() // 256), 2, device=dev) for k in names]
    table = m3.adamw_table([p[k].detach() for k in names], [grads[k] for k in names], *state8,
                           weight_decay=[0.01 if p[k].dim() > 1 else 0.0 for k in names],
                           low=[low[k].detach() for k in names], scales=scales)
    losses = []
    for t in range(1, steps + 1):
        u, want = batch_of(gen, dev, B, L)
        loss = F.mse_loss(stack(f32, leaves, u), want)
        inputs = [f32.get(k, leaves[k]) for k in names]
        got = torch.autograd.grad(loss, inputs)
        for k, g in zip(names, got):
            grads[k].copy_(g)
        # clip the gradients' norm: one number that stays on the device
        total = torch.stack([g.float().norm() for g in grads.values()]).norm()
        clip = torch.clamp(1.0 / (total + 1e-6), max=1.0).view(1)
        m3.adamw_step(table, step=t, lr=lr, betas=(0.9, 0.95), grad_scale=clip, seed=t)
        losses.append(loss.detach())
        if t % 20 == 0 or t == 1:
            tell(f"step {t}: loss {losses[-1].item():.4f}")
    return f32, low, [v.item() for v in losses]


def serve(f32, low, B=4, L=200, seed=1, dev="cuda:0"):
    """The whole sequence at once, and token by token from zero states."""
    gen = torch.Generator(dev).manual_seed(seed)
    u, want = batch_of(gen, dev, B, L)
    with torch.no_grad():
        whole = stack(f32, low, u)
        state = zero_state(B, dev)
        steps = torch.stack([stack(f32, low, u[:, t], state) for t in range(L)], 1)
    return whole, steps, want


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    f32, low, losses = train(a.steps)
    whole, steps, want = serve(f32, low)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    print(f"served token by token: {(whole - steps).abs().max().item():.4f} from the whole sequence, "
          f"{F.mse_loss(steps, want).item():.4f} from the target")


if __name__ == "__main__":
    main()
