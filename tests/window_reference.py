"""The attention with a sliding window and sinks, and rotary positions, from their definitions in 64 bits (test infrastructure), with
element-wise bounds of what the library may be off: every rounding to bf16 is half a step, 2^-8 of the value."""
import math

import torch

HALF = torch.finfo(torch.bfloat16).eps / 2  # largest relative rounding error of bf16
# Beside each rounding to bf16 stand errors of 32-bit sums, exponentials and the saved log-sum-exp: scores off by less than
# 3e-4 (64 to 128 products of a few units each, 2^-22 a step) make weights off by less than 0.1 of a rounding.
SLACK = 1.1


def kept(T, window, sinks, device="cpu"):
    i = torch.arange(T, device=device)
    back = i[:, None] - i
    return (back >= 0) & ((back < window) | (i < sinks))


def forward(q, k, v, scale, window, sinks):
    """O, LSE, P of [B,H,T,D] against [B,KV,T,D], all in 64 bits."""
    G = q.shape[1] // k.shape[1]
    k, v = (x.repeat_interleave(G, 1) for x in (k, v))
    s = (q @ k.mT * scale).masked_fill(~kept(q.shape[2], window, sinks, q.device), -math.inf)
    return torch.softmax(s, -1) @ v, torch.logsumexp(s, -1), torch.softmax(s, -1)


def backward(q, k, v, do, scale, window, sinks):
    """dQ, dK, dV by the formulas, and the bound of each."""
    KV, G = k.shape[1], q.shape[1] // k.shape[1]
    o, _, p = forward(q, k, v, scale, window, sinks)
    kx, vx = (x.repeat_interleave(G, 1) for x in (k, v))
    delta = (do * o).sum(-1, keepdim=True)
    ds = p * (do @ vx.mT - delta)
    share = lambda x: x.unflatten(1, (KV, G)).sum(2)
    dq, dk, dv = ds @ kx * scale, share(ds.mT @ q) * scale, share(p.mT @ do)
    # Delta's error: that of O's sum of rounded weights (what O's own rounding took is kept), and 2^-16 of O
    d_delta = (do.abs() * (SLACK * HALF * (p @ vx.abs()) + HALF**2 * o.abs())).sum(-1, keepdim=True)
    d_ds = SLACK * HALF * ds.abs() + p * d_delta + 1e-6 * p
    bounds = (d_ds @ kx.abs() * scale + HALF * dq.abs() + 1e-6,
              share(d_ds.mT @ q.abs()) * scale + HALF * dk.abs() + 1e-6,
              SLACK * HALF * share(p.mT @ do.abs()) + HALF * dv.abs() + 1e-6)
    return (dq, dk, dv), bounds, delta


def forward_bound(p, v, o):
    v = v.repeat_interleave(p.shape[1] // v.shape[1], 1)
    return SLACK * HALF * (p @ v.abs()) + HALF * o.abs() + 1e-6


def decode(q, k, v, lengths, scale, window, sinks):
    """O, LSE and sum of weighted |V| of one token per sequence; reads nothing that is not kept."""
    B, H, _, D = q.shape
    KV = k.shape[1]
    o, lse, mass = torch.zeros_like(q), torch.full((B, H, 1), -math.inf, dtype=q.dtype, device=q.device), torch.zeros_like(q)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), k.shape[2])
        at = torch.tensor([j for j in range(n) if n - 1 - j < window or j < sinks], device=q.device, dtype=torch.long)
        if n == 0:
            continue
        kx, vx = (x[b, :, at].repeat_interleave(H // KV, 0) for x in (k, v))
        s = (q[b] @ kx.mT * scale)
        lse[b] = torch.logsumexp(s, -1)
        p = torch.softmax(s, -1)
        o[b], mass[b] = p @ vx, p @ vx.abs()
    return o, lse, mass


def rope(x, positions, inv_freq, interleaved, amplitude, backward=False):
    """x [B,H,T,D] turned by positions [B,T], in 64 bits."""
    R = 2 * inv_freq.numel()
    a = positions.double()[:, None, :, None] * inv_freq.double() * (-1.0 if backward else 1.0)
    c, s = a.cos() * amplitude, a.sin() * amplitude
    y = x.double().clone()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    x0, x1 = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def rel_rms(got, ref):
    return float((got.double() - ref).norm() / ref.norm())
