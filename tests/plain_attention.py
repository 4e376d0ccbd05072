"""Decayed linear attention and windowed attention with sinks in 64 bits, from their definitions, and the bounds that the
GPU tests hold the kernels to.

A rounding to bf16 is off by at most U = 2^-8 of the value, one to fp32 by 2^-24.  An output is a sum of products whose
factors may have been rounded on the way; with `size` the same sum over absolute values, r roundings of the terms and one
of the result move it by at most r U size + U |out| (and a few fp32 roundings).  Signs are random in these inputs, so
the 2-norm is held to a bound of its own: independent roundings of r stages, each at most U / sqrt(3) in the mean square.
"""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def rows_of(lens, B, L):
    n = torch.full((B,), L) if lens is None else torch.as_tensor(lens)
    return torch.arange(L) < n[:, None]                                  # [B,L]


def decay_of(log_decay):
    """lambda of each head, as the library reads log_decay."""
    g = log_decay.double()
    return torch.exp(torch.where(g < 0, g, torch.zeros_like(g)))


def decay_prefill(q, k, v, log_decay, scale, S=None, lens=None):
    """Token by token.  Returns out, the state, and both again over absolute values."""
    B, H, L, d = q.shape
    live = rows_of(lens, B, L)[:, None, :, None]
    q, k, v = (torch.where(live, x, 0.0) for x in (q, k, v))
    lam = decay_of(log_decay)[:, None, None]
    S = torch.zeros((B, H, d, d), dtype=torch.float64) if S is None else S
    A, out, size = S.abs(), [], []
    for t in range(L):
        there = live[:, :, t, :, None]
        S = torch.where(there, lam * S + k[:, :, t, :, None] * v[:, :, t, None, :], S)
        A = torch.where(there, lam * A + (k[:, :, t, :, None] * v[:, :, t, None, :]).abs(), A)
        out.append(torch.where(live[:, :, t], scale * (q[:, :, t, None] @ S)[:, :, 0], 0.0))
        size.append(abs(scale) * (q[:, :, t, None].abs() @ A)[:, :, 0].detach())
    z = torch.zeros_like(q)
    return (torch.stack(out, 2) if L else z), S, (torch.stack(size, 2) if L else z), A


def window_seen(at, t, W, sinks):
    """Whether the tokens at places t see those at places `at` (broadcast)."""
    return (at <= t) & ((at > t - W) | (at < sinks))


def window_attend(q, k, v, seen, scale):
    """q [B,H,n,d], k, v [B,Hkv,m,d], seen [.., n, m].  Returns out, lse, and out over absolute values."""
    G = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    z = torch.where(seen, scale * (q @ k.transpose(2, 3)), -math.inf)
    p = torch.softmax(z, 3)
    return p @ v, torch.logsumexp(z, 3), (p @ v.abs()).detach()


def window_prefill(q, k, v, W, sinks, scale, lens=None):
    B, H, L, d = q.shape
    live = rows_of(lens, B, L)
    q, k, v = (torch.where(live[:, None, :, None], x, 0.0) for x in (q, k, v))
    t = torch.arange(L)
    out, lse, size = window_attend(q, k, v, window_seen(t[None], t[:, None], W, sinks), scale)
    return torch.where(live[:, None, :, None], out, 0.0), torch.where(live[:, None], lse, -math.inf), size


def near(got, want, size, dtype, roundings, what, norm=None):
    """got within roundings U size + U |want| of want; the 2-norms within sqrt(roundings + 1) U / sqrt(3), or `norm`.
    fp32 sums of a few hundred to a few thousand terms: roundings counts them."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), what
    want, u = want.detach(), U[dtype]
    off = (got - want).abs() - u * want.abs() - (roundings * u + 2.0 ** -18 * (dtype == torch.bfloat16)) * size - 1e-30
    assert float(off.max() if off.numel() else 0) <= 0, f"{what}: {float(off.max()):.3e} over the bound at {int(off.argmax())}"
    norm = math.sqrt(roundings + 1) * u / math.sqrt(3) if norm is None else norm
    if float(want.norm()) > 0:
        rel = float((got - want).norm() / want.norm())
        assert rel <= norm, f"{what}: 2-norm off by {rel:.3e} > {norm:.3e}"
