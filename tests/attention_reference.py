"""Attention with a window and sinks, and its gradient, from the definition in 64 bits, with the error bounds that the GPU tests use.

Bounds.  Inputs are bfloat16 and products of two of them exact in fp32.  A rounding to bfloat16 is off by at most 2^-8 of the value.
  scores   d fp32 additions: off by at most d 2^-24 sum_c |q_c k_c| / sqrt(d); with the hardware exp2 (2^-22) a weight is off by
           that much relative to itself, SCORE below.
  lse      that, n additions of positive terms (n 2^-24) and a few roundings.
  O        weights rounded once (2^-8 of each), then O rounded: 2^-8 (sum_j P_j |V_j| + |O|), and SCORE sum_j P_j |V_j|.
  dV       likewise: 2^-8 (sum_i P_i |dO_i| + |dV|), and SCORE sum_i P_i |dO_i|.
  dQ, dK   dS is rounded once, and P (dP - D) itself carries SCORE |dS| and P times the error of the two dot products,
           d 2^-24 (sum_c |dO_c V_c| + sum_c |dO_c O_c|).
Second-order terms are covered by taking 2^-8 as 1.02 * 2^-8.
"""
from __future__ import annotations

import math

import torch

HALF = 1.02 * 2.0 ** -8


def visible(N, M, window, sinks, device="cpu"):
    """(N, M): which keys the queries, the last N of M positions, see."""
    p = torch.arange(N, device=device).view(N, 1) + (M - N)
    j = torch.arange(M, device=device).view(1, M)
    seen = j <= p
    if window is not None:
        seen = seen & ((p - j < window) | (j < sinks))
    return seen


def _scores(q, k, seen):
    """Scores with -inf where nothing is seen, and the relative error that fp32 sums may leave in a weight (per query)."""
    d = q.shape[-1]
    s = (q @ k.transpose(-1, -2)) / math.sqrt(d)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    size = torch.where(seen, (q.abs() @ k.abs().transpose(-1, -2)) / math.sqrt(d), torch.zeros_like(s))
    top = size.amax(-1, keepdim=True) if size.shape[-1] else torch.zeros(*q.shape[:-1], 1, dtype=q.dtype, device=q.device)
    return s, 2.0 ** -24 * d * top + 2.0 ** -21


def _weights(s):
    if s.shape[-1] == 0:
        return s, torch.full(s.shape[:-1], -math.inf, dtype=s.dtype, device=s.device)
    lse = torch.logsumexp(s, -1)
    return torch.exp(s - torch.where(lse.isneginf(), torch.zeros_like(lse), lse)[..., None]), lse


def forward(Q, K, V, window, sinks, seen=None):
    """(O, lse, bound of O, bound of lse) in 64 bits; Q (batch, heads, N, d), K, V (batch, kv_heads, M, d)."""
    Q, K, V = Q.double(), K.double(), V.double()
    group = Q.shape[1] // K.shape[1]
    K, V = K.repeat_interleave(group, 1), V.repeat_interleave(group, 1)
    N, M = Q.shape[2], K.shape[2]
    if seen is None:
        seen = visible(N, M, window, sinks, Q.device)
    # unseen rows of K and V must not matter: whatever they hold is cleared where no query of the call sees it
    s, score = _scores(Q, K, seen)
    P, lse = _weights(s)
    O, size = P @ V, P @ V.abs()
    bound = (HALF + score) * size + HALF * O.abs() + 1e-30
    lse_bound = 2 * score[..., 0] + 2.0 ** -24 * (seen.sum(-1).double() + 16 + 4 * torch.where(lse.isneginf(), 0.0, lse).abs())
    return O, lse, bound, lse_bound


def gradient(Q, K, V, O, lse, dO, window, sinks):
    """((dQ, dK, dV), their bounds) in 64 bits, from O and lse as they are given."""
    Q, K, V, O, lse, dO = (t.double() for t in (Q, K, V, O, lse, dO))
    batch, kv, M, d = K.shape
    group = Q.shape[1] // kv
    K, V = K.repeat_interleave(group, 1), V.repeat_interleave(group, 1)
    N = Q.shape[2]
    seen = visible(N, M, window, sinks, Q.device)
    s, score = _scores(Q, K, seen)
    score = score + 2.0 ** -22 * torch.where(lse.isneginf(), 0.0, lse).abs()[..., None]
    P = torch.exp(s - torch.where(lse.isneginf(), torch.zeros_like(lse), lse)[..., None])
    D = (dO * O).sum(-1, keepdim=True)
    dS = P * (dO @ V.transpose(-1, -2) - D)
    dot = 2.0 ** -24 * d * (dO.abs() @ V.abs().transpose(-1, -2) + (dO * O).abs().sum(-1, keepdim=True))
    wrong = (HALF + score) * dS.abs() + P * dot
    shared = lambda x: x.view(batch, kv, group, M, d).sum(2)  # noqa: E731
    T = lambda x: x.transpose(-1, -2)  # noqa: E731
    dQ, dK, dV = dS @ K / math.sqrt(d), shared(T(dS) @ Q) / math.sqrt(d), shared(T(P) @ dO)
    bounds = (wrong @ K.abs() / math.sqrt(d), shared(T(wrong) @ Q.abs()) / math.sqrt(d), shared(T((HALF + score) * P) @ dO.abs()))
    # fp32 sums of up to group * N products
    slack = 2.0 ** -24 * group * max(N, M)
    sizes = (dS.abs() @ K.abs(), shared(T(dS.abs()) @ Q.abs()), shared(T(P) @ dO.abs()))
    return (dQ, dK, dV), tuple(b + slack * z + HALF * g.abs() + 1e-30 for b, z, g in zip(bounds, sizes, (dQ, dK, dV)))


def within(got, want, bound, what=""):
    """Every element of `got` within `bound` of `want`; infinities and zeros where `want` has them."""
    got, want, bound = got.double().cpu(), want.cpu(), bound.cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(got[odd], want[odd]), f"{what}: values that are not finite differ"
    off = torch.where(odd, torch.zeros_like(got), (got - torch.where(odd, got, want)).abs() / torch.where(odd, torch.ones_like(bound), bound))
    if off.numel():
        assert not off.isnan().any(), f"{what}: NaN"
        worst = off.max().item()
        assert worst <= 1.0, f"{what}: {worst:.3f} of the bound at {torch.unravel_index(off.argmax(), off.shape)}"
