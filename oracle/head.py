"""The losses at the output head and their gradients, written from their definitions in float64 (torch, on whatever device the
inputs are).  Shares no code with the library: whole matrices, targets as dense rows.

Besides the results every function returns what an error bound needs (magnitudes), see ``bounds`` below."""
from __future__ import annotations

import torch

F64 = torch.float64


def targets(top_index, top_logits, N, tau):
    """Dense teacher probabilities [T][N], which rows have any, and sum_j q_j log q_j."""
    T, k = top_index.shape
    Q = torch.zeros(T, N, dtype=F64, device=top_index.device)
    there = torch.zeros(T, dtype=torch.bool, device=top_index.device)
    neg_entropy = torch.zeros(T, dtype=F64, device=top_index.device)
    for t in range(T):
        has = top_index[t] >= 0
        l = top_logits[t][has].to(F64)
        if l.numel() == 0 or bool((l == -float("inf")).all()):
            continue
        there[t] = True
        e = ((l - l.max()) / tau).exp()
        q = e / e.sum()
        Q[t].index_put_((top_index[t][has],), q, accumulate=True)
        neg_entropy[t] = torch.special.xlogy(q, q).sum()
    return Q, there, neg_entropy


def head_loss(x, head, labels=None, top_index=None, top_logits=None, tau=1.0, d_ce=None, d_distill=None):
    """Returns a dict: ce, lse_ce, distill, lse_distill per token, and with gradients given dz, dx, dhead.  Rows of x that no
    loss asks for do not matter, whatever they hold."""
    T, N = x.shape[0], head.shape[0]
    dev = x.device
    counts = torch.zeros(T, dtype=torch.bool, device=dev)
    if labels is not None:
        counts |= labels >= 0
    if top_index is not None:
        Q, there, neg_entropy = targets(top_index, top_logits, N, tau)
        counts |= there
    X = torch.where(counts[:, None], x, torch.zeros_like(x)).to(F64)
    W = head.to(F64)
    Z = X @ W.T
    out = dict(counts=counts, Z=Z, X=X, W=W)
    dz = torch.zeros_like(Z)
    if labels is not None:
        has = labels >= 0
        lse = torch.logsumexp(Z, 1)
        onehot = torch.zeros_like(Z)
        onehot[torch.arange(T, device=dev)[has], labels[has]] = 1.0
        out["lse_ce"] = torch.where(has, lse, 0.0)
        out["ce"] = torch.where(has, lse - (Z * onehot).sum(1), 0.0)
        if d_ce is not None:
            dz += torch.where(has, d_ce.to(F64), 0.0)[:, None] * (torch.exp(Z - lse[:, None]) - onehot)
    if top_index is not None:
        lse = torch.logsumexp(Z / tau, 1)
        log_p = Z / tau - lse[:, None]
        out["Q"] = Q
        out["lse_distill"] = torch.where(there, lse, 0.0)
        out["distill"] = torch.where(there, neg_entropy - (Q * log_p).sum(1), 0.0)
        if d_distill is not None:
            dz += torch.where(there, d_distill.to(F64) / tau, 0.0)[:, None] * (torch.exp(log_p) - Q)
    if d_ce is not None or d_distill is not None:
        out.update(dz=dz, dx=dz @ W, dhead=dz.T @ X)
    return out


def bounds(o, tau=1.0, d_ce=None, d_distill=None):
    """How far a GPU result may be from the float64 one, from the arithmetic alone: exact products of bf16 values, every partial
    sum rounded or truncated once to 24 bits, ex2 with a relative error of 2^-22, probabilities and their gradient rounded
    once to bf16 (2^-8) before the second product, results rounded once to their type.

      z      |dz_| <= K 2^-23 sum |x w|                                  =: bz
      lse    errors of z move it by at most max bz / tau; a sum of at most 128 terms by one thread, its rescaling and ex2's
             argument (relative 2^-23 of a difference of logits, in units of the logits' range) by less than
             2^-16 + 2^-21 range / tau; the result is rounded to fp32
      loss   the same and bz of the target's logit / tau
      p      relative: (bz + max bz) / tau + 2^-16 + 2^-20 (|z| + |lse|) / tau (fma of z and lse in fp32); and 2^-126: ex2 gives
             0 for what is below the smallest normal number (the ftz of its name)
      dz     that share of g p, and 2^-8 |dz| for the rounding to bf16 (2^-7 |g q| where a target is taken off in fp32: its
             own rounding is 2^-24, covered)
      dx     sum |err dz| |w| + N 2^-23 sum |dz w| + 2^-8 |dx|;  dhead alike over the tokens"""
    X, W, Z = o["X"], o["W"], o["Z"]
    K, N, T = X.shape[1], W.shape[0], X.shape[0]
    bz = K * 2.0 ** -23 * (X.abs() @ W.abs().T)
    mz = bz.max(1).values
    spread = Z.max(1).values - Z.min(1).values
    b = {}
    for name, t in (("ce", 1.0), ("distill", tau)):
        if name in o:
            lse = o["lse_" + name]
            e = mz / t + 2.0 ** -16 + 2.0 ** -21 * spread / t
            b["lse_" + name] = e + 2.0 ** -23 * lse.abs()
            b[name] = 2 * e + 2.0 ** -22 * (lse.abs() + Z.abs().max(1).values / t) + 2.0 ** -23 * o[name].abs()
    if "dz" in o:
        err = 2.0 ** -8 * o["dz"].abs()
        for name, t, g in (("ce", 1.0, d_ce), ("distill", tau, d_distill)):
            if g is None:
                continue
            lse = torch.logsumexp(Z / t, 1)[:, None]
            p = torch.exp(Z / t - lse)
            rel = (bz + mz[:, None]) / t + 2.0 ** -16 + 2.0 ** -20 * (Z.abs() / t + lse.abs())
            asked = o["lse_" + name] != 0
            gg = torch.where(asked, g.to(F64).abs() / t, 0.0)[:, None]
            err += 1.01 * gg * p * rel + gg * 2.0 ** -126
            if name == "distill":
                err += 2.0 ** -20 * gg * o["Q"]
        dz = o["dz"].abs()
        b["dx"] = err @ W.abs() + N * 2.0 ** -23 * (dz @ W.abs()) + 2.0 ** -8 * o["dx"].abs() + 1e-37
        b["dhead"] = err.T @ X.abs() + T * 2.0 ** -23 * (dz.T @ X.abs()) + 2.0 ** -8 * o["dhead"].abs() + 1e-37
    return b
