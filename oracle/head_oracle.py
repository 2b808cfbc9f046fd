"""Plain float64 definitions of the operators around the LM head: the norm in front of it, 8-bit
activation checkpoints, and the preference loss over the completions of a question.  numpy only,
loops where a definition is a loop; shares no code with the CUDA path."""
from __future__ import annotations

import math
from typing import Dict, List, Optional, Tuple

import numpy as np

GROUP = 128
TINY = 2.0 ** -119


# ------------------------------------------------------------------------------------------ norm
def norm_fwd(x, gamma: Optional[np.ndarray], beta: Optional[np.ndarray], eps: float, kind: str) -> Dict[str, np.ndarray]:
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1) if kind == "layer" else np.zeros(x.shape[0])
    xc = x - mean[:, None]
    rstd = 1.0 / np.sqrt((xc ** 2).mean(axis=1) + eps)
    return {"y": norm_apply(x, mean, rstd, gamma, beta), "mean": mean, "rstd": rstd}


def norm_apply(x, mean, rstd, gamma, beta) -> np.ndarray:
    y = (np.asarray(x, np.float64) - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    return y if beta is None else y + np.asarray(beta, np.float64)


def norm_bwd(dy, x, gamma, mean, rstd, kind: str) -> Dict[str, np.ndarray]:
    dy, rstd = np.asarray(dy, np.float64), np.asarray(rstd, np.float64)
    xh = norm_apply(x, mean, rstd, None, None)
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = g - xh * (g * xh).mean(axis=1, keepdims=True)
    if kind == "layer":
        dx = dx - g.mean(axis=1, keepdims=True)
    return {"dx": dx * rstd[:, None], "dgamma": (dy * xh).sum(axis=0), "dbeta": dy.sum(axis=0), "g": g, "xh": xh}


# ------------------------------------------------------------------------------------------ 8 bits
def ckpt8_store(x) -> Tuple[np.ndarray, np.ndarray]:
    """(data int8 [T, H], scale fp32 [T, ceil(H / 128)]).  The stored integers depend on single
    roundings, so the steps are taken in float32 as the format defines them."""
    x = np.asarray(x, dtype=np.float32)
    T, H = x.shape
    n = -(-H // GROUP)
    data, scale = np.zeros((T, H), np.int8), np.zeros((T, n), np.float32)
    for t in range(T):
        for k in range(n):
            part = x[t, k * GROUP:(k + 1) * GROUP]
            if not np.all(np.isfinite(part)):
                scale[t, k] = np.nan
                continue
            top = np.float32(np.max(np.abs(part)))
            if top < TINY:
                continue
            one, n127 = np.float32(1), np.float32(127)
            scale[t, k] = top * (one / n127)
            data[t, k * GROUP:(k + 1) * GROUP] = np.rint(part * (n127 * (one / top))).astype(np.int8)
    return data, scale


def ckpt8_values(data, scale) -> np.ndarray:
    H = data.shape[1]
    return data.astype(np.float64) * np.repeat(scale.astype(np.float64), GROUP, axis=1)[:, :H]


# ------------------------------------------------------------------------------------------ preference
def preference_pairs(rewards, members: List[int], pairs: str) -> List[Tuple[int, int]]:
    """(preferred, other) among the members of one question."""
    if pairs == "all":
        return [(i, j) for i in members for j in members if rewards[i] > rewards[j]]
    if not members:
        return []
    best = members[0]
    worst = members[0]
    for s in members:
        if rewards[s] > rewards[best]:
            best = s
        if rewards[s] < rewards[worst]:
            worst = s
    return [(best, worst)] if rewards[best] > rewards[worst] else []


def pair_loss(D: float, beta: float, kind: str, e: float) -> Tuple[float, float]:
    """Loss of one pair and its derivative by D = R_i - R_j."""
    h = beta * D
    if kind == "sigmoid":
        sp = lambda z: max(z, 0.0) + math.log1p(math.exp(-abs(z)))
        sig = 1 / (1 + math.exp(-h)) if h >= 0 else math.exp(h) / (1 + math.exp(h))
        return (1 - e) * sp(-h) + e * sp(h), beta * (sig - (1 - e))
    if kind == "squared":
        u = D - 1 / (2 * beta)
        return u * u, 2 * u
    return max(0.0, 1 - h), (-beta if h < 1 else 0.0)


def preference_loss(logp, ref_logp, cu, rewards, group_offsets, beta: float, kind: str = "sigmoid", pairs: str = "all",
                    label_smoothing: float = 0.0, length_norm: bool = False, grad_scale: float = 1.0,
                    masked=None) -> Dict[str, np.ndarray]:
    """masked: tokens left out besides those that are not finite."""
    logp, ref = np.asarray(logp, np.float64), np.asarray(ref_logp, np.float64)
    T, S, Q = len(logp), len(cu) - 1, len(group_offsets) - 1
    with np.errstate(invalid="ignore"):
        d = logp - ref
    out = ~np.isfinite(d)
    if masked is not None:
        out |= np.asarray(masked, bool)
    R, gR = np.zeros(S), np.zeros(S)
    q_loss, q_margin, q_pairs = np.zeros(Q), np.zeros(Q), np.zeros(Q, np.int32)
    g = np.zeros(T)
    for q in range(Q):
        seqs = range(group_offsets[q], group_offsets[q + 1])
        for s in seqs:
            t = slice(cu[s], cu[s + 1])
            R[s] = d[t][~out[t]].sum()
            if length_norm and cu[s + 1] > cu[s]:
                R[s] /= cu[s + 1] - cu[s]
        members = [s for s in seqs if cu[s + 1] > cu[s] and np.isfinite(rewards[s])]
        P = preference_pairs(rewards, members, pairs)
        q_pairs[q] = len(P)
        for i, j in P:
            l, dl = pair_loss(R[i] - R[j], beta, kind, label_smoothing)
            q_loss[q] += l / len(P)
            q_margin[q] += beta * (R[i] - R[j]) / len(P)
            gR[i] += grad_scale * dl / (Q * len(P))
            gR[j] -= grad_scale * dl / (Q * len(P))
        for s in seqs:
            n = cu[s + 1] - cu[s]
            g[cu[s]:cu[s + 1]] = np.where(out[cu[s]:cu[s + 1]], 0.0, gR[s] / n if length_norm and n else gR[s])
    return {"loss": q_loss.sum() / Q, "gscale": g, "seq_logratio": R, "seq_grad": gR, "q_loss": q_loss,
            "q_margin": q_margin, "q_pairs": q_pairs}
