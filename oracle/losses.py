"""fp64 reference of the losses over a vocabulary (test infrastructure only).

For n tokens with hidden states x (n x h), a head w (v x h) and logits z = x w^T / T the softmax cross entropy of hard
labels and the KL divergence from a teacher's top logits, with the gradients of x and w. The logits are held whole.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np


class Loss(NamedTuple):
    loss: float
    token_loss: np.ndarray   # n
    lse: np.ndarray          # n
    dz: np.ndarray           # n x v: d loss / d (x w^T)
    dx: np.ndarray
    dw: np.ndarray
    z: np.ndarray            # n x v


def _finish(x, w, z, q, ent, on, weight, reduction, scale, inv_t, z_loss) -> Loss:
    """q: n x v target weights (rows add up to 1 where `on`), ent: their sum of q log q."""
    n = x.shape[0]
    top = z.max(1) if n else np.zeros(0)
    e = np.exp(z - top[:, None])
    others = e.copy()  # the sum without its largest term, which is 1: a sure token's loss is far below that 1
    others[np.arange(n), z.argmax(1)] = 0.0
    others = np.log1p(others.sum(1))
    lse = top + others
    token = np.where(on, ent + (q * (top[:, None] - z)).sum(1) + others + z_loss * lse ** 2, 0.0)
    a = np.where(on, np.ones(n) if weight is None else np.asarray(weight, np.float64), 0.0)
    denom = a.sum() if reduction == "mean" else 1.0
    g = np.zeros(n) if denom == 0 else scale * a / denom
    p = e / e.sum(1)[:, None]
    # p - q near q = 1: minus the sum of the other probabilities
    one = q == 1.0
    rest = np.where(one, 0.0, p).sum(1)
    pq = np.where(one, -rest[:, None], p - q)
    dz = (g * inv_t)[:, None] * (pq + (2 * z_loss * lse)[:, None] * p)
    loss = 0.0 if denom == 0 else scale * float((a * token).sum()) / denom
    return Loss(loss, token, np.where(on, lse, 0.0), dz, dz @ w, dz.T @ x, z)


def linear_xent(x, w, targets, *, ignore_index: int = -100, reduction: str = "mean", scale: float = 1.0,
                weight: Optional[np.ndarray] = None, z_loss: float = 0.0) -> Loss:
    """l_r = lse_r - z_{r,t_r} + z_loss lse_r^2; tokens labelled ignore_index do not count (their x is taken as 0)."""
    on = np.asarray(targets) != ignore_index
    x = np.where(on[:, None], np.asarray(x, np.float64), 0.0)
    w = np.asarray(w, np.float64)
    z = x @ w.T
    q = np.zeros_like(z)
    q[np.nonzero(on)[0], np.asarray(targets)[on]] = 1.0
    return _finish(x, w, z, q, np.zeros(len(on)), on, weight, reduction, scale, 1.0, z_loss)


def linear_distill(x, w, ids, logits, *, temperature: float = 1.0, reduction: str = "mean", scale: float = 1.0,
                   weight: Optional[np.ndarray] = None) -> Loss:
    """l_r = KL(q_r || p_r): q_r the softmax of logits_r / T over the slots with ids >= 0, p_r that of z_r over the
    vocabulary. A token without such a slot does not count."""
    ids = np.asarray(ids)
    t = np.where(ids >= 0, np.asarray(logits, np.float64) / temperature, -np.inf)
    on = (t > -np.inf).any(1)
    x = np.where(on[:, None], np.asarray(x, np.float64), 0.0)
    w = np.asarray(w, np.float64)
    z = x @ w.T / temperature
    top = np.where(on, t.max(1), 0.0)
    qs = np.exp(t - top[:, None])
    qs = qs / np.where(on, qs.sum(1), 1.0)[:, None]
    ent = np.where(qs > 0, qs * np.log(np.where(qs > 0, qs, 1.0)), 0.0).sum(1)
    q = np.zeros_like(z)
    np.add.at(q, (np.arange(len(on))[:, None], np.maximum(ids, 0)), np.where(ids >= 0, qs, 0.0))
    return _finish(x, w, z, q, ent, on, weight, reduction, scale, 1.0 / temperature, 0.0)
