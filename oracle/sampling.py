"""Sampling of one token a row of logits from a given number, in fp64 numpy,
written from the definition (temperature, then top-k, top-p of what it leaves,
min-p; inverse cumulative mass in the order of ids)."""

from __future__ import annotations

import numpy as np


def kept_mass(x, allowed=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Kept mass per token (0: not kept), or None if the row has no distribution."""
    x = np.asarray(x, dtype=np.float64)
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    if np.isnan([temperature, top_p, min_p]).any() or np.isnan(x).any() or np.isposinf(x).any() or not (x > -np.inf).any():
        return None
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if temperature <= 0:
        mass = np.zeros(len(x))
        mass[order[0]] = 1.0
        return mass
    with np.errstate(over="ignore"):
        m = np.exp((x[order] - x[order[0]]) / temperature)
    keep = np.ones(len(order), dtype=bool)
    if top_k > 0:
        keep[top_k:] = False
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(m)[:-1]])
        keep &= before < max(top_p, 0.0) * m[keep].sum()
    if min_p > 0:
        keep &= m >= min(min_p, 1.0)
    keep[0] = True
    mass = np.zeros(len(x))
    mass[order[keep]] = m[keep]
    return mass


def confidence(x, allowed=None) -> float:
    x = np.asarray(x, dtype=np.float64)
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    return float(1.0 / np.exp(x - x.max()).sum())


def sample(x, u, allowed=None, **how):
    """(token, prob, confidence, distance of the goal from the nearest border, relative to the kept mass)."""
    mass = None if np.isnan(u) else kept_mass(x, allowed, **how)
    if mass is None:
        return -1, 0.0, 0.0, np.inf
    upto = np.cumsum(mass)
    total, ids = upto[-1], np.flatnonzero(mass)
    over = ids[upto[ids] > u * total]
    token = int(over[0] if len(over) else ids[-1])
    borders = upto[ids[:-1]]
    gap = np.abs(borders - u * total).min() / total if len(borders) else np.inf
    return token, mass[token] / total, confidence(x, allowed), gap
