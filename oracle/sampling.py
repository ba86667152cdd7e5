"""CPU oracle, part 6: one token of a row of logits from a given random number (test infrastructure only; nothing in the product path imports this).

Tokens in the order of their logits, descending, ties to the lower index; a token's mass is exp((logit - largest) / temperature).  Kept are the first
top_k of them, of those the tokens before which less than top_p of their mass lies (the first always), of those the ones whose mass is at least
min_p times the largest's; drawn is the first kept token up to and with which more than u of the kept mass lies.
"""
from __future__ import annotations

import numpy as np


def kept_tokens(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token ids in their order, their masses), in 64 bits; both empty where nothing can be drawn."""
    l = np.asarray(logits, dtype=np.float64) + 0.0
    can = l > -np.inf
    if np.isposinf(l).any():
        can = np.isposinf(l)
    ids = np.flatnonzero(can)
    if ids.size == 0:
        return ids, np.zeros(0)
    order = ids[np.argsort(-l[ids], kind="stable")]
    largest = l[order[0]]
    diff = np.where(l[order] == largest, 0.0, l[order] - largest if np.isfinite(largest) else 0.0)
    if not temperature > 0:
        return order[:1], np.ones(1)
    mass = np.exp(diff / temperature) if np.isfinite(temperature) else np.ones(order.size)
    if 0 < top_k < order.size:
        order, mass = order[:top_k], mass[:top_k]
    if top_p < 1:
        keep = np.cumsum(mass) - mass < top_p * mass.sum()
        keep[0] = True
        order, mass = order[keep], mass[keep]
    if min_p > 0:
        keep = mass >= min(min_p, 1.0)
        order, mass = order[keep], mass[keep]
    return order, mass


def draw(logits, u, **settings):
    """(token, probability, distance of u from the nearest border between two tokens, as a share of the kept mass)."""
    order, mass = kept_tokens(logits, **settings)
    if order.size == 0:
        return -1, 0.0, 1.0
    through = np.cumsum(mass) / mass.sum()
    u = min(max(float(u), 0.0), 1.0) if u == u else 0.0
    j = min(int(np.searchsorted(through, u, side="right")), int((mass > 0).sum()) - 1)
    return int(order[j]), float(mass[j] / mass.sum()), float(np.abs(through[:-1] - u).min()) if order.size > 1 else 1.0
