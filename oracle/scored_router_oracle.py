"""CPU oracle for scored routing and the gradients of the gate.  TEST INFRASTRUCTURE ONLY.

Per token, in explicit loops over fp64 numbers: scores (softmax over all experts, or a sigmoid of each), choice values
(score + balance bias, or the logits themselves without one), the best groups, the k best experts of those, weights
from the unbiased scores.  A logit of -inf masks its expert; a NaN (or +inf under softmax) spoils its token's weights.

Pins (tests/test_scored_router_oracle.py): the plain rule against ``moe_oracle.topk_route``, hand-worked groups, ties
and masks, weights that sum to the scale, and both gradients against central differences of the forward functions.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np


@dataclass(frozen=True)
class Rule:
    score: str = "softmax"
    n_group: int = 1
    topk_group: int = 1
    group_top: int = 1
    renormalise: bool = True
    weight_scale: float = 1.0


def scores(x: np.ndarray, rule: Rule) -> np.ndarray:
    """x [E] fp64 -> scores; masked experts score 0 (all zeros when every expert is masked)."""
    x = np.asarray(x, dtype=np.float64)
    if rule.score == "sigmoid":
        return np.array([0.0 if v == -math.inf else (1.0 / (1.0 + math.exp(-v)) if v > -700 else math.exp(v)) for v in x])
    top = np.max(x)
    if top == -math.inf:
        return np.zeros_like(x)
    with np.errstate(invalid="ignore"):
        e = np.exp(x - top)
    return e / e.sum()


def spoiled(x: np.ndarray, rule: Rule) -> bool:
    return bool(np.isnan(x).any() or (rule.score == "softmax" and np.isposinf(x).any()))


def choice_values(x: np.ndarray, bias, rule: Rule) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    c = x.copy() if bias is None else scores(x, rule) + np.asarray(bias, dtype=np.float64)
    c[x == -math.inf] = -math.inf
    c[np.isnan(c)] = -math.inf
    return c


def select(x: np.ndarray, bias, rule: Rule, k: int):
    """Chosen experts of one token, in slot order, and the choice values."""
    E = len(x)
    c = choice_values(x, bias, rule)
    size = E // rule.n_group
    rank = c
    if bias is None and rule.group_top == 2:
        rank = np.where(np.isneginf(c), -math.inf, scores(np.where(np.isnan(x), -math.inf, x), rule))
    worth = []
    for g in range(rule.n_group):
        best = sorted(rank[g * size:(g + 1) * size], reverse=True)[:rule.group_top]
        worth.append(best[0] + sum(v for v in best[1:] if v > -math.inf))
    kept = sorted(range(rule.n_group), key=lambda g: (-worth[g], g))[:rule.topk_group]
    open_ = [e for e in range(E) if e // size in kept]
    return sorted(open_, key=lambda e: (-c[e], e))[:k], c


def weights(x: np.ndarray, ids, rule: Rule) -> np.ndarray:
    if spoiled(x, rule):
        return np.full(len(ids), np.nan)
    s = scores(x, rule)[list(ids)]
    if rule.renormalise:
        if rule.score == "softmax":      # relative to the largest chosen logit, so that nothing underflows
            s = scores(np.asarray(x, np.float64)[list(ids)], rule)
        total = s.sum()
        s = s / total if total > 0 else np.zeros_like(s)
    return s * rule.weight_scale


def route(logits: np.ndarray, bias, rule: Rule, k: int):
    """ids [T,k] int32, weights [T,k] fp64."""
    T = logits.shape[0]
    ids = np.zeros((T, k), dtype=np.int32)
    w = np.zeros((T, k))
    for t in range(T):
        ids[t] = select(logits[t], bias, rule, k)[0]
        w[t] = weights(logits[t], ids[t], rule)
    return ids, w


def routing_backward(logits: np.ndarray, ids: np.ndarray, d_w: np.ndarray, rule: Rule) -> np.ndarray:
    """d(sum_j w_j d_w_j) / d logits with the choice held fixed, fp64 [T,E]."""
    out = np.zeros(logits.shape)
    for t in range(logits.shape[0]):
        x, sel = np.asarray(logits[t], np.float64), list(ids[t])
        if spoiled(x, rule):
            out[t] = np.nan
            continue
        g = np.asarray(d_w[t], np.float64) * rule.weight_scale
        s = scores(x, rule)
        if rule.score == "sigmoid":
            ds = g.copy()
            if rule.renormalise:
                total = s[sel].sum()
                ds = (g - (g * s[sel]).sum() / total) / total if total > 0 else np.zeros_like(g)
            for j, e in enumerate(sel):
                out[t, e] += ds[j] * s[e] * (1.0 - s[e])
        elif rule.renormalise:
            q = scores(x[sel], rule)
            for j, e in enumerate(sel):
                out[t, e] += q[j] * (g[j] - (g * q).sum())
        else:
            full = np.zeros_like(x)
            full[sel] = g
            out[t] = s * (full - (g * s[sel]).sum())
    return out


def combine_backward(d_out: np.ndarray, y_perm: np.ndarray, inv_perm: np.ndarray, w: np.ndarray):
    """d_y_perm [R,H] (before its rounding) and d_topk_w [T,k], fp64, slot by slot."""
    T, k = w.shape
    d_y = np.zeros(y_perm.shape)
    d_w = np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            row = inv_perm[t * k + j]
            d_y[row] = w[t, j] * d_out[t]
            d_w[t, j] = float(np.dot(d_out[t], y_perm[row]))
    return d_y, d_w
