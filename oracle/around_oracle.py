"""CPU oracle of the operators around the expert layer.  TEST INFRASTRUCTURE ONLY.

Residual addition and RMS norm with its gradients, the balance loss of a router with its gradient, and low-rank adapters
added to a projection's output: fp64 throughout; the residual's sum alone is rounded to bf16, since the norm is one of the
stored stream.

Pins (tests/test_around_oracle.py): gradients against central differences, loss values of even and one-sided loads, empty
and masked cases, adapters against scalar loops.
"""
from __future__ import annotations

import numpy as np

from oracle import fp8_oracle as f8


# ------------------------------------------------------------------------------------------------------------- norm
def residual_sum(x, residual):
    """bf16(x + residual), as fp64."""
    x = np.asarray(x, np.float64)
    return x if residual is None else f8.round_to_bf16(x + np.asarray(residual, np.float64)).astype(np.float64)


def rms_norm(s, gain, eps, offset=0.0):
    """n [rows, cols] of the stream s."""
    s = np.asarray(s, np.float64)
    return s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * (np.asarray(gain, np.float64) + offset)


def rms_norm_backward(s, gain, d_out, d_sum, eps, offset=0.0):
    """d_x, d_gain and what their rounding errors are relative to."""
    s, d = np.asarray(s, np.float64), np.asarray(d_out, np.float64)
    rstd = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    h, g = s * rstd, d * (np.asarray(gain, np.float64) + offset)
    dx = rstd * (g - h * (g * h).mean(1, keepdims=True))
    size = rstd * (np.abs(g) + np.abs(h) * np.abs(g * h).mean(1, keepdims=True))
    if d_sum is not None:
        dx = dx + d_sum
        size = size + np.abs(d_sum)
    return dx, (d * h).sum(0), size, np.abs(d * h).sum(0)


# ---------------------------------------------------------------------------------------------------------- balance
def sequence_of(T, offsets, mask):
    """Sequence of every token, -1 for those that do not count."""
    seq = np.zeros(T, np.int64) if offsets is None else np.searchsorted(np.asarray(offsets)[1:], np.arange(T), side="right")
    if offsets is not None:
        seq[np.arange(T) >= offsets[-1]] = -1
        seq[np.arange(T) < offsets[0]] = -1
    if mask is not None:
        seq[np.asarray(mask) == 0] = -1
    return seq


def probabilities(x, score):
    """p [T, E] and log(sum(exp(x))) [T]; rows without an expert have p = 0 and -inf."""
    x = np.asarray(x, np.float64)
    top = x.max(1, keepdims=True)
    top = np.where(np.isneginf(top), 0.0, top)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        e = np.exp(x - top)
        total = e.sum(1, keepdims=True)
        lse = (np.log(total) + top)[:, 0]
        if score == "sigmoid":
            # sigma(x) over its largest: in range for any x
            ls = -np.logaddexp(0.0, -x)
            most = ls.max(1, keepdims=True)
            e = np.exp(ls - np.where(np.isneginf(most), 0.0, most))
            total = e.sum(1, keepdims=True)
        p = np.where(total > 0, e / np.where(total == 0, 1, total), 0.0)
    return p, lse


def balance_loss(logits, ids, score, coef, z_coef, offsets=None, mask=None, sequences=1):
    """counts [S,E], tokens [S+1], mean [S,E], loss [2]."""
    T, E = logits.shape
    k = ids.shape[1]
    seq = sequence_of(T, offsets, mask)
    p, lse = probabilities(logits, score)
    counts, mean = np.zeros((sequences, E), np.int64), np.zeros((sequences, E))
    tokens = np.zeros(sequences + 1, np.int64)
    loss = 0.0
    for q in range(sequences):
        mine = seq == q
        n = tokens[q] = mine.sum()
        if n:
            chosen = ids[mine].reshape(-1)
            counts[q] = np.bincount(chosen[(chosen >= 0) & (chosen < E)], minlength=E)
            mean[q] = p[mine].mean(0)
            loss += (E * counts[q] / (k * n) * mean[q]).sum()
    used = seq >= 0
    tokens[-1] = used.sum()
    z = np.where(np.isneginf(lse), 0.0, lse)[used]
    return counts, tokens, mean, np.array([coef / sequences * loss, z_coef * (z * z).mean() if used.any() else 0.0])


def balance_loss_backward(logits, counts, tokens, k, score, coef, z_coef, d_loss=1.0, offsets=None, mask=None, sequences=1):
    """Gradient [T,E], and per element what its rounding errors are relative to."""
    T, E = logits.shape
    seq = sequence_of(T, offsets, mask)
    p, lse = probabilities(logits, score)
    soft, _ = probabilities(logits, "softmax")
    n = np.maximum(np.asarray(tokens, np.float64)[:-1], 1)
    u = d_loss * coef * E / (sequences * k) * np.asarray(counts, np.float64) / (n * n)[:, None]
    u = np.where((seq >= 0)[:, None], u[np.maximum(seq, 0)], 0.0)
    own = 1.0
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            own = 1 / (1 + np.exp(np.asarray(logits, np.float64)))
    dx = p * (u - (u * p).sum(1, keepdims=True)) * own
    size = p * (np.abs(u) + (np.abs(u) * p).sum(1, keepdims=True)) * own
    if z_coef:
        f = d_loss * 2 * z_coef / max(1, int(tokens[-1])) * np.where(np.isneginf(lse) | (seq < 0), 0.0, lse)
        dx = dx + f[:, None] * soft
        size = size + np.abs(f)[:, None] * soft
    return dx, size


# --------------------------------------------------------------------------------------------------------- adapters
def add_adapters(x, a, b, scale, adapter_of, y, offsets=None):
    """y + scale b (a x) by segments, fp64; and the sizes its rounding errors are relative to: of t's sums carried through b, and
    of the second product's."""
    y = np.array(y, np.float64)
    size_t, size_y = np.zeros_like(y), np.zeros_like(y)
    bounds = np.arange(len(x) + 1) if offsets is None else np.asarray(offsets)
    for i, adapter in enumerate(adapter_of):
        lo, hi = int(bounds[i]), int(bounds[i + 1])
        if hi > lo and 0 <= adapter < len(a):
            f = 1.0 if scale is None else float(scale[adapter])
            xs, A, B = (np.asarray(v, np.float64) for v in (x[lo:hi], a[adapter], b[adapter]))
            t = xs @ A.T
            y[lo:hi] += f * (t @ B.T)
            size_t[lo:hi] = abs(f) * ((np.abs(xs) @ np.abs(A).T) @ np.abs(B).T)
            size_y[lo:hi] = abs(f) * (np.abs(t) @ np.abs(B).T)
    return y, size_t, size_y
