"""The router's definition in 64 bits, and how far fp32 may be from it.

Errors are counted in steps of u = 2^-24, a rounding's relative size.  With t the
distance of a logit from its row's largest, exp(t) is made of t's rounding (|t|
in the result), t / ln 2 with a constant of 24 bits (2 |t|) and an exponential off
by a step of the type (2): r = 3 |t| + 3 covers it.  A row's sum adds 16 terms on
a lane and 6 levels of lanes: its relative error is s = sum_e p_e r_e + 22, and
p's is r + s + 3 with the reciprocal and the product.  The largest of the logarithm of
the sum: s for the sum, 2 steps of the type for the logarithm, one for the addition.
"""
import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126  # exponentials below the smallest normal number may be 0


class Row:
    """Softmax of logits [n, E] in 64 bits with its error bounds; rows that do not count are zeros."""

    def __init__(self, logits, live=None):
        l64 = logits.astype(np.float64)
        with np.errstate(invalid="ignore"):
            self.counted = (l64 > -np.inf).any(1)
        if live is not None:
            self.counted &= live.astype(bool)
        l64 = np.where(self.counted[:, None], l64, 0.0)
        self.logits = l64
        top = l64.max(1, keepdims=True)
        t = np.where(np.isneginf(l64), 0.0, top - l64)
        e = np.exp(l64 - top)
        total = e.sum(1, keepdims=True)
        self.p = np.where(self.counted[:, None], e / total, 0.0)
        self.r = 3 * t + 3
        self.s = (self.p * self.r).sum(1, keepdims=True) + 22
        self.p_err = self.p * (self.r + self.s + 3) * U + TINY
        log = np.log(total[:, 0])
        self.lse = np.where(self.counted, top[:, 0] + log, 0.0)
        self.lse_err = (self.s[:, 0] + 4 * log + np.abs(self.lse)) * U


def choices(logits, k, bias=None, live=None):
    """The experts of the largest scores, int32 [n, k]: equal ones from the lowest number on."""
    row = Row(logits, live)
    score = logits.astype(np.float32) + (np.float32(0) if bias is None else bias.astype(np.float32))
    ids = np.full((logits.shape[0], k), -1, dtype=np.int32)
    for n in np.nonzero(row.counted)[0]:
        fit = np.nonzero(score[n] > -np.inf)[0]
        order = fit[np.argsort(-score[n][fit], kind="stable")][:k]
        ids[n, :len(order)] = order
    return ids


def weights(row, ids, normalise):
    """(weights, error bounds) [n, k]."""
    at = np.maximum(ids, 0)
    here = (ids >= 0) & row.counted[:, None]
    n = np.arange(ids.shape[0])[:, None]
    if not normalise:
        return np.where(here, row.p[n, at], 0.0), np.where(here, row.p_err[n, at], 0.0)
    l = np.where(here, row.logits[n, at], -np.inf)
    top = np.where(here.any(1), l.max(1), 0.0)[:, None]
    t = np.where(here, top - l, 0.0)
    e = np.where(here, np.exp(-t), 0.0)
    w = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
    s = (w * (3 * t + 3)).sum(1, keepdims=True) + ids.shape[1] + 6
    return w, np.where(here, w * (3 * t + 3 + s + 2) * U + TINY, 0.0)


def totals(row, ids, E, chain):
    """(counts [E + 1], sums [E + 1] and their bounds, losses and their bounds); chain: the most additions of a sum."""
    k = ids.shape[1]
    T = int(row.counted.sum())
    counts = np.append(np.bincount(ids[ids >= 0], minlength=E), T).astype(np.int64)
    sums = np.append(row.p.sum(0), (row.lse ** 2).sum())
    err = np.append(row.p_err.sum(0), (2 * np.abs(row.lse) * row.lse_err).sum()) + (chain + 2) * U * sums
    if not T:
        return counts, sums, err, np.zeros(2), np.zeros(2)
    balance = E / (k * T * T) * (counts[:-1] * sums[:-1]).sum()
    balance_err = E / (k * T * T) * (counts[:-1] * err[:-1]).sum() + 40 * U * balance
    return counts, sums, err, np.array([balance, sums[-1] / T]), np.array([balance_err, err[-1] / T + 3 * U * sums[-1] / T])


def gradient(row, ids, normalise, dweights, counts, dlosses):
    """(dlogits, error bounds) [n, E]."""
    n, E = row.p.shape
    k = ids.shape[1]
    grad, err = np.zeros((n, E)), np.zeros((n, E))
    shift, shift_err = np.zeros(n), np.zeros(n)
    pull = np.zeros(E)
    size = np.zeros(n)  # of what is added up to a shift
    if dlosses is not None and counts[-1] > 0:
        T = float(counts[-1])
        pull = dlosses[0] * E / (k * T * T) * counts[:-1]
        q = 2 * dlosses[1] / T * row.lse
        dot = (row.p * pull).sum(1)
        shift = q - dot
        shift_err = 2 * np.abs(dlosses[1]) / T * row.lse_err + 6 * U * np.abs(q) + (row.p_err * np.abs(pull)).sum(1) + 40 * U * np.abs(dot)
        size = np.abs(q) + np.abs(dot)
    direct, direct_err = np.zeros((n, E)), np.zeros((n, E))
    if dweights is not None:
        w, w_err = weights(row, ids, normalise)
        here = (ids >= 0) & (ids < E) & row.counted[:, None]
        d = np.where(here, dweights, 0.0)
        dot = (w * d).sum(1)
        dot_err = (w_err * np.abs(d)).sum(1) + (k + 8) * U * (w * np.abs(d)).sum(1)
        inner = d - (dot[:, None] if normalise else 0.0)
        part = w * inner
        part_err = w_err * np.abs(inner) + 3 * U * np.abs(part) + (w * (dot_err + U * np.abs(dot))[:, None] if normalise else 0.0)
        rows, places = np.nonzero(here)
        np.add.at(direct, (rows, ids[rows, places]), part[rows, places])
        np.add.at(direct_err, (rows, ids[rows, places]), part_err[rows, places])
        if not normalise:
            shift, shift_err, size = shift - dot, shift_err + dot_err, size + np.abs(dot)
    inside = pull[None] + shift[:, None]
    grad = row.p * inside + direct
    err = (row.p_err * np.abs(inside) + row.p * (shift_err + 3 * U * size)[:, None] + row.p * 8 * U * np.abs(pull)[None] + direct_err +
           4 * U * (np.abs(row.p * inside) + np.abs(direct)) + 4 * TINY)
    grad[~row.counted], err[~row.counted] = 0.0, 0.0
    return grad, err
