"""A gradient of a projection against the forward product along it (test infrastructure).

y = x w^T is linear in each operand, so sum(dy * y(u, w)) = sum(dx * u) for every u, and sum(dy * y(x, v)) =
sum(dw * v) for every v, but for roundings.  Along the gradient itself both sides are its sum of squares, where no
error can hide: a gradient of zeros leaves the whole of it, one that lacks a part of its sum that part.

Roundings to bf16 are off by up to 2^-8 of a value, one way or the other: sums of n such errors b_i exceed
6 sqrt(sum b_i^2) with a probability of 2 e^-18 (Hoeffding).  What the sums themselves may be off by is added as it is.
"""
import numpy as np


def rounded(a):
    """What bf16 roundings of a's entries do to their sum."""
    return 6.0 * np.sqrt(((2.0 ** -8 * a) ** 2).sum())


def sums_off(x, w):
    """By how much each of x w^T may be off before its rounding (include/aeris_fp8.h)."""
    n, c = x.shape
    most = lambda a: np.abs(a).reshape(a.shape[0], c // 8, 8).max(axis=2)
    return 7 * 2.0 ** -13 * (most(x) @ most(w).T) + (c / 16 + 8) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def along_dx(y, dx, u, dy, w, wt):
    """(gap, tolerance, size) for y = y(u, w) and dx = dy wt^T.  w [f, c] and its transpose wt [c, f] are quantised apart:
    what they differ by is taken out exactly."""
    gap = (y * dy).sum() - (dx * u).sum() - (dy * (u @ (w - wt.T).T)).sum()
    allow = (rounded(y * dy) + (sums_off(u, w) * np.abs(dy)).sum() +
             rounded(dx * u) + (sums_off(dy, wt) * np.abs(u)).sum())
    return abs(gap), allow, (dx * u).sum()


def along_dw(y, dw, v, dy, x):
    """(gap, tolerance, size) for y = y(x, v) and dw = dy^T x in fp32, whose sums are off by up to 1e-5 of their terms."""
    gap = (y * dy).sum() - (dw * v).sum()
    allow = (rounded(y * dy) + (sums_off(x, v) * np.abs(dy)).sum() +
             1e-5 * ((np.abs(dy).T @ np.abs(x)) * np.abs(v)).sum())
    return abs(gap), allow, (dw * v).sum()
