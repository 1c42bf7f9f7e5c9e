"""Pages of sequences and log probabilities, from their definitions -- TEST INFRASTRUCTURE ONLY.

Plain Python and numpy on float64; shares no code with the product library.

pages(old, keep, new, table, free, page)  -> the counts, slots and positions after a step, table and free list in place
order(row)                                -> indices of a row of logits, largest first, equal ones by index, NaN last
logprobs(row, scale)                      -> Row: log-sum, entropy, log probabilities, and bounds on fp32 errors
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np


def pages(old, keep, new, table, free, page):
    """old, keep, new: tokens of each sequence (a sequence keeps at most what it has).  table: list of lists of page ids;
    free: list.  Returns (lengths, refused, [(slot, position)] of the new tokens in order)."""
    blocks = len(table[0])
    need = [(-(-o // page), -(-(k + n) // page)) for o, k, n in zip(old, keep, new)]
    for b, (have, want) in enumerate(need):
        if want <= blocks:
            free += table[b][want:have]
    there, asked, lengths, refused, out = len(free), 0, [], 0, []
    for b, (have, want) in enumerate(need):
        ok = want <= blocks
        if ok and want > have:
            asked += want - have
            ok = asked <= there
            if ok:
                for i in range(have, want):
                    table[b][i] = free.pop()
        lengths.append(keep[b] + new[b] if ok else old[b])
        refused += not ok
        for i in range(keep[b], keep[b] + new[b]):
            out.append((table[b][i // page] * page + i % page, i) if ok else (-1, -1))
    return lengths, refused, out


def order(row: np.ndarray) -> np.ndarray:
    nan = np.isnan(row)
    return np.lexsort((np.arange(len(row)), -np.where(nan, 0, row) + 0.0, nan))


@dataclass
class Row:
    lse: float
    entropy: float
    p: np.ndarray      # log probabilities
    tol_lse: float
    tol_entropy: float
    tol_p: np.ndarray


def logprobs(row: np.ndarray, scale: float) -> Row:
    """Bounds, u = 2^-24: an exponent x = (l - m) scale log2 e has 4 roundings (difference, two in the constant, product), so a
    term 2^x is off by 4 u ln2 |x| and 2 u of the exponential itself; a moved reference adds the same again for the way that it
    moves.  Sums run over at most n = V / 64 + 200 terms, joins and moves in a row, a rounding each (of an fp64 sum they are
    less, which the tests of single elements bound for themselves).  The logarithm is off by
    4 u of itself, a result by one rounding."""
    row = np.asarray(row, np.float64)
    V = len(row)
    if np.isnan(row).any() or np.isposinf(row).any():
        nan = np.full(V, math.nan)
        return Row(math.nan, math.nan, nan, 0.0, 0.0, nan)
    top = row.max()
    if np.isneginf(top):
        return Row(-math.inf, 0.0, np.full(V, -math.inf), 0.0, 0.0, np.zeros(V))
    u, n = 2.0 ** -24, V / 64 + 200
    s = (row - top) * scale
    e = np.exp(s)
    total = e.sum()
    log_s = math.log(total)
    w, x = e / total, np.where(e > 0, np.abs(s), 0)
    d_sum = u * (8 * (w @ x) + 2 + n) + 1e-30         # relative, of the sum
    d_log = d_sum + 4 * u * log_s
    d_mean = u * (8 * (w @ (x * x)) + (6 + n) * (w @ x)) + (w @ x) * d_sum
    p = s - log_s
    with np.errstate(invalid="ignore"):
        tol_p = d_log + u * (2 * np.abs(s) + np.abs(p))
    return Row(top * scale + log_s, log_s + (w @ x), p, d_log + u * (abs(top * scale + log_s) + abs(top * scale)),
               d_log + d_mean + u * (log_s + 3 * (w @ x)), tol_p)
