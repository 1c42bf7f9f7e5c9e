"""The norm, the attention and the 8-bit cache in 64 bits, from their definitions -- TEST INFRASTRUCTURE ONLY.

Plain numpy on float64 values of the inputs, one query row at a time; shares no code with the product library.

rmsnorm(x, residual, weight, eps)        -> (v, u): the residual sum and the norm
group_scales(u, fmt)                     -> (scales, width of a group) of the 8-bit forms: "group", "mx", "row"
attend(q, k, v, scale)                   -> Attended of one query row over keys k [n, dk], values v [n, dv]
append(...)                              -> the 8-bit cache after new tokens, in place
E4M3                                     float64 value of every e4m3fn code
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np


def _e4m3_table() -> np.ndarray:
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if (e, m) == (15, 7) else (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = -v if c & 0x80 else v
    return out


E4M3 = _e4m3_table()
_POS = E4M3[:127]  # 0 .. 448, ascending with the code


def e4m3(v: np.ndarray) -> np.ndarray:
    """Nearest codes, ties to the even code, saturating at 448; NaN gives 0x7f."""
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(v), 0, v)), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    code = code | (np.signbit(v).astype(np.int64) << 7)
    return np.where(np.isnan(v), 0x7F, code).astype(np.uint8)


def rmsnorm(x, residual, weight, eps):
    v = np.asarray(x, np.float64) + (0 if residual is None else np.asarray(residual, np.float64))
    return v, v / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps) * np.asarray(weight, np.float64)


def group_scales(u, fmt):
    """fp64 scales [T, groups] of the norm u [T, d] by format, and the width of a group."""
    d = u.shape[1]
    width = {"group": 128, "mx": 32, "row": d}[fmt]
    top = np.stack([np.abs(u[:, i:i + width]).max(1) for i in range(0, d, width)], 1)
    if fmt != "mx":
        return np.maximum(top, 2.0 ** -100) / 448, width
    e = np.where(top == 0, -127, np.clip(np.floor(np.log2(np.where(top == 0, 1, top))) - 8, -127, 127))
    return 2.0 ** e, width


@dataclass
class Attended:
    o: np.ndarray      # [dv]
    lse: float
    spread: np.ndarray  # [dv]: sum of weight * |value|, what a relative error of the weights moves at most
    delta: float       # bound on an fp32 score's error: roundings of the products' sum and of the scaling


def attend(q, k, v, scale) -> Attended:
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    if not len(k):
        return Attended(np.zeros(v.shape[1]), -math.inf, np.zeros(v.shape[1]), 0.0)
    s = scale * (k @ q)
    top = s.max()
    e = np.exp(s - top)
    w = e / e.sum()
    size = abs(scale) * (np.abs(k) @ np.abs(q)).max()
    delta = 2.0 ** -24 * ((len(q) + 4) * size + 8 * np.abs(s).max() + 4)
    return Attended(w @ v, top + math.log(e.sum()), w @ np.abs(v), delta)


def tolerances(a: Attended, n: int):
    """Elementwise bound on a bf16 output and bound on the fp32 log-sum, from the arithmetic that the library states: bf16
    weights (2^-8 of each), fp32 scores (delta each, twice: a weight and the sum), fp32 sums over n keys, one final bf16
    rounding."""
    rel = 2.0 ** -8 + 2 * a.delta + (n + 64) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(a.o) + 1.01 * rel * a.spread + 1e-38, a.delta + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * abs(a.lse)


def power_scale(top: float) -> float:
    """The smallest power of two >= top / 448, at least 2^-126."""
    if top == 0:
        return 2.0 ** -126
    m, e = math.frexp(top)  # top = m * 2^e, 448 = 0.875 * 2^9
    return 2.0 ** max(e - 9 if m <= 0.875 else e - 8, -126)


def append(k_new, v_new, rows, offsets, k, v, k_scale, v_scale, table, cache_len):
    """The cache arrays (codes u8 k [P, H, page, D], v [P, H, D, page], scales) after the new tokens, in place."""
    page, blocks = k.shape[2], table.shape[1]
    for b in range(len(cache_len)):
        mine = [int(rows[i]) for i in range(offsets[b], offsets[b + 1])]
        mine = mine[:max(0, blocks * page - int(cache_len[b]))]
        done = 0
        while done < len(mine):
            at = int(cache_len[b]) + done
            slot, pg = at % page, int(table[b, at // page])
            m = min(page - slot, len(mine) - done)
            for src, codes, scales, turn in ((k_new, k, k_scale, False), (v_new, v, v_scale, True)):
                for h in range(k.shape[1]):
                    new = np.asarray(src[mine[done:done + m], h], np.float64)
                    fin = np.abs(new[np.isfinite(new)])
                    need = power_scale(float(fin.max()) if fin.size else 0.0)
                    page_codes = codes[pg, h].T if turn else codes[pg, h]  # [page, D], a view
                    was = float(scales[pg, h]) if slot else 0.0
                    unit = max(was, need)
                    if slot and unit > was:  # every slot; the new tokens' are written next
                        page_codes[:] = e4m3(E4M3[page_codes] * (was / unit))
                    page_codes[slot:slot + m] = e4m3(new / unit)
                    scales[pg, h] = unit
            done += m
