"""Seeded draws for the attention and cache operators: paged caches, ragged batches of drafts, tree masks.

Like the rest of the package it only draws inputs; none of the operators' arithmetic is here.
"""
from __future__ import annotations

import numpy as np
import torch

from . import generator


def normal(seed: int, tag: str, *shape, std: float = 1.0) -> torch.Tensor:
    return torch.empty(*shape).normal_(0.0, std, generator=generator(seed, tag)).to(torch.bfloat16)


def offsets(counts) -> torch.Tensor:
    return torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32)


def tree_masks(counts, seed: int) -> torch.Tensor:
    """int64 [N]: each draft sees itself and its ancestors in a random tree of its sequence."""
    rng, out = np.random.default_rng(seed), []
    for n in counts:
        m = []
        for i in range(n):
            up = int(rng.integers(max(0, i - 5), i)) if i else -1
            m.append((m[up] if up >= 0 else 0) | 1 << i)
        out += [w - (1 << 64) if w >> 63 else w for w in m]
    return torch.tensor(out, dtype=torch.int64)


def page_table(lens, page: int, seed: int, spare: int = 2, room: int = 0):
    """(int32 [B, blocks], number of pages): pages in random order, some that no sequence has, and `room` tokens more
    than each length; entries past a sequence's pages name page 0."""
    rng = np.random.default_rng(seed)
    need = [max(1, -(-(n + room) // page)) for n in lens]
    order = rng.permutation(sum(need) + spare).astype(np.int32)
    table = np.zeros((len(lens), max(need)), np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table), len(order)


def codes(seed: int, tag: str, *shape) -> torch.Tensor:
    """uint8 e4m3fn codes of finite values."""
    c = torch.randint(0, 254, shape, generator=generator(seed, tag), dtype=torch.int64)
    return torch.where(c < 127, c, c + 1).to(torch.uint8)  # 0x7f and 0xff are NaN


def power_scales(seed: int, tag: str, *shape) -> torch.Tensor:
    return torch.exp2(torch.randint(-9, -6, shape, generator=generator(seed, tag)).float())
