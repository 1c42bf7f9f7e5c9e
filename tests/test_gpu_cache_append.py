"""moe_cache_append against its definition, bit for bit: codes and scales, pages begun, continued and left alone, scales
that grow, gathered rows, positions past the table, and non-finite values."""
import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import attention as ref
from synth import attention as draw

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")


def empty_cache(lens, Hkv, D, page, room, seed, fill=True):
    table, pages = draw.page_table(lens, page, seed, room=room)
    c = dict(k=draw.codes(seed, "k", pages, Hkv, page, D), v=draw.codes(seed, "v", pages, Hkv, D, page),
             ks=draw.power_scales(seed, "ks", pages, Hkv), vs=draw.power_scales(seed, "vs", pages, Hkv), table=table,
             len=torch.tensor(lens, dtype=torch.int32))
    return c


def run(c, kn, vn, off, rows=None, max_tokens=None):
    d = {x: t.to(DEV) for x, t in c.items()}
    moe.moe_cache_append(kn.to(DEV), vn.to(DEV), off.to(DEV), d["k"], d["v"], d["ks"], d["vs"], d["table"], d["len"],
                         rows=None if rows is None else rows.to(DEV), max_tokens=max_tokens)
    return d


def expect(c, kn, vn, off, rows=None):
    w = {x: t.numpy().copy() for x, t in c.items()}
    rows = np.arange(kn.shape[0]) if rows is None else rows.numpy()
    ref.append(kn.double().numpy(), vn.double().numpy(), rows, off.tolist(), w["k"], w["v"], w["ks"], w["vs"], w["table"], w["len"])
    return w


def same(d, w):
    for x in ("k", "v", "ks", "vs"):
        got = d[x].cpu().numpy()
        if got.dtype == np.uint8:  # the sign of a NaN code is not specified
            got, want = np.where(got == 0xFF, 0x7F, got), np.where(w[x] == 0xFF, 0x7F, w[x])
        else:
            want = w[x]
        assert np.array_equal(got, want), (x, np.argwhere(got != want)[:5])


CASES = [  # new tokens, cached tokens, Hkv, D, page
    ([1], [0], 1, 64, 16), ([3], [0], 2, 128, 16), ([1], [15], 2, 64, 16), ([1], [16], 2, 64, 16), ([40], [37], 3, 64, 16),
    ([5, 2, 7], [10, 31, 64], 8, 64, 32), ([4, 0, 1], [63, 5, 127], 4, 128, 64), ([300], [100], 4, 128, 128),
    ([129, 16], [0, 128], 2, 64, 128), ([700, 33], [3, 0], 1, 128, 64),
]


@pytest.mark.parametrize("counts,lens,Hkv,D,page", CASES)
@pytest.mark.parametrize("std", [0.01, 3.0, 900.0])
def test_append(counts, lens, Hkv, D, page, std):
    print(f"append counts={counts} lens={lens} Hkv={Hkv} D={D} page={page} std={std}", flush=True)
    N = sum(counts)
    c = empty_cache(lens, Hkv, D, page, max(counts), seed=N)
    kn, vn = draw.normal(N, "kn", N, Hkv, D, std=std), draw.normal(N, "vn", N, Hkv, D, std=std)
    off = draw.offsets(counts)
    w = expect(c, kn, vn, off)
    same(run(c, kn, vn, off, max_tokens=max(counts)), w)
    same(run(c, kn, vn, off), w)


def test_gathered_rows_and_growth_over_calls():
    """Accepted rows of a larger call, three verifications in a row with growing values; then the same tokens through the
    attention agree with the oracle's cache (the codes are the same arrays)."""
    lens, Hkv, D, page = [30, 5], 2, 64, 16
    c = empty_cache(lens, Hkv, D, page, 40, seed=8)
    for step in range(3):
        kn, vn = (draw.normal(step, t, 12, Hkv, D, std=0.1 * 7 ** step) for t in ("kn", "vn"))
        rows, off = torch.tensor([0, 3, 4, 9, 6, 11, 2], dtype=torch.int32), draw.offsets([4, 3])
        w = expect(c, kn, vn, off, rows)
        d = run(c, kn, vn, off, rows, max_tokens=4)
        same(d, w)
        c.update({x: d[x].cpu() for x in ("k", "v", "ks", "vs")})
        c["len"] = c["len"] + torch.tensor([4, 3], dtype=torch.int32)


def test_positions_past_the_table_are_dropped():
    c = empty_cache([20, 3], 2, 64, 16, 0, seed=9)  # two blocks and one
    kn, vn = draw.normal(9, "kn", 30, 2, 64), draw.normal(9, "vn", 30, 2, 64)
    off = draw.offsets([20, 10])
    same(run(c, kn, vn, off), expect(c, kn, vn, off))


def test_special_values():
    c = empty_cache([4, 0], 2, 64, 16, 20, seed=10)
    kn, vn = draw.normal(10, "kn", 12, 2, 64), draw.normal(10, "vn", 12, 2, 64)
    kn[1, 0, 5], kn[2, 1, 6], vn[3, 0, 7] = float("inf"), float("nan"), float("-inf")
    kn[6:, 0] = 0            # a head of zeros in a new page
    vn[6:, 1] = 2.0 ** -126  # below the smallest scale's range
    off = draw.offsets([6, 6])
    same(run(c, kn, vn, off), expect(c, kn, vn, off))


@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (128, 128)])
def test_scales_that_are_no_powers_of_two(D, page):
    """A continued page whose scale the caller chose: kept where it is enough, a power of two where it grows."""
    lens, counts = [page // 2 + 1, page - 1, 3], [4, 3, page]
    c = empty_cache(lens, 3, D, page, page, seed=11)
    for x in ("ks", "vs"):
        c[x] = torch.from_numpy(np.random.default_rng(11).uniform(0.002, 0.02, c[x].shape).astype(np.float32))
    kn, vn = draw.normal(11, "kn", sum(counts), 3, D, std=1.5), draw.normal(11, "vn", sum(counts), 3, D, std=0.7)
    kn[:, 1] *= 9
    off = draw.offsets(counts)
    same(run(c, kn, vn, off), expect(c, kn, vn, off))


def test_many_sequences_and_gathered_rows():
    """200 sequences, some with nothing new; rows in any order, the same one more than once."""
    rng = np.random.default_rng(12)
    lens, counts = [int(n) for n in rng.integers(0, 100, 200)], [int(n) for n in rng.integers(0, 25, 200)]
    c = empty_cache(lens, 2, 64, 16, 25, seed=12)
    kn, vn = draw.normal(12, "kn", 64, 2, 64), draw.normal(12, "vn", 64, 2, 64, std=4.0)
    rows = torch.from_numpy(rng.integers(0, 64, sum(counts)).astype(np.int32))
    off = draw.offsets(counts)
    w = expect(c, kn, vn, off, rows)
    same(run(c, kn, vn, off, rows), w)
    same(run(c, kn, vn, off, rows, max_tokens=24), w)


def test_other_stream_and_graph():
    """Captured once, replayed as the cache grows: the lengths are read on the device."""
    lens, counts, D, page = [5, 30], [3, 2], 64, 16
    c = empty_cache(lens, 2, D, page, 30, seed=13)
    d = {x: t.to(DEV) for x, t in c.items()}
    kn, vn = draw.normal(13, "kn", 5, 2, D).to(DEV), draw.normal(13, "vn", 5, 2, D).to(DEV)
    off = draw.offsets(counts).to(DEV)

    def call():
        moe.moe_cache_append(kn, vn, off, d["k"], d["v"], d["ks"], d["vs"], d["table"], d["len"], max_tokens=3)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call()
    torch.cuda.synchronize()
    same(d, expect(c, kn.cpu(), vn.cpu(), off.cpu()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(4):
        d["len"] += off.diff()
        kn.copy_(draw.normal(50 + step, "kn", 5, 2, D, std=3.0 ** step))
        vn.copy_(draw.normal(50 + step, "vn", 5, 2, D, std=2.0 ** step))
        torch.cuda.synchronize()
        c = {x: t.cpu() for x, t in d.items()}
        g.replay()
        torch.cuda.synchronize()
        same(d, expect(c, kn.cpu(), vn.cpu(), off.cpu()))
