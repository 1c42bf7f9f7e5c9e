"""The attention of draft tokens over a latent cache and over the 8-bit cache, and of prompts, against the definitions in
64 bits: caches of no token, one, less and more than a tile and a page; pages that end inside a tile; odd head counts;
trees, chains, drafts that see nothing and sequences without drafts; NaN in everything that is not attended to."""
import math

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
R, P = 512, 64
NAN = float("nan")


def dev(*ts):
    return [t if t is None else t.to(DEV) for t in ts]


def visible(mask, n):
    return [j for j in range(n) if (int(mask) >> j) & 1]


def compare(rows, o, lse):
    """rows: (t, h, Attended, keys) of the query rows to check."""
    o, lse = o.cpu().double().numpy(), lse.cpu().double().numpy()
    for t, h, a, n in rows:
        tol, tol_lse = ref.tolerances(a, n)
        assert np.all(np.abs(o[t, h] - a.o) <= tol), (t, h, n, np.abs(o[t, h] - a.o).max(), tol.min())
        if math.isinf(a.lse):
            assert lse[t, h] == -math.inf, (t, h)
        else:
            assert abs(lse[t, h] - a.lse) <= tol_lse, (t, h, n, lse[t, h], a.lse)


def batch(counts, lens, page, seed, masks):
    off = draw.offsets(counts)
    N = sum(counts)
    mask = {"tree": lambda: draw.tree_masks(counts, seed), "causal": lambda: None}[masks]()
    bits = mask.tolist() if mask is not None else [(1 << i + 1) - 1 for n in counts for i in range(n)]
    table, pages = draw.page_table(lens, page, seed)
    return off, N, mask, bits, table, pages


def some_rows(counts, H, rng, most=40):
    """(b, t, i, h): all rows of a small call, a spread of a large one."""
    off = np.cumsum([0, *counts])
    rows = [(b, int(off[b]) + i, i, h) for b, n in enumerate(counts) for i in range(n) for h in range(H)]
    return rows if len(rows) <= most else [rows[int(i)] for i in sorted(rng.choice(len(rows), most, replace=False))] + [rows[-1]]


# ----------------------------------------------------------------------------- latent, absorbed

def latent_case(counts, lens, H, page, seed=0, masks="tree", std=0.8, poison=False):
    off, N, mask, bits, table, pages = batch(counts, lens, page, seed, masks)
    q, new = draw.normal(seed, "q", N, H, R + P, std=std), draw.normal(seed, "new", N, R + P)
    store = draw.normal(seed, "pages", pages, page, R + P)
    if poison:  # everything past a sequence's tokens
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for i in range(n):
                used[int(table[b, i // page]), i % page] = True
        store[~used] = NAN
    return dict(off=off, N=N, mask=mask, bits=bits, table=table, q=q, new=new, store=store, counts=counts, lens=lens, H=H,
                page=page, scale=1 / math.sqrt(192))


def latent_run(c, **more):
    ln = torch.tensor(c["lens"], dtype=torch.int32)
    q, new, off, store, table, ln, mask = dev(c["q"], c["new"], c["off"], c["store"], c["table"], ln, c["mask"])
    return moe.moe_latent_attn(q, new, off, store, table, ln, R, c["scale"], mask=mask, **more)


def latent_rows(c, rows):
    off = c["off"].tolist()
    for b, t, i, h in rows:
        n, m = c["lens"][b], c["counts"][b]
        flat = c["store"][c["table"][b].long()].reshape(-1, R + P)[:n]
        see = [off[b] + j for j in visible(c["bits"][t], m)]
        keys = torch.cat([flat, c["new"][see]]).double().numpy()
        yield t, h, ref.attend(c["q"][t, h].double().numpy(), keys, keys[:, :R], c["scale"]), len(keys)


LATENT = [  # drafts of each sequence, cached tokens, heads, page
    ([1], [0], 1, 16), ([1], [1], 16, 16), ([4], [63], 16, 64), ([4], [64], 128, 64), ([1], [65], 128, 16),
    ([3], [700], 5, 32), ([1, 1, 1], [17, 0, 300], 20, 16), ([2, 0, 5], [33, 50, 129], 8, 128), ([64], [100], 3, 64),
    ([17, 40], [1000, 31], 16, 32), ([4], [9000], 128, 64), ([1] * 9, [900 + 37 * i for i in range(9)], 128, 64),
    ([8, 1, 30], [2500, 5, 640], 64, 64),
]


@pytest.mark.parametrize("counts,lens,H,page", LATENT)
@pytest.mark.parametrize("masks", ["tree", "causal"])
def test_latent(counts, lens, H, page, masks):
    print(f"latent counts={counts} lens={lens} H={H} page={page} {masks}", flush=True)
    c = latent_case(counts, lens, H, page, seed=len(counts) + H, masks=masks, poison=True)
    o, lse = latent_run(c)
    rng = np.random.default_rng(1)
    compare(latent_rows(c, some_rows(counts, H, rng)), o, lse)
    again = latent_run(c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_latent_peaked_scores():
    """Scores in the hundreds: one key takes nearly all the weight, and the running maximum moves late."""
    c = latent_case([3, 2], [333, 1500], 16, 64, seed=3, std=12.0)
    c["store"] = c["store"].clone()
    compare(latent_rows(c, some_rows([3, 2], 16, np.random.default_rng(0))), *latent_run(c))


def test_latent_rows_that_see_nothing_and_stray_bits():
    c = latent_case([5, 3], [0, 40], 16, 16, seed=4)
    m = c["mask"].tolist()
    m[2] = 0          # no cache, no draft
    m[3] |= 1 << 40   # a bit past the sequence's drafts
    m[6] = -(1 << 63)  # only stray bits: the cache alone
    c["mask"], c["bits"] = torch.tensor(m, dtype=torch.int64), m
    o, lse = latent_run(c)
    assert torch.all(o[2] == 0) and torch.all(lse[2] == -math.inf)
    compare(latent_rows(c, [(b, t, i, h) for b, t, i in ((0, 2, 2), (0, 3, 3), (1, 6, 1), (1, 7, 2)) for h in range(16)]), o, lse)


@pytest.mark.parametrize("bad", [NAN, math.inf])
def test_latent_masked_draft_is_not_felt(bad):
    """A draft with a non-finite row, seen by some and not by others."""
    c = latent_case([6, 2], [70, 9], 16, 16, seed=5)
    m = [0b1, 0b11, 0b101, 0b1001, 0b11011, 0b100101, 0b1, 0b11]
    c["mask"], c["bits"] = torch.tensor(m, dtype=torch.int64), m
    c["new"][1, ::3] = bad  # seen by rows 1 and 4
    o, lse = latent_run(c)
    compare(latent_rows(c, [(0, t, t, h) for t in (0, 2, 3, 5) for h in (0, 7, 15)] + [(1, 6, 0, 3), (1, 7, 1, 15)]), o, lse)
    assert torch.isnan(o[[1, 4]].float()).any(-1).all()


def test_latent_long_cache_past_32_bit_offsets():
    """Pages past 4 GiB: two sequences whose pages sit at the end of a 5 GiB cache."""
    page, pages = 128, 36000
    store = torch.zeros(pages, page, R + P, dtype=torch.bfloat16, device=DEV)
    lens, counts, H = [300, 129], [2, 1], 16
    table = torch.tensor([[35990, 35999, 35991], [35995, 35992, 0]], dtype=torch.int32)
    c = latent_case(counts, lens, H, page, seed=6)
    small = c["store"]
    for b in range(2):
        for i in range(3):
            store[int(table[b, i])] = small[int(c["table"][b, min(i, c["table"].shape[1] - 1)])].to(DEV)
    q, new, off, mask = dev(c["q"], c["new"], c["off"], c["mask"])
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = moe.moe_latent_attn(q, new, off, store, table.to(DEV), ln, R, c["scale"], mask=mask)
    compare(latent_rows(c, some_rows(counts, H, np.random.default_rng(0))), o, lse)


# ----------------------------------------------------------------------------- 8-bit cache

def cache_case(counts, lens, H, Hkv, D, page, seed=0, masks="tree", poison=False):
    off, N, mask, bits, table, pages = batch(counts, lens, page, seed, masks)
    c = dict(off=off, N=N, mask=mask, bits=bits, table=table, counts=counts, lens=lens, H=H, Hkv=Hkv, D=D, page=page,
             scale=1 / math.sqrt(D), q=draw.normal(seed, "q", N, H, D), kn=draw.normal(seed, "kn", N, Hkv, D),
             vn=draw.normal(seed, "vn", N, Hkv, D), k=draw.codes(seed, "k", pages, Hkv, page, D),
             v=draw.codes(seed, "v", pages, Hkv, D, page), ks=draw.power_scales(seed, "ks", pages, Hkv),
             vs=draw.power_scales(seed, "vs", pages, Hkv))
    if poison:
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for i in range(n):
                used[int(table[b, i // page]), i % page] = True
        c["k"][(~used)[:, None, :, None].expand_as(c["k"])] = 0x7F
        c["v"][(~used)[:, None, None, :].expand_as(c["v"])] = 0xFF
        idle = ~used.any(1)
        c["ks"][idle] = NAN
        c["vs"][idle] = math.inf
    return c


def cache_run(c, **more):
    ln = torch.tensor(c["lens"], dtype=torch.int32)
    q, kn, vn, off, k, v, ks, vs, table, ln, mask = dev(*(c[x] for x in ("q", "kn", "vn", "off", "k", "v", "ks", "vs", "table")), ln, c["mask"])
    return moe.moe_cache_attn(q, kn, vn, off, k, v, ks, vs, table, ln, c["scale"], mask=mask, **more)


def cache_rows(c, rows):
    off, G = c["off"].tolist(), c["H"] // c["Hkv"]
    for b, t, i, h in rows:
        n, m, g = c["lens"][b], c["counts"][b], h // G
        ids = c["table"][b].long()
        k = ref.E4M3[c["k"][ids, g].numpy()] * c["ks"][ids, g].double().numpy()[:, None, None]
        v = ref.E4M3[c["v"][ids, g].numpy()] * c["vs"][ids, g].double().numpy()[:, None, None]
        k, v = k.reshape(-1, c["D"])[:n], v.transpose(0, 2, 1).reshape(-1, c["D"])[:n]
        see = [off[b] + j for j in visible(c["bits"][t], m)]
        k, v = np.concatenate([k, c["kn"][see, g].double().numpy()]), np.concatenate([v, c["vn"][see, g].double().numpy()])
        yield t, h, ref.attend(c["q"][t, h].double().numpy(), k, v, c["scale"]), len(k)


CACHE = [  # drafts of each sequence, cached tokens, heads, key/value heads, width, page
    ([1], [0], 1, 1, 64, 16), ([1], [1], 8, 8, 128, 16), ([4], [63], 64, 4, 128, 64), ([4], [64], 64, 8, 64, 64),
    ([1], [65], 16, 1, 128, 32), ([3], [700], 10, 2, 64, 32), ([1, 1, 1], [17, 0, 300], 40, 8, 64, 16),
    ([2, 0, 5], [33, 50, 129], 12, 4, 128, 128), ([64], [100], 6, 2, 128, 64), ([17, 40], [1000, 31], 64, 8, 64, 32),
    ([4], [9000], 64, 4, 128, 64), ([1] * 9, [900 + 37 * i for i in range(9)], 64, 8, 64, 16),
    ([8, 1, 30], [2500, 5, 640], 32, 2, 128, 128), ([64, 3], [513, 255], 16, 1, 64, 128),
]


@pytest.mark.parametrize("counts,lens,H,Hkv,D,page", CACHE)
@pytest.mark.parametrize("masks", ["tree", "causal"])
def test_cache(counts, lens, H, Hkv, D, page, masks):
    print(f"cache counts={counts} lens={lens} H={H} Hkv={Hkv} D={D} page={page} {masks}", flush=True)
    c = cache_case(counts, lens, H, Hkv, D, page, seed=len(counts) + H, masks=masks, poison=True)
    o, lse = cache_run(c)
    compare(cache_rows(c, some_rows(counts, H, np.random.default_rng(1))), o, lse)
    again = cache_run(c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_cache_rows_that_see_nothing_and_stray_bits():
    c = cache_case([5, 3], [0, 40], 16, 2, 64, 16, seed=4)
    m = c["mask"].tolist()
    m[2] = 0
    m[3] |= 1 << 40
    m[6] = -(1 << 63)
    c["mask"], c["bits"] = torch.tensor(m, dtype=torch.int64), m
    o, lse = cache_run(c)
    assert torch.all(o[2] == 0) and torch.all(lse[2] == -math.inf)
    compare(cache_rows(c, [(b, t, i, h) for b, t, i in ((0, 2, 2), (0, 3, 3), (1, 6, 1), (1, 7, 2)) for h in range(16)]), o, lse)


@pytest.mark.parametrize("bad", [NAN, math.inf])
def test_cache_masked_draft_is_not_felt(bad):
    c = cache_case([6, 2], [70, 9], 16, 2, 128, 16, seed=5)
    m = [0b1, 0b11, 0b101, 0b1001, 0b11011, 0b100101, 0b1, 0b11]
    c["mask"], c["bits"] = torch.tensor(m, dtype=torch.int64), m
    c["kn"][1, :, ::3] = bad
    c["vn"][1, :, ::3] = bad
    o, lse = cache_run(c)
    compare(cache_rows(c, [(0, t, t, h) for t in (0, 2, 3, 5) for h in (0, 7, 15)] + [(1, 6, 0, 3), (1, 7, 1, 15)]), o, lse)
    assert torch.isnan(o[[1, 4]].float()).any(-1).all()


def test_cache_past_32_bit_offsets():
    """A 5 GiB key cache whose last pages are the ones read."""
    page, pages, Hkv, D, H = 128, 42000, 8, 128, 16
    lens, counts = [300, 129], [2, 1]
    c = cache_case(counts, lens, H, Hkv, D, page, seed=6)
    table = torch.tensor([[41990, 41999, 41991], [41995, 41992, 0]], dtype=torch.int32)
    big = {x: torch.zeros(pages, *c[x].shape[1:], dtype=c[x].dtype, device=DEV) for x in ("k", "v", "ks", "vs")}
    for b in range(2):
        for i in range(3):
            src = int(c["table"][b, min(i, c["table"].shape[1] - 1)])
            for x in big:
                big[x][int(table[b, i])] = c[x][src].to(DEV)
    q, kn, vn, off, mask = dev(c["q"], c["kn"], c["vn"], c["off"], c["mask"])
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = moe.moe_cache_attn(q, kn, vn, off, big["k"], big["v"], big["ks"], big["vs"], table.to(DEV), ln, c["scale"], mask=mask)
    compare(cache_rows(c, some_rows(counts, H, np.random.default_rng(0))), o, lse)


# ----------------------------------------------------------------------------- latent, expanded

def prompt_case(nq, nk, H, seed=0, apart=False):
    N, M = sum(nq), sum(nk)
    kv = draw.normal(seed, "kv", M, H, 256 + (8 if apart else 0))
    return dict(nq=nq, nk=nk, H=H, qo=draw.offsets(nq), ko=draw.offsets(nk), q=draw.normal(seed, "q", N, H, 192, std=1.5), kv=kv,
                rope=draw.normal(seed, "rope", M, 64), scale=1 / math.sqrt(192))


def prompt_run(c, **more):
    q, kv, rope, qo, ko = dev(c["q"], c["kv"], c["rope"], c["qo"], c["ko"])
    return moe.moe_latent_prompt(q, kv[..., :128], rope, kv[..., -128:], qo, ko, c["scale"], **more)


def prompt_rows(c, rows):
    qo, ko = c["qo"].tolist(), c["ko"].tolist()
    for b, t, i, h in rows:
        n = max(0, min(c["nk"][b], i + 1 + c["nk"][b] - c["nq"][b]))
        k = torch.cat([c["kv"][ko[b]:ko[b] + n, h, :128], c["rope"][ko[b]:ko[b] + n]], 1).double().numpy()
        v = c["kv"][ko[b]:ko[b] + n, h, -128:].double().numpy()
        yield t, h, ref.attend(c["q"][t, h].double().numpy(), k, v, c["scale"]), n


PROMPT = [  # queries of each sequence, keys, heads
    ([1], [1], 1), ([1], [200], 3), ([17], [17], 2), ([64], [64], 1), ([65], [65], 5), ([130], [130], 16), ([256], [256], 2),
    ([257], [400], 2), ([5, 0, 33], [5, 7, 90], 4), ([100, 1, 300], [100, 70, 300], 8), ([1500], [1500], 4),
    ([40], [10], 2), ([3, 1], [0, 1], 2), ([70, 900], [2000, 901], 3),
]


@pytest.mark.parametrize("nq,nk,H", PROMPT)
def test_prompt(nq, nk, H):
    print(f"prompt nq={nq} nk={nk} H={H}", flush=True)
    c = prompt_case(nq, nk, H, seed=H + len(nq), apart=H % 2 == 1)
    o, lse = prompt_run(c, max_tokens=max(nq))
    compare(prompt_rows(c, some_rows(nq, H, np.random.default_rng(2), most=60)), o, lse)
    again = prompt_run(c)  # the grid sized by all tokens
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("bad", [NAN, math.inf])
def test_prompt_later_keys_are_not_felt(bad):
    """Non-finite keys and values: only the queries at or past them have them."""
    c = prompt_case([90, 20], [90, 20], 2, seed=9)
    c["kv"][41, :, ::5] = bad
    c["rope"][41, 3] = bad
    o, lse = prompt_run(c)
    rows = [(0, t, t, h) for t in (0, 1, 15, 31, 32, 40) for h in range(2)] + [(1, 90 + t, t, h) for t in (0, 19) for h in range(2)]
    compare(prompt_rows(c, rows), o, lse)
    assert torch.isnan(o[41:90].float()).any(-1).all()


def test_other_stream_and_graph():
    """The three calls on a stream of their own, then captured once and replayed on other inputs."""
    lc = latent_case([4, 2], [500, 90], 16, 64, seed=11)
    cc = cache_case([4, 2], [500, 90], 16, 4, 64, 64, seed=11)
    pc = prompt_case([70], [100], 4, seed=11)
    want = latent_run(lc), cache_run(cc), prompt_run(pc)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = latent_run(lc), cache_run(cc), prompt_run(pc)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])

    ln = torch.tensor(lc["lens"], dtype=torch.int32)
    q, new, off, store, table, ln, mask = dev(lc["q"], lc["new"], lc["off"], lc["store"], lc["table"], ln, lc["mask"])
    ws = torch.empty(moe.moe_latent_attn_workspace_size(store, table, ln, R, lc["N"], 16), dtype=torch.uint8, device=DEV)
    o, lse = torch.empty(lc["N"], 16, R, dtype=torch.bfloat16, device=DEV), torch.empty(lc["N"], 16, device=DEV)

    def call():
        moe.moe_latent_attn(q, new, off, store, table, ln, R, lc["scale"], mask=mask, o=o, lse=lse, workspace=ws)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step, n in enumerate((500, 333, 64, 0)):
        ln[0] = n  # the cache's length is read on the device
        q.copy_(draw.normal(20 + step, "q", *q.shape, std=0.8))
        g.replay()
        torch.cuda.synchronize()
        lc["lens"][0], lc["q"] = n, q.cpu()
        got = o.clone(), lse.clone()
        call()
        assert torch.equal(o, got[0]) and torch.equal(lse, got[1])
        compare(latent_rows(lc, some_rows([4, 2], 16, np.random.default_rng(step), most=12)), *got)


# ----------------------------------------------------------------------------- each variant and plan

@pytest.mark.parametrize("scale", [-0.07, 0.0])
def test_scales_that_are_not_positive(scale):
    for c, run, rows, n, H in ((latent_case([3, 1], [90, 33], 8, 16, seed=21), latent_run, latent_rows, [3, 1], 8),
                               (cache_case([3, 1], [90, 33], 8, 2, 64, 16, seed=22), cache_run, cache_rows, [3, 1], 8),
                               (prompt_case([60, 9], [70, 9], 2, seed=23), prompt_run, prompt_rows, [60, 9], 2)):
        c["scale"] = scale
        compare(rows(c, some_rows(n, H, np.random.default_rng(4))), *run(c))


@pytest.mark.parametrize("counts,lens,H", [([3, 4, 2], [70, 300, 1025], 16), ([1, 2], [640, 31], 40), ([4] * 5, [2000, 0, 7, 96, 129], 12)])
def test_latent_of_two_row_tiles(counts, lens, H):
    """33 to 64 rows a sequence on average."""
    assert 32 * len(counts) < sum(counts) * H <= 64 * len(counts)
    c = latent_case(counts, lens, H, 32, seed=24, poison=True)
    compare(latent_rows(c, some_rows(counts, H, np.random.default_rng(5), most=80)), *latent_run(c))


def test_more_sequences_than_lanes():
    """150 sequences, some without drafts, some without a cache."""
    rng = np.random.default_rng(6)
    counts = [int(n) for n in rng.integers(0, 4, 150)]
    lens = [int(n) for n in rng.integers(0, 400, 150)]
    c = latent_case(counts, lens, 8, 16, seed=25, poison=True)
    compare(latent_rows(c, some_rows(counts, 8, rng)), *latent_run(c))
    c = cache_case(counts, lens, 8, 2, 64, 16, seed=26, poison=True)
    compare(cache_rows(c, some_rows(counts, 8, rng)), *cache_run(c))
    c = prompt_case(counts, [n + m for n, m in zip(counts, lens)], 2, seed=27)
    compare(prompt_rows(c, some_rows(counts, 2, rng)), *prompt_run(c, max_tokens=3))


@pytest.mark.parametrize("B", [700, 1024])
def test_many_row_groups(B):
    """More row groups than run at once, cut (700) and whole (1024 latent, 4 x 1024 of four key/value heads)."""
    rng = np.random.default_rng(7)
    lens = [int(n) for n in rng.integers(0, 90, B)]
    c = latent_case([1] * B, lens, 16, 16, seed=28, poison=True)
    compare(latent_rows(c, some_rows([1] * B, 16, rng)), *latent_run(c))
    c = cache_case([1] * B, lens, 8, 4, 128, 16, seed=29, poison=True)
    compare(cache_rows(c, some_rows([1] * B, 8, rng)), *cache_run(c))


def test_latent_chunks_in_two_rounds():
    """178 row groups of 140 and 70 tiles: at once they would be 256 chunks of 140 tiles or fewer, in two rounds 484 of 47."""
    counts, lens = [64, 64, 50], [4400, 4390, 2170]
    c = latent_case(counts, lens, 128, 64, seed=34, poison=True)
    o, lse = latent_run(c)
    compare(latent_rows(c, some_rows(counts, 128, np.random.default_rng(10), most=24)), o, lse)
    again = latent_run(c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
def test_cache_scales_of_any_value(D, page):
    """Page scales that are no powers of two, over 12 orders of magnitude within a sequence."""
    counts, lens = [3, 2], [777, 40]
    c = cache_case(counts, lens, 16, 4, D, page, seed=30, poison=True)
    rng = np.random.default_rng(8)
    for x in ("ks", "vs"):
        used = torch.isfinite(c[x])
        c[x][used] = torch.from_numpy((0.004 * rng.lognormal(0.0, 0.8, c[x].shape)).astype(np.float32))[used]
    c["vs"][int(c["table"][0, 1])] = 3e-14
    compare(cache_rows(c, some_rows(counts, 16, rng)), *cache_run(c))


def test_prompt_of_separate_strided_tensors():
    c = prompt_case([140, 3], [150, 40], 3, seed=31)
    k = draw.normal(31, "k", 190, 3, 144)[..., :128]  # rows of 3 * 144
    v = draw.normal(31, "v", 3, 190, 136).transpose(0, 1)[..., :128]  # heads apart
    c["kv"] = torch.cat([k, v], 2)
    q, rope, qo, ko = dev(c["q"], c["rope"], c["qo"], c["ko"])
    kd = torch.empty(190, 3, 144, dtype=torch.bfloat16, device=DEV)[..., :128]
    vd = torch.empty(3, 190, 136, dtype=torch.bfloat16, device=DEV).transpose(0, 1)[..., :128]
    kd.copy_(k)
    vd.copy_(v)
    o, lse = moe.moe_latent_prompt(q, kd, rope, vd, qo, ko, c["scale"])
    compare(prompt_rows(c, some_rows([140, 3], 3, np.random.default_rng(9), most=80)), o, lse)


def test_given_outputs_and_no_log_sums():
    """Outputs in the caller's buffers, nothing past them written; and a null lse through the C interface."""
    import ctypes as C
    c = cache_case([3, 2], [50, 700], 16, 4, 64, 16, seed=32)
    want, _ = cache_run(c)
    room = torch.full((7, 16, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((7, 16), 5.0, device=DEV)
    cache_run(c, o=room[:5], lse=lse[:5])
    assert torch.equal(room[:5], want) and torch.all(room[5:] == 5) and torch.all(lse[5:] == 5)

    p = prompt_case([40], [40], 2, seed=33)
    q, kv, rope, qo, ko = dev(p["q"], p["kv"], p["rope"], p["qo"], p["ko"])
    want, _ = moe.moe_latent_prompt(q, kv[..., :128], rope, kv[..., 128:], qo, ko, p["scale"])
    o = torch.empty_like(want)
    a = moe.moe_prompt_t(40, 40, 1, 2, 128, 64, 128, 40, qo.data_ptr(), ko.data_ptr(), q.data_ptr(), kv.data_ptr(), rope.data_ptr(),
                         kv.data_ptr() + 256, 512, 256, 512, 256, p["scale"])
    assert moe.lib().moe_latent_prompt(C.byref(a), o.data_ptr(), None, torch.cuda.current_stream().cuda_stream) == moe.MOE_OK
    assert torch.equal(o, want)
