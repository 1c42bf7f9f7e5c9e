"""Attention of whole prompts with grouped heads against the definition in 64 bits: lengths from one token on, around every tile
and row block, behind keys of their own or with fewer keys than queries; groups of every size; strided parts of a projection; NaN
in everything that is not attended to; infinities and NaN that some rows see and others do not."""
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
NAN, INF = math.nan, math.inf


def case(nq, nk, H, Hkv, D, seed=0, spare=5, std=1.3, scale=None):
    """Packed inputs, `spare` rows of NaN keys, values and queries behind the last sequence's."""
    N, M = sum(nq), sum(nk)
    q = draw.normal(seed, "q", max(N, 1) + spare, H, D, std=std)
    kv = draw.normal(seed, "kv", max(M, 1) + spare, 2, Hkv, D)
    q[N:], kv[M:] = NAN, NAN
    return dict(nq=nq, nk=nk, H=H, Hkv=Hkv, D=D, q=q, k=kv[:, 0], v=kv[:, 1], kv=kv, qo=draw.offsets(nq), ko=draw.offsets(nk),
                scale=1 / math.sqrt(D) if scale is None else scale)


def run(c, **more):
    kv = c["kv"].to(DEV)
    return moe.moe_grouped_prompt(c["q"].to(DEV), kv[:, 0], kv[:, 1], c["qo"].to(DEV), c["ko"].to(DEV), c["scale"],
                                  **{"max_tokens": max(max(c["nq"]), 1), **more})


def some_rows(c, rng, most=40):
    """(b, query, head): all of a small call, else a spread with the first and last of each sequence."""
    rows = [(b, i, h) for b, n in enumerate(c["nq"]) for i in range(n) for h in range(c["H"])]
    if len(rows) <= most:
        return rows
    ends = [(b, i, c["H"] - 1 - b % c["H"]) for b, n in list(enumerate(c["nq"]))[:6] if n for i in (0, n - 1)]
    return [rows[int(i)] for i in rng.choice(len(rows), most, replace=False)] + ends


def check(c, o, lse, rows):
    o, lse = o.cpu().double().numpy(), lse.cpu().double().numpy()
    q, k, v = (c[x].double().numpy() for x in "qkv")
    qo, ko, G = c["qo"].tolist(), c["ko"].tolist(), c["H"] // c["Hkv"]
    for b, i, h in rows:
        n = min(max(i + 1 + c["nk"][b] - c["nq"][b], 0), c["nk"][b])
        with np.errstate(invalid="ignore"):
            a = ref.attend(q[qo[b] + i, h], k[ko[b]:ko[b] + n, h // G], v[ko[b]:ko[b] + n, h // G], c["scale"])
            got, want = o[qo[b] + i, h], a.o
            tol, tol_lse = ref.tolerances(a, n)
            fin = np.isfinite(want)
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (b, i, h)
            assert np.all(np.abs(got - want)[fin] <= tol[fin]), (b, i, h, n, np.abs(got - want)[fin].max(), tol[fin].min())
        if not math.isfinite(a.lse):
            assert lse[qo[b] + i, h] == a.lse or math.isnan(a.lse) and math.isnan(lse[qo[b] + i, h]), (b, i, h)
        else:
            assert abs(lse[qo[b] + i, h] - a.lse) <= tol_lse, (b, i, h, n, lse[qo[b] + i, h], a.lse)


LENGTHS = [  # queries, keys
    ([1], [1]), ([2], [2]), ([31], [31]), ([33], [64]), ([64, 65], [64, 97]), ([127, 1, 129], [127, 700, 129]), ([0, 5, 0, 40], [9, 5, 0, 47]),
    ([257, 256], [257, 513]), ([7], [4001]), ([1] * 9, [1 + 50 * i for i in range(9)]), ([30, 8], [20, 0]), ([600], [611]), ([1], [3000]),
]
HEADS = [(1, 1), (4, 1), (5, 5), (12, 4), (10, 2), (64, 4), (33, 1)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
def test_lengths(H, Hkv, D):
    rng = np.random.default_rng(H)
    for n, (nq, nk) in enumerate(LENGTHS):
        print(f"grouped prompt H={H}/{Hkv} D={D} queries={nq} keys={nk}", flush=True)
        c = case(nq, nk, H, Hkv, D, seed=n)
        o, lse = run(c)
        check(c, o, lse, some_rows(c, rng, most=24))
        again = run(c)
        N = sum(nq)
        assert torch.equal(o[:N], again[0][:N]) and torch.equal(lse[:N], again[1][:N])


@pytest.mark.parametrize("nq,nk,H,Hkv,D", [([2500], [2500], 8, 2, 128), ([1900, 3], [2111, 1500], 16, 2, 64), ([100], [30000], 16, 1, 128),
                                           ([5], [70000], 8, 8, 64), ([2], [60000], 4, 1, 128),
                                           ([40, 2, 17], [9000, 11, 20000], 20, 4, 128), ([600], [20600], 64, 8, 64),
                                           ([300], [20301], 64, 4, 128)])
def test_long(nq, nk, H, Hkv, D):
    c = case(nq, nk, H, Hkv, D, seed=3)
    check(c, *run(c), some_rows(c, np.random.default_rng(2), most=60))


@pytest.mark.parametrize("D", [64, 128])
def test_many_sequences(D):
    rng = np.random.default_rng(D)
    for B, top in ((300, 40), (1024, 3)):
        nq = [int(n) for n in rng.integers(0, top, B)]
        nk = [n + int(rng.integers(0, 60)) for n in nq]
        c = case(nq, nk, 8, 2, D, seed=B)
        check(c, *run(c), some_rows(c, rng, most=60))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,Hkv", [(5, 16, 2), (64, 2, 1), (65, 2, 2), (100, 1, 1), (300, 4, 2)])
def test_few_long_ones_among_short(B, H, Hkv, D):
    """Sequences of a few queries, of which some have long keys behind, some nothing: cut by what the device finds."""
    rng = np.random.default_rng(B)
    nq = [int(n) for n in rng.integers(0, 4, B)]
    nk = [n + int(rng.choice([0, rng.integers(0, 300), 6000 if rng.random() < 0.3 else 900])) for n in nq]
    nq[0], nk[0], nk[B // 2], nk[-1] = 40, 9041, 0, nq[-1] + 7777
    c = case(nq, nk, H, Hkv, D, seed=B)
    o, lse = run(c)
    last = [(b, n - 1, H - 1) for b, n in enumerate(nq) if n][-30:]
    check(c, o, lse, some_rows(c, rng, most=60) + last)
    again, N = run(c), sum(nq)  # rows behind are left as they were
    assert torch.equal(o[:N], again[0][:N]) and torch.equal(lse[:N], again[1][:N])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", ["peaked", "large", "zero", "negative", "tiny"])
def test_scores(what, D):
    """Scores that a few keys win, that are far from zero and grow along the keys, and scales that are not positive."""
    c = case([150, 70], [400, 70], 6, 2, D, seed=5, scale={"zero": 0.0, "negative": -0.1, "tiny": 1e-30}.get(what))
    if what == "peaked":
        c["k"][::13] *= 12
    if what == "large":
        c["k"] += torch.linspace(-3, 3, len(c["k"]))[:, None, None].to(torch.bfloat16)
        c["q"][:, 3] += 8
    c["kv"] = torch.stack([c["k"], c["v"]], 1)
    check(c, *run(c), some_rows(c, np.random.default_rng(1), most=80))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_later_keys_are_not_felt(bad, D):
    """A key, and a value, of `bad` late in the sequence: rows before them are as without, rows that see a bad value get it."""
    for H, Hkv, n, at in ((4, 1, 300, 290), (8, 8, 200, 130), (32, 2, 90, 64)):
        c = case([n], [n], H, Hkv, D, seed=7)
        clean, clean_lse = run(c)
        c["v"][at, :, 1::3] = bad
        c["v"][at + 3, 0, 1] = -bad
        c["kv"][:, 1] = c["v"]
        o, lse = run(c)
        assert torch.equal(o[:at], clean[:at]) and torch.equal(lse[:n], clean_lse[:n])
        check(c, o, lse, [(0, i, h) for i in (at - 1, at, at + 2, at + 3, n - 1) for h in (0, H - 1)])
        c["k"][at + 5:] = NAN
        c["kv"][:, 0] = c["k"]
        o, lse = run(c)
        rows = [(0, i, h) for i in (0, at - 1, at, at + 4) for h in range(H)]
        check(c, o, lse, rows)
        assert torch.isnan(o[at + 5:n]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [1, 40])
def test_bad_values_in_every_tile(B, D):
    """One value that is not a number, in each tile in turn, in cut and in whole row blocks: rows that do not see it are as without."""
    n, H = 299, 8
    c = case([n] * B, [n] * B, H, H, D, seed=12, spare=0)
    clean, clean_lse = run(c)
    kv = c["kv"].to(DEV)
    for at in range(5, n, 32):
        print(f"grouped prompt bad value B={B} D={D} key={at}", flush=True)
        for b in (0, B - 1):
            i = n * b + at
            was = kv[i, 1].clone()
            kv[i, 1, :, 7::19] = NAN
            o, lse = moe.moe_grouped_prompt(c["q"].to(DEV), kv[:, 0], kv[:, 1], c["qo"].to(DEV), c["ko"].to(DEV), c["scale"], max_tokens=n)
            felt = torch.isnan(o)
            assert torch.equal(lse, clean_lse) and felt[i:n * (b + 1), :, 7::19].all()
            felt[i:n * (b + 1), :, 7::19] = False
            assert not felt.any()
            o[i:n * (b + 1), :, 7::19] = clean[i:n * (b + 1), :, 7::19]
            assert torch.equal(o, clean)
            kv[i, 1] = was


def test_values_that_all_see():
    """Infinities before every query's first key: they reach every row."""
    c = case([40], [400], 4, 2, 64, seed=8)
    c["v"][17, 0, 5] = INF
    c["v"][18, 1, 6] = NAN
    c["kv"][:, 1] = c["v"]
    o, lse = run(c)
    check(c, o, lse, some_rows(c, np.random.default_rng(0)))
    assert torch.isinf(o[:40, :2, 5]).all() and torch.isnan(o[:40, 2:, 6]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_strided_parts_and_rows_behind(D):
    """Queries, keys and values as they lie in one projection; given outputs, whose rows behind the last query stay."""
    nq, H, Hkv, spare = [70, 3, 131], 12, 3, 9
    N = sum(nq)
    x = draw.normal(4, "qkv", N + spare, H + 2 * Hkv, D).to(DEV)
    x[N:] = NAN
    q, k, v = x.split([H, Hkv, Hkv], 1)
    off = draw.offsets(nq).to(DEV)
    o = torch.full((N + spare, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((N + spare, H), 7.0, device=DEV)
    moe.moe_grouped_prompt(q, k, v, off, off, 0.1, max_tokens=131, o=o, lse=lse)
    assert (o[N:] == 7).all() and (lse[N:] == 7).all()
    c = dict(nq=nq, nk=nq, H=H, Hkv=Hkv, D=D, q=q.cpu(), k=k.cpu(), v=v.cpu(), qo=off.cpu(), ko=off.cpu(), scale=0.1)
    check(c, o, lse, some_rows(c, np.random.default_rng(0), most=80))
    # Heads apart, one head's keys for all: a stride of zero.
    k1, v1 = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (k, v))
    again = moe.moe_grouped_prompt(q.contiguous(), k1, v1, off, off, 0.1)
    assert torch.equal(again[0][:N], o[:N])
    shared = moe.moe_grouped_prompt(q, k[:, :1].expand(-1, Hkv, -1), v[:, :1].expand(-1, Hkv, -1), off, off, 0.1)
    single = moe.moe_grouped_prompt(q, k[:, :1], v[:, :1], off, off, 0.1)
    c.update(Hkv=1)
    check(c, *single, some_rows(c, np.random.default_rng(0), most=40))
    check(c, *shared, some_rows(c, np.random.default_rng(0), most=40))


def test_past_32_bit_offsets():
    """Keys that end past 4 GiB, queries past 2^31 elements."""
    M, Hkv, D = 70000, 4, 128
    kv = torch.zeros(M, 70, Hkv, D, dtype=torch.bfloat16, device=DEV)  # 5 GB; the 70 layers of a cache side by side
    c = case([9], [400], 16, Hkv, D, seed=9, spare=0)
    kv[M - 400:, 68], kv[M - 400:, 69] = c["k"].to(DEV), c["v"].to(DEV)
    ko = torch.tensor([0, M - 400, M], dtype=torch.int32, device=DEV)
    qo = torch.tensor([0, 0, 9], dtype=torch.int32, device=DEV)
    o, lse = moe.moe_grouped_prompt(c["q"].to(DEV), kv[:, 68], kv[:, 69], qo, ko, c["scale"])
    check(c, o, lse, some_rows(c, np.random.default_rng(0), most=60))
    del kv
    q = torch.zeros(9, 1 << 28, dtype=torch.bfloat16, device=DEV)  # a query every 512 MB
    for h in range(16):
        q[:, h * 1024:h * 1024 + D] = c["q"][:, h].to(DEV)
    view = q.as_strided((9, 16, D), (1 << 28, 1024, 1))
    again = moe.moe_grouped_prompt(view, c["k"].to(DEV), c["v"].to(DEV), draw.offsets([9]).to(DEV), draw.offsets([400]).to(DEV), c["scale"])
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("nq,nk", [([200, 30], [260, 30]), ([6, 1], [2500, 40])])
def test_stream_and_graph(nq, nk):
    """Another stream than the current one; a captured call replayed on other lengths and inputs."""
    c = case(nq, nk, 12, 4, 128, seed=11, spare=0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out = run(c)
    side.synchronize()
    rng = np.random.default_rng(0)
    check(c, *out, some_rows(c, rng))
    q, kv, qo, ko = (c[x].to(DEV) for x in ("q", "kv", "qo", "ko"))
    ws = torch.empty(moe.moe_grouped_prompt_workspace_size(128), dtype=torch.uint8, device=DEV)
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)

    def call():
        moe.moe_grouped_prompt(q, kv[:, 0], kv[:, 1], qo, ko, c["scale"], max_tokens=nq[0], o=o, lse=lse, workspace=ws)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step, (a, b) in enumerate(((nq, nk), ([1, 3], [nk[0], 9]), ([nq[0], 0], [nk[0] - 200, 0]), ([0, 2], [0, nk[0]]), (nq, nk))):
        fresh = case(a, b, 12, 4, 128, seed=20 + step, spare=0)
        c.update(fresh)
        q[:len(c["q"])], kv[:len(c["kv"])] = c["q"].to(DEV), c["kv"].to(DEV)
        qo.copy_(c["qo"])
        ko.copy_(c["ko"])
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        check(c, o, lse, some_rows(c, rng, most=20))


def test_calls_at_once():
    """Calls on two streams that overlap, each with a workspace of its own: as one after the other."""
    cases = [case([5, 9], [6000, 3000], 16, 2, 128, seed=31), case([300], [300], 8, 8, 64, seed=32), case([3], [9000], 8, 1, 64, seed=33)]
    inputs = [[c[x].to(DEV) for x in ("q", "kv", "qo", "ko")] + [c["scale"], max(c["nq"])] for c in cases]

    def call(i, out):
        q, kv, qo, ko, scale, most = inputs[i]
        out.append(moe.moe_grouped_prompt(q, kv[:, 0], kv[:, 1], qo, ko, scale, max_tokens=most))

    want = []
    for i in range(3):
        call(i, want)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i, got)
    torch.cuda.synchronize()
    for n, (o, lse) in enumerate(got):
        rows = sum(cases[n % 3]["nq"])
        assert torch.equal(o[:rows], want[n % 3][0][:rows]) and torch.equal(lse[:rows], want[n % 3][1][:rows])
