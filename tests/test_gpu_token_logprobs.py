"""Log probabilities, entropy and alternatives against the definitions in 64 bits: rows of one element to more than a
wavefront's tile, every alignment, ties, masks that leave few tokens or none, infinities and NaN, more alternatives than there are
numbers, rows in which every element passes what came before."""
import math

import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import step as ref
from synth import generator

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")
INF, NAN = math.inf, math.nan
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def fill(kind, N, V, seed):
    g = generator(seed, kind)
    x = torch.empty(N, V).normal_(0, 2.5, generator=g)
    if kind == "peaked":
        x[:, V // 3] += 40
    elif kind == "equal":
        x[:] = x[:, :1]
    elif kind == "ties":
        x = torch.randint(-3, 4, (N, V), generator=g).float()
        x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), generator=g) < 0.5, -1.0, 1.0)  # zeros of both signs
    elif kind == "rising":
        x = torch.arange(V).float().expand(N, V) * (30.0 / V) + torch.arange(N)[:, None]
    elif kind == "falling":
        x = -torch.arange(V).float().expand(N, V) * (30.0 / V)
    elif kind == "masked":  # few tokens allowed, from none on
        keep = torch.zeros(N, V, dtype=torch.bool)
        for n in range(N):
            keep[n, torch.randperm(V, generator=g)[:min(n, V)]] = True
        x[~keep] = -INF
    elif kind == "lowest":  # the same, with the type's lowest value
        x[:, ::2] = -3.3e38
        x[0] = -3.3e38
    elif kind == "odd":  # infinities and NaN
        for n in range(N):
            i = int(torch.randint(0, V, (1,), generator=g))
            x[n, i] = (INF, NAN, -INF)[n % 3]
            if n % 6 > 2:
                x[n] = torch.where(torch.rand(V, generator=g) < 0.97, x[n, i], x[n])
    elif kind == "large":
        x *= 1e4
    return x


def check(logits, tokens, k, scale, r, rows=None):
    x = logits.detach().float().cpu().numpy()
    N, V = x.shape
    get = {n: None if getattr(r, n) is None else getattr(r, n).cpu().numpy() for n in ("logprob", "lse", "entropy", "top_idx", "top_logprob")}
    for n in range(N) if rows is None else rows:
        w = ref.logprobs(x[n], scale)

        def same(got, want, tol, what):
            if math.isnan(want):
                assert math.isnan(got), (n, what, got, want)
            elif math.isinf(want):
                assert got == want, (n, what, got, want)
            else:
                assert abs(float(got) - want) <= tol, (n, what, got, want, tol)

        if get["lse"] is not None:
            same(get["lse"][n], w.lse, w.tol_lse, "lse")
        if get["entropy"] is not None:
            same(get["entropy"][n], w.entropy, w.tol_entropy, "entropy")
        if tokens is not None:
            given = tokens.cpu().numpy().reshape(N, -1)[n]
            mine = get["logprob"].reshape(N, -1)[n]
            for i, t in enumerate(given):
                if 0 <= t < V:
                    same(mine[i], w.p[t], w.tol_p[t], ("token", i, t))
                else:
                    assert mine[i] == -INF
        if k:
            best = ref.order(x[n])[:k]
            assert get["top_idx"][n].tolist() == best.tolist(), (n, get["top_idx"][n], best)
            if get["top_logprob"] is not None:
                for i, t in enumerate(best):
                    same(get["top_logprob"][n, i], w.p[t], w.tol_p[t], ("top", i, t))


def given(N, V, M, seed):
    g = generator(seed, "tokens")
    t = torch.randint(0, V, (N, M), generator=g, dtype=torch.int32)
    if M > 1:
        t[:, 1] = torch.where(torch.rand(N, generator=g) < 0.5, -1, V).int()
        t[:, -1] = t[:, 0]
    return t.to(DEV)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 500, 2047, 2048, 2056, 2057, 4101, 32000])
def test_sizes(V, type):
    for N, k, M in ((1, min(V, 64), 1), (3, min(V, 20), 5), (5, 1, 2), (4, 0, 3)):
        print(f"logprobs N={N} V={V} {type} k={k} M={M}", flush=True)
        x = fill("normal", N, V, V + N).to(TYPES[type]).to(DEV)
        t = given(N, V, M, V)
        check(x, t, k, 1.0, moe.moe_token_logprobs(x, t, k=k))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("kind", ["peaked", "equal", "ties", "rising", "falling", "masked", "lowest", "odd", "large"])
def test_values(kind, type):
    for N, V, k in ((12, 700, 64), (70, 3001, 20), (7, 40003, 64), (9, 40003, 5), (30, 33, 33), (2, 140003, 64)):
        print(f"logprobs {kind} N={N} V={V} {type} k={k}", flush=True)
        x = fill(kind, N, V, V).to(TYPES[type]).to(DEV)
        t = given(N, V, 3, V)
        for scale in (1.0, 0.37):
            check(x, t, k, scale, moe.moe_token_logprobs(x, t, k=k, scale=scale))


@pytest.mark.parametrize("type", TYPES)
def test_rows_of_every_alignment(type):
    """Views of a wider tensor whose other elements would win and would spoil every sum."""
    for shift in range(9):
        for V in (3, 517, 5003):
            wide = torch.full((6, V + 23), NAN, dtype=TYPES[type], device=DEV)
            x = wide[:, shift:shift + V]
            x.copy_(fill("normal", 6, V, shift))
            t = given(6, V, 2, shift)
            check(x, t, min(V, 12), 1.5, moe.moe_token_logprobs(x, t, k=min(V, 12), scale=1.5))


def test_many_rows_and_few():
    for N, V, k in ((5000, 70, 9), (4097, 1, 1), (300, 9000, 3), (2, 700001, 30)):
        x = fill("normal", N, V, N).to(torch.bfloat16).to(DEV)
        t = given(N, V, 2, N)
        rows = sorted({0, 1, N // 2, N - 2, N - 1})
        r = moe.moe_token_logprobs(x, t, k=k)
        check(x, t, k, 1.0, r, rows)
        again = moe.moe_token_logprobs(x, t, k=k)
        assert all(torch.equal(getattr(r, n), getattr(again, n)) for n in ("logprob", "lse", "entropy", "top_idx", "top_logprob"))


@pytest.mark.parametrize("V", [9, 4097, 19999])
def test_as_many_rows_as_workgroups_and_one_more(V):
    """Row counts at which another number of wavefronts takes a row."""
    whole = fill("ties", 2600, V, V).to(torch.bfloat16).to(DEV)
    for N in (256, 257, 511, 512, 513, 1023, 1024, 1025, 1280, 1281, 2048, 2049, 2560, 2561):
        print(f"logprobs rows N={N} V={V}", flush=True)
        x = whole[-N:]
        t = given(N, V, 1, N)
        check(x, t, 6, 1.0, moe.moe_token_logprobs(x, t, k=6), [0, N // 2, N - 1])


def test_forms_of_the_call():
    x = fill("normal", 6, 3000, 1).to(DEV)
    t = given(6, 3000, 4, 1)
    full = moe.moe_token_logprobs(x, t, k=7)
    one = moe.moe_token_logprobs(x, t[:, 2].contiguous())
    assert one.logprob.shape == (6,) and torch.equal(one.logprob, full.logprob[:, 2]) and one.top_idx is None
    none = moe.moe_token_logprobs(x, k=7)
    assert none.logprob is None and torch.equal(none.top_idx, full.top_idx) and torch.equal(none.lse, full.lse)
    out = moe.TokenLogprobs(None, None, None, torch.empty(6, 7, dtype=torch.int32, device=DEV), None)
    assert torch.equal(moe.moe_token_logprobs(x, k=7, out=out).top_idx, full.top_idx)
    workspace = torch.full((moe.moe_token_logprobs_workspace_size(500),), 0xff, dtype=torch.uint8, device=DEV)
    assert torch.equal(moe.moe_token_logprobs(x, t, k=7, workspace=workspace).top_logprob, full.top_logprob)


def test_rows_past_two_giga_elements():
    """Offsets of more than 32 bits; the largest element first and last in memory."""
    N, V = 17000, 131077
    x = torch.zeros(N, V, dtype=torch.bfloat16, device=DEV)
    x[0, 0] = x[-1, -1] = 3.0
    t = torch.full((N,), V - 1, dtype=torch.int32, device=DEV)
    check(x[[0, 1, -1]], t[:3], 0, 1.0, moe.moe_token_logprobs(x[[0, 1, -1]].contiguous(), t[:3]))
    r = moe.moe_token_logprobs(x, t, k=2)
    check(x[[0, 1, -1]], t[:3], 2, 1.0, moe.TokenLogprobs(*(getattr(r, n)[[0, 1, -1]] for n in ("logprob", "lse", "entropy", "top_idx", "top_logprob"))))


def test_stream_and_graph():
    """Another stream than the current one, and a captured call replayed on other logits and tokens."""
    x, t = fill("normal", 5, 20011, 3).to(torch.bfloat16).to(DEV), given(5, 20011, 2, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = moe.moe_token_logprobs(x, t, k=10)
    side.synchronize()
    check(x, t, 10, 1.0, r)
    ws = torch.empty(moe.moe_token_logprobs_workspace_size(5), dtype=torch.uint8, device=DEV)
    out = moe.moe_token_logprobs(x, t, k=10, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moe.moe_token_logprobs(x, t, k=10, out=out, workspace=ws)
    for step, kind in enumerate(("normal", "ties", "rising", "masked", "odd")):
        x.copy_(fill(kind, 5, 20011, step))
        t.copy_(given(5, 20011, 2, step + 50))
        out.top_idx.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        check(x, t, 10, 1.0, out)


@pytest.mark.parametrize("type", TYPES)
def test_rows_with_almost_all_probability_on_one_token(type):
    """Entropy and the token's log probability are as small as what is left to the others, and right to fp32's precision: the
    exponents' roundings (|x| up to 60: 60 * 4 * 2^-24 of a term), the terms' sums and one rounding of the result."""
    for N, V, over in ((4, 500, 12), (3, 40000, 25), (2, 130003, 18)):
        x = fill("normal", N, V, V)
        x[:, V // 2] = x.amax(1) + over
        x = x.to(TYPES[type])
        r = moe.moe_token_logprobs(x.to(DEV), torch.full((N,), V // 2, dtype=torch.int32, device=DEV), k=1)
        d = x.double()
        rest = torch.exp(d - d[:, V // 2:V // 2 + 1])
        rest[:, V // 2] = 0
        total, mean = rest.sum(1), (rest * (d - d[:, V // 2:V // 2 + 1])).sum(1)
        log_s = torch.log1p(total)
        entropy = log_s - mean / (1 + total)
        rel = 60 * 4 * 2.0 ** -24 + (V / 64 + 200) * 2.0 ** -24
        for got, want in ((r.logprob, -log_s), (r.top_logprob[:, 0], -log_s), (r.entropy, entropy)):
            assert ((got.cpu().double() - want).abs() <= rel * want.abs()).all(), (N, V, got, want)
