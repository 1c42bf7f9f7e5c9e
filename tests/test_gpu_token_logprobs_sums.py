"""Log probabilities' sums element by element: bounds so small that one element left out, or taken twice, at the ends of a tile
or of a wavefront's part fails; rows of fp32 by a workgroup each."""
import math

import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import step as ref

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U, INF = 2.0 ** -24, math.inf
# Rows in parts that a second kernel joins, up to 64 of them; a workgroup a row, of each number of wavefronts.
SHAPES = ((1, 32769), (2, 700001), (7, 140003), (63, 40003), (64, 65537), (100, 150001), (300, 17001), (511, 33333),
          (1, 32000), (200, 9001), (512, 33333), (700, 20011), (1100, 9001), (2049, 4101))


def rows(N, V, type, fill):
    """A view of a wider tensor, so that rows begin at every alignment."""
    wide = torch.full((N, V + 1 + V % 2), math.nan, dtype=TYPES[type], device=DEV)
    x = wide[:, :V]
    x.fill_(fill)
    return x


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_equal_logits_count_to_the_vocabulary(N, V, type):
    """Every term is 1 and every reference the same: the fp64 sum is V, and its logarithm is rounded once, by at most U of
    itself.  One element more or less is 1 / V of the sum, which is more."""
    assert U * math.log(V) < 0.7 / V
    print(f"equal N={N} V={V} {type}", flush=True)
    x, t = rows(N, V, type, 0.0), torch.full((N, 1), V - 1, dtype=torch.int32, device=DEV)
    r, want = moe.moe_token_logprobs(x, t, k=3, scale=0.37), math.log(V)
    for got, sign in ((r.lse, 1), (r.entropy, 1), (r.logprob, -1), (r.top_logprob, -1)):
        assert ((sign * got.double() - want).abs() <= 1.0001 * U * want).all(), (got, want)
    assert (r.top_idx == torch.arange(3, device=DEV, dtype=torch.int32)).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_one_number_in_a_row(N, V, type):
    """Rows that are -inf but for one place, around the ends of vectors, tiles and parts: the sum is that one, exactly."""
    print(f"one N={N} V={V} {type}", flush=True)
    places = sorted({min(max(t * 2048 + d, 0), V - 1) for t in range(V // 2048 + 2) for d in (-9, -8, -1, 0, 1, 7, 8)} | {V - 2, V - 9})
    for at in range(0, len(places), N):
        mine = torch.tensor([places[(at + n) % len(places)] for n in range(N)], device=DEV)
        x = rows(N, V, type, -INF)
        x[torch.arange(N, device=DEV), mine] = 1.5
        r = moe.moe_token_logprobs(x, mine.int()[:, None].contiguous(), k=2)
        assert (r.lse == 1.5).all() and (r.entropy == 0).all() and (r.logprob == 0).all()
        assert torch.equal(r.top_idx[:, 0].long(), mine) and (r.top_idx[:, 1] == (mine == 0).int()).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_what_one_token_leaves(N, V, type):
    """All others 20 below it: the sum is 1 and (V - 1) e^-20, and the token's log probability is that little.  A term's
    exponent has three roundings of 20, its power one of 2 U, and a moved reference as much again; the entropy's sum is fp32,
    of at most V / 2048 + 100 terms one after the other."""
    print(f"left N={N} V={V} {type}", flush=True)
    x = rows(N, V, type, -20.0)
    mine = torch.arange(N, device=DEV) * 977 % V
    x[torch.arange(N, device=DEV), mine] = 0.0
    r = moe.moe_token_logprobs(x, mine.int()[:, None].contiguous(), k=1)
    rest = (V - 1) * math.exp(-20)
    log_s, tol = math.log1p(rest), 2 * (3 * 20 + 2) * U + 2 * U
    entropy = log_s + 20 * rest / (1 + rest)
    for got, want, bound in ((-r.logprob, log_s, tol), (-r.top_logprob, log_s, tol), (r.lse, log_s, tol),
                             (r.entropy, entropy, 2 * tol + (V / 2048 + 100) * U)):
        assert ((got.double() - want).abs() <= bound * want).all(), (got, want)


@pytest.mark.parametrize("N,V,k", [(512, 20011, 5), (700, 5000, 20), (1100, 9001, 64), (2600, 3001, 1), (5000, 701, 9)])
def test_many_rows_of_fp32(N, V, k):
    print(f"fp32 N={N} V={V} k={k}", flush=True)
    g = torch.Generator().manual_seed(N)
    x = torch.empty(N, V).normal_(0, 2.5, generator=g)
    x[1::3] = torch.randint(-3, 4, (len(x[1::3]), V), generator=g).float()  # ties
    x[2::5, ::2] = -INF
    x = x.to(DEV)
    t = torch.randint(0, V, (N, 2), generator=g, dtype=torch.int32).to(DEV)
    r = moe.moe_token_logprobs(x, t, k=k, scale=0.8)
    for n in sorted({0, 1, 2, 3, 4, 7, N // 2, N - 2, N - 1}):
        row = x[n].cpu().numpy()
        w, best = ref.logprobs(row, float(np.float32(0.8))), ref.order(row)[:k]
        assert r.top_idx[n].tolist() == best.tolist(), n
        assert abs(float(r.lse[n]) - w.lse) <= w.tol_lse and abs(float(r.entropy[n]) - w.entropy) <= w.tol_entropy
        for got, at in [*zip(r.logprob[n].tolist(), t[n].tolist()), *zip(r.top_logprob[n].tolist(), best.tolist())]:
            assert got == w.p[at] if math.isinf(w.p[at]) else abs(got - w.p[at]) <= w.tol_p[at], (n, at)
