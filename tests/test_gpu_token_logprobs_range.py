"""Log probabilities at the ends of fp32's range: scaled logits that pass it, and differences of logits that do."""
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
INF = math.inf
# Rows by one workgroup, one launch; by parts and a join; more rows than workgroups at once.
SHAPES = ((1, 9), (3, 700), (5, 3001), (2, 40003), (2, 140003), (600, 5000))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_a_scaled_logit_that_overflows(N, V, type):
    """One logit of the row times the scale is past fp32: no sum of the row is a number, but the order of the logits stands.
    The rows beside it are as they were."""
    print(f"overflow N={N} V={V} {type}", flush=True)
    g = torch.Generator().manual_seed(V)
    x = torch.empty(N, V).normal_(0, 1e3, generator=g)
    bad = [0] if N == 1 else [0, N - 1]
    for n in bad:
        x[n, V // 3] = 3e38
    x = x.to(TYPES[type]).to(DEV)
    t = torch.full((N, 3), V // 3, dtype=torch.int32, device=DEV)
    t[:, 1], t[:, 2] = 0, -1
    for scale in (1.25, 2.0, 1e30):
        r = moe.moe_token_logprobs(x, t, k=4, scale=scale)
        for n in bad:
            assert all(torch.isnan(y[n]).all() for y in (r.lse, r.entropy, r.logprob[:, :2], r.top_logprob)), (n, scale)
            assert r.logprob[n, 2] == -INF
            assert r.top_idx[n].tolist() == ref.order(x[n].float().cpu().numpy())[:4].tolist()
        good = torch.tensor([n for n in range(N) if n not in bad], dtype=torch.long, device=DEV)
        if len(good):
            assert torch.isfinite(r.lse[good]).all() and torch.isfinite(r.entropy[good]).all()
    # The largest scaled logit that is a number: so are the results.
    r = moe.moe_token_logprobs(x, t, k=4, scale=1.0)
    assert torch.isfinite(r.lse).all() and (r.logprob[bad, 0] == 0).all() and (r.entropy[bad] == 0).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_logits_further_apart_than_fp32_reaches(N, V, type):
    """Logits of both signs near the type's ends, and a scale that makes ordinary numbers of them: their difference is past
    fp32, the scaled one is not.  Bounds of the definition; the halves that the difference is taken of are exact."""
    print(f"apart N={N} V={V} {type}", flush=True)
    g = torch.Generator().manual_seed(V + 1)
    x = torch.empty(N, V).normal_(0, 1.2e38, generator=g).clamp_(-3.3e38, 3.3e38)
    x[:, V // 2] = 3.3e38
    x[:, 0] = -3.3e38
    if N > 1:
        x[1] = torch.where(torch.rand(V, generator=g) < 0.5, 3.2e38, -3.2e38)
        x[N - 1, 1:V // 2] = -INF
    x = x.to(TYPES[type]).to(DEV)
    t = torch.tensor([0, V // 2, V - 1, V, V // 3], dtype=torch.int32, device=DEV).expand(N, 5).contiguous()
    rows = range(N) if N < 10 else (0, 1, 2, N // 2, N - 1)
    for scale in (2e-38, 1e-37, 5e-36):
        scale = float(np.float32(scale))
        r = moe.moe_token_logprobs(x, t, k=5, scale=scale)
        for n in rows:
            row = x[n].float().cpu().numpy()
            w, best = ref.logprobs(row, scale), ref.order(row)[:5]
            assert r.top_idx[n].tolist() == best.tolist()
            assert abs(float(r.lse[n]) - w.lse) <= w.tol_lse and abs(float(r.entropy[n]) - w.entropy) <= w.tol_entropy, (n, scale)
            for got, at in [*zip(r.logprob[n].tolist(), t[n].tolist()), *zip(r.top_logprob[n].tolist(), best.tolist())]:
                if at >= V or w.p[at] == -INF:
                    assert got == -INF
                else:
                    assert abs(got - w.p[at]) <= w.tol_p[at], (n, scale, at, got, w.p[at])


@pytest.mark.parametrize("type", TYPES)
def test_the_largest_scale(type):
    """2^126: twice its product with log2 e is a number, and equal logits are as probable as each other."""
    for V in (1, 5, 3001, 40003):
        x = torch.full((3, V), 0.25, dtype=TYPES[type], device=DEV)
        x[2, 1:] = 0.125
        r = moe.moe_token_logprobs(x, torch.zeros(3, 1, dtype=torch.int32, device=DEV), scale=2.0 ** 126)
        for n, (lse, p) in enumerate(((2.0 ** 124, -math.log(V)), (2.0 ** 124, -math.log(V)), (2.0 ** 124, 0.0))):
            assert r.lse[n] == lse and abs(float(r.logprob[n, 0]) - p) <= 2.0 ** -22 * abs(p)
            assert abs(float(r.entropy[n]) + p) <= 2.0 ** -22 * abs(p)
