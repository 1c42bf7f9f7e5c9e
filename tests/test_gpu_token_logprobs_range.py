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
