"""The most that the parts of a call's rows leave in the workspace fits it, and nothing behind it is written."""
import pytest
import torch

import paper_2607_12696_amd as moe

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("N,V", [(1, 140003), (64, 140003), (63, 200000), (85, 200000), (511, 40000), (512, 40000), (3000, 40000)])
def test_parts_stay_inside(N, V):
    print(f"workspace N={N} V={V}", flush=True)
    size = moe.moe_token_logprobs_workspace_size(N)
    buffer = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    x = torch.empty(N, V, dtype=torch.bfloat16, device=DEV).normal_(0, 3, generator=torch.Generator(DEV).manual_seed(N))
    r = moe.moe_token_logprobs(x, k=64, workspace=buffer[:size])
    assert (buffer[size:] == 0xa5).all()
    other = moe.moe_token_logprobs(x, k=64)
    assert all(torch.equal(getattr(r, n), getattr(other, n)) for n in ("lse", "entropy", "top_idx", "top_logprob"))
