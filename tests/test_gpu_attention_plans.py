"""How the cached attention is shared out: batches with more row groups than run at once whose groups are still cut (the plan
read back from the workspace, so that the case stays one), batches with many idle sequences, a workspace larger than the call
needs; and graphs of the calls replayed on other lengths and inputs."""
import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from synth import attention as draw
from test_gpu_attention import (DEV, R, cache_case, cache_rows, cache_run, compare, dev, latent_case, latent_rows, latent_run,
                                prompt_case, prompt_rows, some_rows)

pytestmark = pytest.mark.gpu

CUS = 256


def plan(workspace):
    """(sequence, group, chunks, first slot, stride) of each row group."""
    n = int(workspace[:4].view(torch.int32).item())
    return workspace[256:256 + 20 * n].view(torch.int32).view(n, 5).cpu()


def workspace_of(size, *args):
    return torch.zeros(size(*args), dtype=torch.uint8, device=DEV)


def latent_workspace(c, N=None, B=None):
    B = B or len(c["lens"])
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    table = torch.zeros(B, c["table"].shape[1], dtype=torch.int32, device=DEV)
    return workspace_of(moe.moe_latent_attn_workspace_size, c["store"].to(DEV), table, n, R, N or c["N"], c["H"])


def cache_workspace(c, N=None, B=None):
    B = B or len(c["lens"])
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    table = torch.zeros(B, c["table"].shape[1], dtype=torch.int32, device=DEV)
    return workspace_of(moe.moe_cache_attn_workspace_size, *dev(*(c[x] for x in ("k", "v", "ks", "vs"))), table, n, N or c["N"], c["H"])


@pytest.mark.parametrize("B", [300, 400])
def test_more_row_groups_than_slots_and_cut(B):
    """Single tokens over 0 to 400 cached ones, and one over 4000: several rounds of chunks, most row groups in parts."""
    rng = np.random.default_rng(7)
    lens = [4000] + [int(n) for n in rng.integers(0, 400, B - 1)]
    rows = lambda H: some_rows([1] * B, H, rng) + [(0, 0, 0, H - 1)]  # noqa: E731
    c = latent_case([1] * B, lens, 16, 16, seed=40, poison=True)
    ws = latent_workspace(c)
    o, lse = latent_run(c, workspace=ws)
    p = plan(ws)
    assert len(p) == B > CUS and (p[:, 2] > 1).sum() > 20 and int(p[:, 2].sum()) > CUS, p[:, 2]
    compare(latent_rows(c, rows(16)), o, lse)
    again = latent_run(c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])

    c = cache_case([1] * B, lens, 4, 2, 64, 16, seed=41, poison=True)
    ws = cache_workspace(c)
    o, lse = cache_run(c, workspace=ws)
    p = plan(ws)
    assert len(p) == 2 * B > 2 * CUS and (p[:, 2] > 1).sum() > 20 and int(p[:, 2].sum()) > 2 * CUS, p[:, 2]
    compare(cache_rows(c, rows(4)), o, lse)
    again = cache_run(c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("counts", [[0] * 20 + [40] + [0] * 19, [3] + [0] * 60 + [4, 0, 0]])
def test_idle_sequences(counts):
    """A few trees among many sequences that have nothing to verify."""
    lens = [(37 * i) % 500 + (900 if n else 0) for i, n in enumerate(counts)]
    rng = np.random.default_rng(3)
    c = latent_case(counts, lens, 16, 32, seed=42, poison=True)
    compare(latent_rows(c, some_rows(counts, 16, rng)), *latent_run(c))
    c = cache_case(counts, lens, 16, 4, 64, 32, seed=43, poison=True)
    compare(cache_rows(c, some_rows(counts, 16, rng)), *cache_run(c))


def test_one_workspace_for_the_largest_call():
    """Calls of every smaller kind in the workspace of 64 tokens of 32 sequences, give what they give in their own."""
    for counts, lens in (([64], [3000]), ([1] * 32, list(range(0, 3200, 100))), ([8] * 8, [700] * 8), ([2] * 20 + [0] * 12, [333] * 32)):
        c = latent_case(counts, lens, 16, 64, seed=44)
        want = latent_run(c)
        got = latent_run(c, workspace=latent_workspace(c, 64, 32))
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        c = cache_case(counts, lens, 64, 8, 64, 64, seed=45)
        want = cache_run(c)
        got = cache_run(c, workspace=cache_workspace(c, 64, 32))
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# ----------------------------------------------------------------------------- graphs

def captured(call):
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    return g


def test_graph_of_the_8_bit_cache():
    """Captured once; lengths, queries and codes change between replays."""
    c = cache_case([4, 2], [1500, 90], 16, 4, 64, 64, seed=50)
    ln = torch.tensor(c["lens"], dtype=torch.int32)
    q, kn, vn, off, k, v, ks, vs, table, ln, mask = dev(*(c[x] for x in ("q", "kn", "vn", "off", "k", "v", "ks", "vs", "table")), ln, c["mask"])
    ws = cache_workspace(c)
    o, lse = torch.empty_like(q), torch.empty(c["N"], 16, device=DEV)

    def call():
        moe.moe_cache_attn(q, kn, vn, off, k, v, ks, vs, table, ln, c["scale"], mask=mask, o=o, lse=lse, workspace=ws)

    g = captured(call)
    for step, n in enumerate((1500, 333, 64, 0, 1)):
        ln[0], c["lens"][0] = n, n
        c["q"], c["k"] = draw.normal(60 + step, "q", *q.shape), draw.codes(60 + step, "k", *k.shape)
        q.copy_(c["q"])
        k.copy_(c["k"])
        o.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        call()
        assert torch.equal(o, got[0]) and torch.equal(lse, got[1])
        compare(cache_rows(c, some_rows([4, 2], 16, np.random.default_rng(step), most=12)), *got)


def test_graph_of_prompts():
    """Captured for up to 200 queries a sequence; the offsets and the inputs change between replays."""
    c = prompt_case([200, 30], [260, 30], 3, seed=51)
    q, kv, rope, qo, ko = dev(c["q"], c["kv"], c["rope"], c["qo"], c["ko"])
    o, lse = torch.empty(230, 3, 128, dtype=torch.bfloat16, device=DEV), torch.empty(230, 3, device=DEV)

    def call():
        moe.moe_latent_prompt(q, kv[..., :128], rope, kv[..., -128:], qo, ko, c["scale"], max_tokens=200, o=o, lse=lse)

    g = captured(call)
    for step, (nq, nk) in enumerate((([200, 30], [260, 30]), ([1, 64], [200, 64]), ([100, 0], [90, 0]), ([0, 190], [0, 290]))):
        c.update(nq=nq, nk=nk, qo=draw.offsets(nq), ko=draw.offsets(nk), q=draw.normal(70 + step, "q", *q.shape, std=1.5))
        q.copy_(c["q"])
        qo.copy_(c["qo"])
        ko.copy_(c["ko"])
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        call()
        n = sum(nq)
        assert torch.equal(o[:n], got[0][:n]) and torch.equal(lse[:n], got[1][:n])
        compare(prompt_rows(c, some_rows(nq, 3, np.random.default_rng(step), most=20)), *got)
