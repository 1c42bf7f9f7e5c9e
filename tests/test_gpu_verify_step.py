"""The example that runs a verification step's operators together: its bookkeeping, and the two forms of latent attention
against one definition on the cache that it leaves."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "verify_step.py")
spec = importlib.util.spec_from_file_location("verify_step", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_decode(kind):
    print(f"decode {kind}", flush=True)
    model, prompts, out = example.decode(kind, lengths=(70, 1, 33), steps=5)
    assert all(len(o) >= 6 for o in out)  # a token of the prompt, then at least one a step
    assert model.pages.len.tolist() == [len(p) + len(o) - 1 for p, o in zip(prompts, out)]  # the last is not in the cache yet
    again = example.decode(kind, lengths=(70, 1, 33), steps=5)[2]
    assert out == again
    logits, _ = model.forward(torch.tensor([o[-1] for o in out], device=model.dev), model.pages.len,
                              lambda a, q, n: a.drafts(q, n, torch.arange(4, dtype=torch.int32, device=model.dev), None))
    assert torch.isfinite(logits).all()


def test_absorbed_and_expanded_forms_agree():
    """Both within their roundings of the definition in 64 bits.  Expanded: keys and values are bf16 (2^-8 of each).  Absorbed:
    the folded query is bf16, and so is the latent output before its expansion.  Both: bf16 weights and a bf16 output.  An
    error d of every score moves a weight by at most a factor of exp(2 d)."""
    model, _, _ = example.decode("latent", lengths=(50, 17), steps=3, seed=1)
    a, pages, u = model.attn[0], model.pages, 2.0 ** -8
    n = pages.len.tolist()
    g = torch.Generator().manual_seed(5)
    x = torch.randn(7, model.shape.d, generator=g).to(torch.bfloat16).to(model.dev)
    counts = [4, 3]
    pos = torch.tensor([n[b] + i for b in range(2) for i in range(counts[b])], device=model.dev)
    q, new = a.project(x, pos)
    off = torch.tensor([0, 4, 7], dtype=torch.int32, device=model.dev)
    o, _ = moe.moe_latent_attn(torch.cat([example.heads(q[0], a.w_k), q[1]], 2), new, off, a.cache, pages.table, pages.len, a.R, a.scale)
    absorbed = example.heads(o, a.w_v).double().cpu().numpy()
    rows = [torch.cat([a.cache[pages.table[b].long()].reshape(-1, 576)[:n[b]], new[off[b]:off[b + 1]]]) for b in range(2)]
    kv_off = torch.tensor([0, len(rows[0]), len(rows[0]) + len(rows[1])], dtype=torch.int32, device=model.dev)
    all_rows = torch.cat(rows)
    kv = (all_rows[:, :512].contiguous() @ a.w_kv).view(len(all_rows), a.H, -1)
    o, _ = moe.moe_latent_prompt(torch.cat(q, 2), kv[..., :128], all_rows[:, 512:].contiguous(), kv[..., 128:], off, kv_off, a.scale)
    expanded = o.double().cpu().numpy()

    w_k, w_v = a.w_k.double().cpu().numpy(), a.w_v.double().cpu().numpy()
    qn, qr = q[0].double().cpu().numpy(), q[1].double().cpu().numpy()
    for b in range(2):
        for i in range(counts[b]):
            t, c = [0, 4][b] + i, rows[b][:n[b] + i + 1].double().cpu().numpy()
            lat, rope = c[:, :512], c[:, 512:]
            for h in range(a.H):
                k, v, folded = lat @ w_k[h].T, lat @ w_v[h], qn[t, h] @ w_k[h]
                s = a.scale * (k @ qn[t, h] + rope @ qr[t, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                want = w @ v
                d = a.scale * u * (np.abs(k) @ np.abs(qn[t, h])).max()
                tol = u * np.abs(want) + 1.02 * (math.expm1(2 * d) + 2 * u) * (w @ np.abs(v)) + 1e-6
                assert np.all(np.abs(expanded[t, h] - want) <= tol), (b, i, h)
                d = a.scale * u * (np.abs(lat) @ np.abs(folded)).max()
                part = u * np.abs(w @ lat) + 1.02 * (math.expm1(2 * d) + u) * (w @ np.abs(lat))
                tol = u * np.abs(want) + 1.02 * (part @ np.abs(w_v[h])) + 1e-6
                assert np.all(np.abs(absorbed[t, h] - want) <= tol), (b, i, h)
