"""The example's loop with requests that end and begin: prompts, drafts, pages, caches and log probabilities run together."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "verify_step.py")
spec = importlib.util.spec_from_file_location("verify_step", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def accounted(pages):
    """Every page is one sequence's or free."""
    n = int(pages.n_free)
    held = [p for b, ln in enumerate(pages.len.tolist()) for p in pages.table[b, :-(-ln // pages.page)].tolist()]
    assert sorted(held + pages.free[:n].tolist()) == list(range(pages.count))
    return n


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_requests_end_and_begin(kind):
    g = torch.Generator().manual_seed(3)
    prompt = lambda n: torch.randint(0, 512, (n,), generator=g).tolist()  # noqa: E731
    model = example.Model(kind, 3, 150, seed=2)
    forward, seen = model.forward, []

    def recorded(*a):
        out = forward(*a)
        seen.append(out[0].clone())
        return out

    model.forward = recorded
    texts = [prompt(40), prompt(3), prompt(97)]
    pending = model.prompt(texts)
    free = accounted(model.pages)
    for step in range(6):
        if step == 3:  # the second request ends, and another takes its place
            before = model.pages.len.tolist()
            model.pages.end(1)
            assert model.pages.len.tolist() == [before[0], 0, before[2]] and accounted(model.pages) > free
            others = model.attn[0].k if kind == "grouped" else model.attn[0].cache
            kept = others[model.pages.table[2, :2].long()].clone()
            new = model.prompt([[], prompt(60), []])
            assert model.pages.len.tolist() == [before[0], 60, before[2]]
            assert torch.equal(kept, others[model.pages.table[2, :2].long()])
            pending[1] = new[1]
        out = model.step(pending)
        pending = [o[-1] for o in out]
        free = accounted(model.pages)
    assert all(torch.isfinite(x).all() for x in seen)

    # Each score is the log probability of a row's best token.
    best = torch.cat([torch.log_softmax(x.double(), 1).amax(1) for x in seen]).cpu()
    for scores in model.scores:
        for s in scores:
            assert float((best - s).abs().min()) <= 1e-5 + 1e-6 * abs(s)
    lens = model.pages.len.tolist()
    assert len(model.scores[0]) == lens[0] - 40 + 1 and len(model.scores[2]) == lens[2] - 97 + 1  # the last is not in the cache
    assert len(model.scores[1]) >= 2 + 6 and all(math.isfinite(s) for scores in model.scores for s in scores)


def test_prompt_and_drafts_of_the_grouped_form_agree():
    """A prompt through its own kernel, and again as drafts over an empty cache: one definition, of bf16 keys and values, a
    bf16 rounding of each weight and of the output, before the output's product."""
    model = example.Model("grouped", 1, 64, seed=4)
    a = model.attn[0]
    x = torch.randn(60, model.shape.d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(model.dev)
    q, new = a.project(x, torch.arange(60, device=model.dev))
    off = torch.tensor([0, 60], dtype=torch.int32, device=model.dev)
    a.w_o = torch.eye(a.H * a.D, dtype=torch.bfloat16, device=model.dev)  # the attention's output itself
    whole, drafts = a.prompt(q, new, off, 60), a.drafts(q, new, off, None)
    size = new[1].abs().amax().item()
    # Either is within 2^-8 of its value and 2^-8 of the weights' values from the definition.
    assert float((whole.float() - drafts.float()).abs().max()) <= 4 * 2.0 ** -8 * size * 1.05
