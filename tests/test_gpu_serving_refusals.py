"""The example's loop where pages run out: a call whose tokens do not fit raises and leaves every sequence as it was."""
import importlib.util
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


def text(n, seed):
    return torch.randint(0, 512, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


def caches(model):
    """Every byte of every layer's cache, scales among them."""
    return [x.clone() for a in model.attn for x in ((a.cache,) if hasattr(a, "cache") else (a.k, a.v, a.ks, a.vs))]


def state(model):
    p = model.pages
    lens = p.len.tolist()
    held = [p.table[b, :-(-n // p.page)].tolist() for b, n in enumerate(lens)]
    return lens, held, p.free[:int(p.n_free)].tolist(), [list(s) for s in model.scores]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_a_prompt_that_does_not_fit(kind):
    """Past its sequence's room, beside one that would fit; the others' pages are not touched, and the loop goes on as one that
    never had the call."""
    print(f"refused prompt {kind}", flush=True)
    model, other = (example.Model(kind, 3, 90, seed=5) for _ in range(2))
    first = [text(40, 1), text(70, 2), []]
    pending, same_pending = model.prompt(first), other.prompt(first)
    assert pending == same_pending
    before, bytes_before = state(model), caches(model)
    for bad in ([[], [], text(97, 3)], [text(3, 4), [], text(200, 5)], [[], text(27, 6), text(10, 7)]):
        with pytest.raises(RuntimeError):
            model.prompt(bad)
        assert state(model) == before and same(bytes_before, caches(model))
    good = [[], [], text(96, 8)]
    pending[2], same_pending[2] = model.prompt(good)[2], other.prompt(good)[2]
    assert pending == same_pending and state(model) == state(other) and same(caches(model), caches(other))


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_a_step_that_does_not_fit(kind):
    """Sequences of one page short of their room's end: the step whose accepted tokens need more raises, as often as it is
    tried, until a request ends."""
    print(f"refused step {kind}", flush=True)
    model = example.Model(kind, 2, 48, seed=6)
    model.draft_tree = lambda token: ([token], [-1], [0])  # one token a step
    pending = model.prompt([text(47, 1), text(5, 2)])
    pending = [o[-1] for o in model.step(pending)]
    assert model.pages.len.tolist() == [48, 6]
    before, bytes_before = state(model), caches(model)
    for _ in range(2):
        with pytest.raises(RuntimeError):
            model.step(pending)
        assert state(model) == before and same(bytes_before, caches(model))
    model.pages.end(0)
    assert model.pages.len.tolist() == [0, 6]
    model.step(pending)
    assert model.pages.len.tolist() == [1, 7]
