"""The example's prompts behind tokens that are cached already: they attend to those too."""
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


def recorded(kind, B=2, room=300):
    """A model that keeps the logits of every call."""
    model, seen = example.Model(kind, B, room, seed=7), []
    forward = model.forward

    def kept(*a):
        out = forward(*a)
        seen.append(out[0].clone())
        return out

    model.forward = kept
    return model, seen


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_a_second_prompt_sees_the_first(kind):
    """Its logits are those of the cached attention on the same tokens, and other ones behind another first prompt."""
    print(f"second prompt {kind}", flush=True)
    model, seen = recorded(kind)
    model.prompt([text(50, 1), text(9, 2)])
    more = [text(130, 3), text(70, 4)]
    nxt, start = model.prompt(more), len(seen) - 3
    assert model.pages.len.tolist() == [180, 79]

    other, _ = recorded(kind)
    other.prompt([text(50, 1), text(9, 2)])
    lens, last = [50, 9], [None, None]
    for i, counts in enumerate(([64, 64], [64, 6], [2, 0])):  # drafts of at most 64 tokens, each one's parent the one before it
        off = other.offsets(counts)
        pieces = [p[64 * i:64 * i + n] for p, n in zip(more, counts)]
        pos = torch.tensor([lens[b] + j for b, n in enumerate(counts) for j in range(n)], device=other.dev)
        tokens = torch.tensor([t for p in pieces for t in p], device=other.dev)
        logits, kept = other.forward(tokens, pos, lambda a, q, n: a.drafts(q, n, off, None))
        assert torch.equal(logits, seen[start + i])
        other.append(kept, torch.arange(len(tokens), dtype=torch.int32, device=other.dev), counts)
        for b, e in enumerate(off[1:].tolist()):
            last[b] = int(logits[e - 1].argmax()) if counts[b] else last[b]
        lens = [n + c for n, c in zip(lens, counts)]
    assert nxt == last

    third, seen_third = recorded(kind)
    third.prompt([text(50, 5), text(9, 2)])
    third.prompt(more)
    n = 64  # the first sequence's tokens of the first piece; the second sequence's have the same before them
    assert not torch.equal(seen[start][:n], seen_third[start][:n])
    assert len(model.scores[0]) == 2 and len(model.scores[1]) == 2


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_a_second_prompt_that_does_not_fit_leaves_everything(kind):
    print(f"refused second prompt {kind}", flush=True)
    model, _ = recorded(kind, room=160)
    model.prompt([text(50, 1), text(9, 2)])
    lens, free, scores = model.pages.len.tolist(), int(model.pages.n_free), [list(s) for s in model.scores]
    with pytest.raises(RuntimeError):
        model.prompt([text(130, 3), text(20, 4)])  # its first pieces alone would fit
    assert model.pages.len.tolist() == lens and int(model.pages.n_free) == free and model.scores == scores
    model.prompt([text(110, 3), text(20, 4)])
    assert model.pages.len.tolist() == [160, 29]


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_a_sequence_without_a_prompt_has_no_next_token(kind):
    print(f"no prompt {kind}", flush=True)
    model, _ = recorded(kind, B=3)
    assert model.prompt([[], [], []]) == [None] * 3 and model.pages.len.tolist() == [0, 0, 0]
    first = model.prompt([text(5, 1), [], text(3, 2)])
    assert first[1] is None and all(isinstance(first[b], int) for b in (0, 2))
    second = model.prompt([[], text(4, 3), text(90, 4)])  # one behind cached tokens
    assert second[0] is None and all(isinstance(second[b], int) for b in (1, 2))
    assert model.pages.len.tolist() == [5, 4, 93] and [len(s) for s in model.scores] == [1, 1, 2]
