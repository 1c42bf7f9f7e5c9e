"""What the example's decoding loop leaves in its caches: the accepted tokens' entries, each at its own position, after
verifications that accept more than the root of their trees."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import attention as ref

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "verify_step.py")
spec = importlib.util.spec_from_file_location("verify_step", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)

U = 2.0 ** -8  # of a bf16 rounding
LENGTHS, ROOM = (70, 1, 33), 40


def model_of(kind):
    return example.Model(kind, len(LENGTHS), max(LENGTHS) + ROOM, seed=0)


def prompts():
    g = torch.Generator().manual_seed(0)
    return [torch.randint(0, 512, (n,), generator=g).tolist() for n in LENGTHS]


def greedy(kind, n):
    """n tokens of each sequence, one a step: trees of a root alone."""
    model = model_of(kind)
    model.draft_tree = lambda token: ([token], [-1], [0])
    out = [[t] for t in model.prompt(prompts())]
    for _ in range(n - 1):
        for mine, new in zip(out, model.step([o[-1] for o in out])):
            assert len(new) == 1
            mine += new
    return out


def speculative(kind, steps, known):
    """Steps whose trees hold the next tokens of `known` among wrong ones (on the second child, then the first, then the
    second) -> the model, each sequence's tokens, and what each call of append got."""
    model = model_of(kind)
    out = [[t] for t in model.prompt(prompts())]
    turn, log = [0], []

    def draft_tree(token):
        b = turn[0] % len(out)
        turn[0] += 1
        n = len(out[b])
        right = known[b][n:n + 3] if known[b][:n] == out[b] else []
        tokens, parent, level, tip = [token], [-1], [0], 0
        for d, t in enumerate(right):
            wrong, at = (t + 1 + d) % 512, len(tokens)
            tokens += [wrong, t] if d % 2 == 0 else [t, wrong]
            parent, level = parent + [tip, tip], level + [d + 1, d + 1]
            tip = at + (1 if d % 2 == 0 else 0)
        return tokens, parent, level

    append = model.append

    def logged(kept, rows, counts):
        log.append(([[x.clone() for x in (k if isinstance(k, tuple) else (k,))] for k in kept], rows.tolist(), list(counts),
                    model.pages.len.tolist()))
        append(kept, rows, counts)

    model.draft_tree, model.append = draft_tree, logged
    accepted = []
    for _ in range(steps):
        new = model.step([o[-1] for o in out])
        accepted += [len(x) for x in new]
        for mine, x in zip(out, new):
            mine += x
    return model, out, log, accepted


def at(model, b, i):
    return int(model.pages.table[b, i // model.pages.page]), i % model.pages.page


def decoded(a, page, slot):
    """Keys and values [HKV, D] of a token in the 8-bit cache, and their pages' scales."""
    ks, vs = a.ks[page].double().cpu().numpy()[:, None], a.vs[page].double().cpu().numpy()[:, None]
    return ref.E4M3[a.k[page, :, slot].cpu().numpy()] * ks, ref.E4M3[a.v[page, :, :, slot].cpu().numpy()] * vs, ks, vs


def coded(want, tol, scale):
    """The bound on an 8-bit entry: half a step of three bits, or of the smallest codes' spacing once for each growth of the
    page's power-of-two scale (halves of halves: twice the last)."""
    return 1.07 * tol + 2.0 ** -4 * np.abs(want) + 2.0 ** -9 * scale


@pytest.mark.parametrize("kind", ["latent", "grouped"])
def test_cache_after_accepted_paths(kind):
    known = greedy(kind, 16)
    model, out, log, accepted = speculative(kind, 5, known)
    print(kind, accepted, flush=True)
    assert max(accepted) == 4 and sum(n > 1 for n in accepted) >= 3  # the root and three drafts; most paths are not the root alone
    lens = model.pages.len.tolist()
    text = [p + o[:-1] for p, o in zip(prompts(), out)]
    assert lens == [len(t) for t in text]

    # Every layer's rows of every accepted path lie at the positions that follow each other.
    for kept, rows, counts, start in log:
        n = 0
        for b, count in enumerate(counts):
            for i in range(count):
                page, slot = at(model, b, start[b] + i)
                for attn, new in zip(model.attn, kept):
                    mine = [x[rows[n]] for x in new]
                    if kind == "latent":
                        assert torch.equal(attn.cache[page, slot], mine[0])
                        continue
                    k, v, ks, vs = decoded(attn, page, slot)
                    for got, x, s in ((k, mine[0], ks), (v, mine[1], vs)):
                        want = x.double().cpu().numpy()
                        assert np.all(np.abs(got - want) <= coded(want, 0.0, s))
                n += 1

    # The first layer's entries follow from a token and its position alone.  In 64 bits, with a bf16 rounding of the norm, of
    # the product and of what is stored, fp32 sums of d terms, and angles of some 1e-4.
    a, e = model.attn[0], model.embed.double().cpu().numpy()
    w = (a.w_c if kind == "latent" else a.w_qkv).double().cpu().numpy()

    def product(token):
        _, y = ref.rmsnorm(e[token][None], None, np.ones(e.shape[1]), example.EPS)
        c = y[0] @ w
        return c, U * np.abs(c) + (U + e.shape[1] * 2.0 ** -24) * (np.abs(y[0]) @ np.abs(w))

    def rotated(x, tol, pos):
        half = x.shape[-1] // 2
        ang = pos * 10000.0 ** (-np.arange(half) / half)
        c, s, x0, x1, t0, t1 = np.cos(ang), np.sin(ang), x[..., :half], x[..., half:], tol[..., :half], tol[..., half:]
        r = np.concatenate([x0 * c - x1 * s, x1 * c + x0 * s], -1)
        size = np.concatenate([np.abs(x0) + np.abs(x1)] * 2, -1)
        return r, U * np.abs(r) + 2e-4 * size + np.concatenate([t0 * np.abs(c) + t1 * np.abs(s), t1 * np.abs(c) + t0 * np.abs(s)], -1)

    def wants(token, pos):
        c, tol = product(token)
        if kind == "latent":
            lat, size = c[:a.R], np.sqrt(np.mean(c[:a.R] ** 2) + example.EPS)
            moved = np.linalg.norm(tol[:a.R]) / np.linalg.norm(lat)
            lat, tol_lat = lat / size, 1.05 * (tol[:a.R] + np.abs(lat) * moved) / size + U * np.abs(lat / size)
            rope, tol_rope = rotated(c[a.R:], tol[a.R:], pos)
            return np.concatenate([lat, rope]), np.concatenate([tol_lat, tol_rope])
        c, tol = (x[a.H * a.D:].reshape(2, a.HKV, a.D) for x in (c, tol))
        k, tol_k = rotated(c[0], tol[0], pos)
        return np.stack([k, c[1]]), np.stack([tol_k, tol[1]])

    def fits(b, i, token, pos):
        page, slot = at(model, b, i)
        want, tol = wants(token, pos)
        if kind == "latent":
            got = a.cache[page, slot].double().cpu().numpy()
        else:
            k, v, ks, vs = decoded(a, page, slot)
            got, tol = np.stack([k, v]), coded(want, tol, np.stack([ks, vs]) * np.ones_like(want))
        return bool(np.all(np.abs(got - want) <= tol))

    for b, mine in enumerate(text):
        for i, token in enumerate(mine):
            assert fits(b, i, token, i), (b, i)
            # The bound tells tokens and positions apart.
            assert not fits(b, i, (token + 1) % 512, i) and not fits(b, i, token, i + 1), (b, i)
