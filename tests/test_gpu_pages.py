"""Pages, slots and positions against the definition, word for word, and the latent cache's rows; then both with the attention
that reads them."""
import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import step as ref
from synth import attention as draw

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DEV = torch.device("cuda:0")


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def pool(old, blocks, free, page, seed):
    """Table, free list and number of pages: pages in random order."""
    rng = np.random.default_rng(seed)
    have = [-(-n // page) for n in old]
    ids = rng.permutation(sum(have) + free).tolist()
    table, at = [[0] * blocks for _ in old], 0
    for b, n in enumerate(have):
        table[b][:n] = ids[at:at + n]
        at += n
    return table, ids[at:], len(ids)


def check(old, keep, new, page, blocks, free, seed=0, extra=3, keep_null=False):
    table, frees, total = pool(old, blocks, free, page, seed)
    total = max(total, 1)
    t_dev, N = dev(table), sum(new) + extra
    f_dev = torch.full((total,), -9, dtype=torch.int32, device=DEV)
    if frees:
        f_dev[:len(frees)] = dev(frees)
    n_free = dev([len(frees)])
    off = draw.offsets(new).to(DEV)
    args = dev(old), off, t_dev, f_dev, n_free, page, max(N, 1)
    r = moe.moe_pages_update(*args, keep_len=None if keep_null else dev(keep))
    want_table, want_free = [list(x) for x in table], list(frees)
    lengths, refused, tokens = ref.pages(old, [min(k, o) for k, o in zip(keep, old)], new, want_table, want_free, page)

    def same():
        assert r.new_len.tolist() == lengths and r.refused.item() == refused
        assert r.n_free.item() == len(want_free) and f_dev[:len(want_free)].tolist() == want_free
        assert t_dev.tolist() == want_table
        assert r.slots.tolist()[:len(tokens)] == [s for s, _ in tokens] and r.positions.tolist()[:len(tokens)] == [p for _, p in tokens]
        assert (r.slots[len(tokens):] == -1).all() and (r.positions[len(tokens):] == -1).all()
        # Nobody's page is anybody else's.
        held = [p for b, n in enumerate(lengths) for p in want_table[b][:-(-n // page)]] + want_free
        assert len(held) == len(set(held))

    same()
    moe.moe_pages_update(*args, keep_len=None if keep_null else dev(keep), out=r)  # the same counts again: the same results
    same()
    return refused


def test_single_tokens_and_page_ends():
    for page in (16, 32, 64, 128):
        for old in (0, 1, page - 1, page, page + 1, 5 * page):
            for new in (0, 1, page - 1, page, page + 1, 3 * page + 2):
                check([old], [old], [new], page, 12, 6, extra=0 if new else 1)


@pytest.mark.parametrize("without", [("slots",), ("positions",), ("slots", "positions")])
def test_what_is_not_asked_for(without):
    table, frees, total = pool([20, 3], 6, 5, 16, 1)

    def call(out):
        t_dev, f_dev = dev(table), torch.zeros(total, dtype=torch.int32, device=DEV)
        f_dev[:5] = dev(frees)
        r = moe.moe_pages_update(dev([20, 3]), dev([0, 15, 40]), t_dev, f_dev, dev([5]), 16, 41, out=out)
        return r, t_dev

    full, t_full = call(None)
    out = moe.PageUpdate(*(torch.full_like(x, -7) for x in (full.new_len, full.n_free, full.refused, full.slots, full.positions)))
    for name in without:
        setattr(out, name, None)
    part, t_part = call(out)
    assert part is out and torch.equal(t_full, t_part) and full.refused.item() == 0
    for name in ("new_len", "n_free", "refused", "slots", "positions"):
        assert getattr(part, name) is None if name in without else torch.equal(getattr(part, name), getattr(full, name))


def test_ends_and_begins():
    assert check([100, 40, 0, 17, 64], [100, 0, 0, 17, 10], [1, 0, 30, 0, 90], 16, 20, 4) == 0
    assert check([100, 40, 0, 17, 64], [1000, 0, 5, 17, 10], [1, 0, 30, 0, 90], 16, 20, 4, keep_null=False) == 0  # more kept than there is
    assert check([33, 48, 16], [33, 48, 16], [4, 4, 4], 16, 9, 2, keep_null=True) == 0
    # All that is taken was returned in the same call.
    assert check([160, 0, 0], [0, 0, 0], [0, 70, 80], 16, 12, 0) == 0


def test_refusals():
    assert check([16, 16, 16, 16], [16] * 4, [1, 33, 17, 0], 16, 3, 2) == 2   # past the table; past the pages
    assert check([0] * 5, [0] * 5, [40, 40, 40, 1, 0], 16, 9, 6) == 2         # nothing for those behind, small as they are
    assert check([64, 64], [64, 0], [1, 1], 64, 2, 0) == 1                    # the other's page is still its own
    assert check([64, 128], [64, 0], [1, 1], 64, 3, 0) == 0
    assert check([10], [10], [1000], 16, 4, 100) == 1


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 256, 257, 700, 1024])
def test_batches(B):
    rng = np.random.default_rng(B)
    for page, short in ((16, False), (64, True), (128, False)):
        old = [int(n) for n in rng.integers(0, 900, B)]
        ended = rng.random(B) < 0.3
        keep = [int(rng.choice([0, n // 2])) if e else n for n, e in zip(old, ended)]
        new = [int(rng.integers(0, 700)) if e or rng.random() < 0.1 else int(rng.integers(0, 6)) for e in ended]
        refused = check(old, keep, new, page, 1700 // page, 3 if short else 700 // page * B, seed=B)
        assert refused == 0 or short


def test_counts_that_break_their_contract_stay_inside():
    """Lengths, offsets and counts of any size: nothing outside the buffers is touched."""
    guard = 64
    for seed in range(6):
        g = torch.Generator().manual_seed(seed)
        wild = lambda n: torch.randint(-(1 << 31), (1 << 31) - 1, (n,), generator=g, dtype=torch.int64).to(torch.int32)  # noqa: E731
        table = torch.zeros(5 * 7 + 2 * guard, dtype=torch.int32, device=DEV)
        frees = torch.zeros(20 + 2 * guard, dtype=torch.int32, device=DEV)
        t, f = table[guard:-guard].view(5, 7), frees[guard:-guard]
        off = wild(6).sort().values.to(DEV) if seed % 2 else wild(6).to(DEV)
        moe.moe_pages_update(wild(5).to(DEV), off, t, f, wild(1).to(DEV), 16, 50, keep_len=wild(5).to(DEV))
        torch.cuda.synchronize()
        assert not table[:guard].any() and not table[-guard:].any() and not frees[:guard].any() and not frees[-guard:].any()


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("N", [1, 2, 63, 300, 5000])
def test_latent_append(N, page):
    g = torch.Generator().manual_seed(N)
    n_pages = -(-N // page) + 2
    for with_rows in (False, True):
        n_rows = N + 7
        new = draw.normal(N, "rows", n_rows, 576).to(DEV)
        cache = draw.normal(N, "cache", n_pages, page, 576).to(DEV)
        slots = torch.randperm(n_pages * page, generator=g)[:N].to(DEV)
        if N > 2:
            slots[1], slots[N - 1] = -1, n_pages * page  # both outside
        rows = torch.randint(0, n_rows, (N,), generator=g, dtype=torch.int32).to(DEV) if with_rows else None
        want = cache.clone().view(-1, 576)
        ok = (slots >= 0) & (slots < len(want))
        want[slots[ok]] = (new[:N] if rows is None else new[rows.long()])[ok]
        moe.moe_latent_append(new, cache, slots, rows=rows)
        assert torch.equal(cache.view(-1, 576).view(torch.int16), want.view(torch.int16))


def test_latent_append_past_four_gigabytes():
    n_pages = (5 << 30) // (128 * 1152)
    cache = torch.zeros(n_pages, 128, 576, dtype=torch.bfloat16, device=DEV)
    new = draw.normal(1, "rows", 3, 576).to(DEV)
    slots = torch.tensor([n_pages * 128 - 1, 0, 1 << 22], device=DEV)
    moe.moe_latent_append(new, cache, slots)
    assert torch.equal(cache.view(-1, 576)[slots], new)
    assert int((cache.view(-1, 576)[:, 0] != 0).sum()) == 3


def test_graph_of_a_step():
    """Update, append and the counts' turn captured once, replayed while requests end and begin."""
    page, B, blocks, room = 16, 3, 8, 24
    table, frees, total = pool([30, 5, 0], blocks, 9, page, 1)
    t, f = dev(table), torch.zeros(total, dtype=torch.int32, device=DEV)
    f[:len(frees)] = dev(frees)
    n, ln, keep, off = dev([len(frees)]), dev([30, 5, 0]), dev([30, 5, 0]), dev([0, 0, 0, 0])
    cache = torch.zeros(total, page, 576, dtype=torch.bfloat16, device=DEV)
    new = draw.normal(2, "rows", room, 576).to(DEV)
    out = moe.moe_pages_update(ln, off, t, f, n, page, room, keep_len=keep)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moe.moe_pages_update(ln, off, t, f, n, page, room, keep_len=keep, out=out)
        moe.moe_latent_append(new, cache, out.slots)
        ln.copy_(out.new_len)
        n.copy_(out.n_free)
    old, expect = [30, 5, 0], torch.zeros(total * page, 576, dtype=torch.bfloat16)
    want_table, want_free = [list(x) for x in table], list(frees)
    for step, (kept, fresh) in enumerate((([30, 5, 0], [4, 2, 18]), ([34, 0, 18], [1, 0, 1]), ([0, 0, 19], [20, 3, 0]), ([20, 3, 19], [0, 0, 1]))):
        new.copy_(draw.normal(step + 5, "rows", room, 576))
        keep.copy_(dev(kept))
        off.copy_(draw.offsets(fresh))
        g.replay()
        torch.cuda.synchronize()
        old, refused, tokens = ref.pages(old, kept, fresh, want_table, want_free, page)
        assert refused == 0 and ln.tolist() == old and n.item() == len(want_free) and t.tolist() == want_table
        for i, (slot, _) in enumerate(tokens):
            expect[slot] = new[i].cpu()
        assert torch.equal(cache.view(-1, 576).cpu(), expect)


def test_a_graph_and_an_eager_call_share_nothing():
    """The same pool updated by a replayed graph and eagerly, in turn: each from the counts that it is given."""
    table, frees, total = pool([20, 40], 6, 5, 16, 3)
    t, f, n = dev(table), dev(frees + [0] * (total - len(frees))), dev([len(frees)])
    ln, off = dev([20, 40]), dev([0, 13, 20])
    out = moe.moe_pages_update(ln, off, t, f, n, 16, 24)
    first = [x.clone() for x in (out.new_len, out.n_free, out.refused, out.slots, out.positions, t, f)]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        moe.moe_pages_update(ln, off, t, f, n, 16, 24, out=out)
    for _ in range(3):
        out.slots.fill_(5)
        g.replay()
        eager = moe.moe_pages_update(ln, off, t, f, n, 16, 24)
        torch.cuda.synchronize()
        for r in (out, eager):
            assert all(torch.equal(x, y) for x, y in zip(first, (r.new_len, r.n_free, r.refused, r.slots, r.positions, t, f)))
