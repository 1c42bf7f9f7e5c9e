"""Speculative decoding with a small random model: every operator of a verification step as a serving loop calls it.

    python examples/verify_step.py [latent|grouped]

A step takes a draft tree of each sequence through all layers at once.  Per layer: residual addition and norm, attention of
the drafts over the paged cache and each other, residual addition and norm, routing, the experts.  Then the longest path
whose tokens the model would have chosen is accepted, gets pages where it needs them, and is appended to the cache; each
token's log probability is kept.  `latent` attends over a cache of latent rows: its prompts go through the expanded form, its
drafts through the absorbed one.  `grouped` has the 8-bit cache of grouped-query attention.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_12696_amd as moe  # noqa: E402
import synth  # noqa: E402

EPS = 1e-6
BF16 = torch.bfloat16


def rotate(x, pos):
    """Rotary embedding of x [N, heads, width] at positions pos [N]."""
    half = x.shape[-1] // 2
    freq = 10000.0 ** (-torch.arange(half, device=x.device) / half)
    a = (pos[:, None] * freq)[:, None]
    x0, x1 = x.float()[..., :half], x.float()[..., half:]
    return torch.cat([x0 * a.cos() - x1 * a.sin(), x1 * a.cos() + x0 * a.sin()], -1).to(BF16)


def heads(x, w):
    """x [N, H, a] times w [H, a, b] of each head -> [N, H, b]."""
    return torch.bmm(x.transpose(0, 1).contiguous(), w).transpose(0, 1).contiguous()


class Pages:
    """Pages of B sequences of at most `room` tokens each: handed out as the sequences grow, in any order."""

    def __init__(self, B, room, page, dev):
        blocks = -(-room // page)
        self.page, self.count, self.B, self.dev = page, B * blocks, B, dev
        self.table = torch.zeros(B, blocks, dtype=torch.int32, device=dev)
        self.free = torch.randperm(B * blocks, generator=torch.Generator().manual_seed(0)).int().to(dev)
        self.n_free = torch.tensor([B * blocks], dtype=torch.int32, device=dev)
        self.len = torch.zeros(B, dtype=torch.int32, device=dev)

    def grow(self, off, n, keep=None):
        """Pages for n new tokens (sequence b's are off[b] .. off[b + 1] - 1): their slots and positions.  The old lengths
        hold until `settle`, so where some sequence's tokens do not fit nothing has changed for any."""
        update = moe.moe_pages_update(self.len, off, self.table, self.free, self.n_free, self.page, n, keep_len=keep)
        if refused := update.refused.item():
            raise RuntimeError(f"there are no pages for the new tokens of {refused} sequences")
        return update

    def settle(self, update):
        self.len, self.n_free = update.new_len, update.n_free

    def end(self, b):
        """Sequence b's pages are free again."""
        keep = self.len.clone()
        keep[b] = 0
        self.settle(self.grow(torch.zeros(self.B + 1, dtype=torch.int32, device=self.dev), 1, keep))


class LatentAttention:
    R, P, DN, DV, H = 512, 64, 128, 128, 4

    def __init__(self, d, pages, weight, dev):
        H, R = self.H, self.R
        self.scale = 1 / math.sqrt(self.DN + self.P)
        self.w_q, self.w_c, self.w_o = weight(d, H * (self.DN + self.P)), weight(d, R + self.P), weight(H * self.DV, d)
        self.w_k, self.w_v = weight(H, self.DN, R, fan=R), weight(H, R, self.DV)  # the expansions of keys and values
        self.w_kv = torch.cat([self.w_k.transpose(1, 2), self.w_v], 2).permute(1, 0, 2).reshape(R, -1).contiguous()
        self.norm = torch.ones(R, dtype=BF16, device=dev)
        self.pages = pages
        self.cache = torch.zeros(pages.count, pages.page, R + self.P, dtype=BF16, device=dev)

    def project(self, x, pos):
        q = (x @ self.w_q).view(len(x), self.H, -1)
        c = x @ self.w_c
        latent = moe.moe_add_rmsnorm(c[:, :self.R].contiguous(), self.norm, EPS, want_sum=False)[1]
        rope = rotate(c[:, None, self.R:], pos)[:, 0]
        return (q[..., :self.DN], rotate(q[..., self.DN:], pos)), torch.cat([latent, rope], 1)

    def prompt(self, q, new, off, most):
        """Queries and latent rows of whole prompts: keys and values are expanded once, for all their queries."""
        kv = (new[:, :self.R].contiguous() @ self.w_kv).view(len(new), self.H, -1)
        o, _ = moe.moe_latent_prompt(torch.cat(q, 2), kv[..., :self.DN], new[:, self.R:].contiguous(), kv[..., self.DN:], off, off,
                                     self.scale, max_tokens=most)
        return o.flatten(1) @ self.w_o

    def drafts(self, q, new, off, mask):
        """The expansions folded into the query and the output: the cache is read as it lies."""
        q = torch.cat([heads(q[0], self.w_k), q[1]], 2)
        o, _ = moe.moe_latent_attn(q, new, off, self.cache, self.pages.table, self.pages.len, self.R, self.scale, mask=mask)
        return heads(o, self.w_v).flatten(1) @ self.w_o

    def append(self, new, off, rows, slots):
        moe.moe_latent_append(new, self.cache, slots, rows=rows)


class GroupedAttention:
    D, H, HKV = 64, 8, 2

    def __init__(self, d, pages, weight, dev):
        self.scale = 1 / math.sqrt(self.D)
        self.w_qkv, self.w_o = weight(d, (self.H + 2 * self.HKV) * self.D), weight(self.H * self.D, d)
        self.pages = pages
        shape = pages.count, self.HKV
        self.k = torch.zeros(*shape, pages.page, self.D, dtype=torch.uint8, device=dev)
        self.v = torch.zeros(*shape, self.D, pages.page, dtype=torch.uint8, device=dev)
        self.ks, self.vs = torch.ones(shape, device=dev), torch.ones(shape, device=dev)

    def project(self, x, pos):
        qkv = (x @ self.w_qkv).view(len(x), -1, self.D)
        q, k, v = qkv.split([self.H, self.HKV, self.HKV], 1)
        return rotate(q, pos), (rotate(k, pos), v.contiguous())

    def prompt(self, q, new, off, most):
        o, _ = moe.moe_grouped_prompt(q, *new, off, off, self.scale, max_tokens=most)
        return o.flatten(1) @ self.w_o

    def drafts(self, q, new, off, mask):
        o, _ = moe.moe_cache_attn(q, *new, off, self.k, self.v, self.ks, self.vs, self.pages.table, self.pages.len, self.scale,
                                  mask=mask)
        return o.flatten(1) @ self.w_o

    def append(self, new, off, rows, slots):
        moe.moe_cache_append(*new, off, self.k, self.v, self.ks, self.vs, self.pages.table, self.pages.len, rows=rows, slots=slots)


class Model:
    def __init__(self, kind, B, room, layers=2, vocab=512, dev="cuda:0", seed=0):
        self.dev, self.shape = torch.device(dev), synth.SHAPES["toy"]
        g = torch.Generator().manual_seed(seed)

        def weight(*shape, fan=None):
            return (torch.randn(*shape, generator=g) / math.sqrt(fan or shape[-2])).to(BF16).to(self.dev)

        d = self.shape.d
        self.pages = Pages(B, room, 16, self.dev)
        self.embed, self.head = weight(vocab, d, fan=1), weight(d, vocab)
        self.scores = [[] for _ in range(B)]  # log probability of every chosen token
        self.ones = torch.ones(d, dtype=BF16, device=self.dev)
        make = LatentAttention if kind == "latent" else GroupedAttention
        self.attn = [make(d, self.pages, weight, self.dev) for _ in range(layers)]
        self.router = [weight(self.shape.E, d, fan=d) for _ in range(layers)]
        self.experts = [moe.pack_layer({n: w.to(self.dev) if hasattr(w, "to") else w
                                        for n, w in synth.layer_weights(self.shape, seed=i).items()}) for i in range(layers)]

    def forward(self, tokens, pos, attend):
        """Logits [N, vocab] and each layer's new cache entries; attend(layer, queries, new) -> the attention's output."""
        h, out, kept = self.embed[tokens.long()], None, []
        for attn, router, experts in zip(self.attn, self.router, self.experts):
            h, y, _, _ = moe.moe_add_rmsnorm(h if out is None else out, self.ones, EPS, residual=None if out is None else h)
            q, new = attn.project(y, pos)
            kept.append(new)
            h, y, _, _ = moe.moe_add_rmsnorm(attend(attn, q, new), self.ones, EPS, residual=h)
            idx, w = moe.moe_route_topk_hidden(y, router, self.shape.k, self.shape.score)
            out = moe.moe_verify_layer(y, experts, moe.routing_for(idx, w, self.shape.E))
        _, y, _, _ = moe.moe_add_rmsnorm(out, self.ones, EPS, residual=h, want_sum=False)
        return (y @ self.head).float(), kept

    def offsets(self, counts):
        return torch.tensor([0, *torch.tensor(counts).cumsum(0)], dtype=torch.int32, device=self.dev)

    def store(self, kept, rows, off, update):
        for attn, new in zip(self.attn, kept):
            attn.append(new, off, rows, update.slots)
        self.pages.settle(update)

    def append(self, kept, rows, counts):
        """Rows of the last forward, counts[b] of them sequence b's, to the caches."""
        off = self.offsets(counts)
        self.store(kept, rows, off, self.pages.grow(off, len(rows)))

    def best(self, logits):
        """Each row's most probable token and its log probability."""
        r = moe.moe_token_logprobs(logits, k=1)
        return r.top_idx[:, 0].tolist(), r.top_logprob[:, 0].tolist()

    def prompt(self, prompts):
        """Whole prompts into the cache -> each one's next token; None for an empty one, which leaves its sequence as it is.
        Where some come behind tokens that are cached, they go through the cached attention, 64 tokens at a time."""
        if not any(prompts):
            return [None] * len(prompts)
        if not any(n and p for n, p in zip(self.pages.len.tolist(), prompts)):
            last = self._piece(prompts, lambda a, q, n, off: a.prompt(q, n, off, max(map(len, prompts))))
        else:
            self.pages.grow(self.offsets([len(p) for p in prompts]), sum(map(len, prompts)))  # raises before the first piece does
            last = [None] * len(prompts)
            for at in range(0, max(map(len, prompts)), 64):
                piece = self._piece([p[at:at + 64] for p in prompts], lambda a, q, n, off: a.drafts(q, n, off, None))
                last = [new or old for old, new in zip(last, piece)]
        for mine, new in zip(self.scores, last):
            mine += [new[1]] if new else []
        return [new and new[0] for new in last]

    def _piece(self, prompts, attend):
        """These tokens into the cache -> each sequence's next one and its log probability, if it has any."""
        off, n = self.offsets([len(p) for p in prompts]), sum(map(len, prompts))
        update = self.pages.grow(off, n)
        tokens = torch.tensor([t for p in prompts for t in p], device=self.dev)
        logits, kept = self.forward(tokens, update.positions, lambda a, q, n: attend(a, q, n, off))
        self.store(kept, None, off, update)
        best, scores = self.best(logits)
        return [(best[e - 1], scores[e - 1]) if p else None for p, e in zip(prompts, off[1:].tolist())]

    def draft_tree(self, token, depth=3):
        """Tokens, parents and depths of a tree below `token`: two guesses a level by the embedding alone, the better one
        continued."""
        tokens, parent, level, tip = [token], [-1], [0], 0
        for n in range(1, depth + 1):
            guess = (self.embed[tokens[tip]].float() @ self.head.float()).topk(2).indices.tolist()
            at = len(tokens)
            tokens, parent, level, tip = tokens + guess, parent + [tip, tip], level + [n, n], at
        return tokens, parent, level

    def step(self, pending):
        """One verification: pending[b] is chosen but not yet in the cache -> accepted tokens, the next pending one last."""
        trees = [self.draft_tree(t) for t in pending]
        start, mask = self.pages.len.tolist(), []
        for _, parent, _ in trees:
            bits = []
            for i, p in enumerate(parent):
                bits.append((bits[p] if p >= 0 else 0) | 1 << i)
            mask += bits
        off = self.offsets([len(t[0]) for t in trees])
        masks = torch.tensor(mask, dtype=torch.int64, device=self.dev)
        tokens = torch.tensor([x for t in trees for x in t[0]], device=self.dev)
        pos = torch.tensor([start[b] + n for b, t in enumerate(trees) for n in t[2]], device=self.dev)
        logits, kept = self.forward(tokens, pos, lambda a, q, n: a.drafts(q, n, off, masks))
        (best, scores), base, rows, counts, out = self.best(logits), off.tolist(), [], [], []
        for b, (toks, parent, _) in enumerate(trees):
            path, at = [0], 0
            while True:
                follow = [i for i, p in enumerate(parent) if p == at and toks[i] == best[base[b] + at]]
                if not follow:
                    break
                at = follow[0]
                path.append(at)
            rows += [base[b] + i for i in path]
            counts.append(len(path))
            out.append([toks[i] for i in path[1:]] + [best[base[b] + at]])
        self.append(kept, torch.tensor(rows, dtype=torch.int32, device=self.dev), counts)
        for mine, at, n in zip(self.scores, self.offsets(counts).tolist(), counts):
            mine += [scores[i] for i in rows[at:at + n]]
        return out


def decode(kind, lengths=(70, 1, 33), steps=8, seed=0):
    """Prompts of these lengths, then `steps` verifications -> the model, the prompts and each sequence's tokens."""
    g = torch.Generator().manual_seed(seed)
    prompts = [torch.randint(0, 512, (n,), generator=g).tolist() for n in lengths]
    model = Model(kind, len(prompts), max(lengths) + 4 * steps, seed=seed)
    out = [[t] for t in model.prompt(prompts)]
    for _ in range(steps):
        for mine, new in zip(out, model.step([o[-1] for o in out])):
            mine += new
    return model, prompts, out


if __name__ == "__main__":
    for which in sys.argv[1:] or ["latent", "grouped"]:
        m, prompts, out = decode(which)
        print(f"{which}: prompts of {[len(p) for p in prompts]} tokens, 8 verifications, {[len(o) for o in out]} tokens of log "
              f"probability {[round(sum(s) / len(s), 2) for s in m.scores]} on average")
