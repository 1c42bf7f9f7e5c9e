"""Performance cases of the operators at the two ends of a decoding step: pages and prompts in, log probabilities out.

A case is a dict of plain values.  `kind` names the operator:

  prompt    grouped-query attention over the prompts of B sequences, causal, packed
  logprobs  log probabilities of given tokens from N rows of V logits, with log-sum, entropy and the k best alternatives
  pages     pages given to and taken back from B sequences as their lengths change, slots and positions of the new tokens
  rows      rows of new tokens into the latent cache, at their slots

Lengths of a batch are drawn from the case alone, so a case's work does not depend on the seed.  Head counts are those of
the benchmark's two grouped-query layers' models (64 heads on 4 of 128; 64 heads on 8 of 64), their shares on several GPUs,
and odd ones; vocabularies are generic.
"""
import math
import random
import zlib

import torch

own = False

DEV = "cuda:0"
WIDTH = 576            # of a latent cache's row: 512 latent and 64 rotary elements
BF16, F32 = "bf16", "f32"


def _prompt(B, H, Hkv, D, T, prefix=0):
    """T: most queries of a sequence; prefix: most keys before its first query."""
    return dict(kind="prompt", B=B, H=H, Hkv=Hkv, D=D, T=T, prefix=prefix)


def _logprobs(N, V, type, M, k, scale=1.0):
    """M: given tokens a row; k: alternatives."""
    return dict(kind="logprobs", N=N, V=V, type=type, M=M, k=k, scale=scale)


def _pages(B, T, L, page, turn, spare=1.0):
    """T: most new tokens and L: longest cache of a sequence; turn: share of the sequences that end, half of them followed
    by a new one; spare: free pages at the start over those that are needed beyond the returned ones."""
    return dict(kind="pages", B=B, T=T, L=L, page=page, turn=turn, spare=spare)


def _rows(N, page, kept):
    """kept: share of the rows that go to the cache."""
    return dict(kind="rows", N=N, page=page, kept=kept)


def listed():
    return [
        # The last tokens of a prompt whose beginning is there already: few rows, a long axis.
        dict(_prompt(1, 64, 4, 128, 7, prefix=4001), name="prompt_b1_t7"),
        # Many requests of a few words, one GPU's share of eight.
        dict(_prompt(40, 8, 1, 64, 53), name="prompt_b40_t53"),
        # A batch of ordinary prompts, some behind a prefix, on a GPT-OSS layer's heads.
        dict(_prompt(6, 64, 8, 64, 1201, prefix=300), name="prompt_b6_t1201"),
        # One long prompt on a Qwen layer's heads.
        dict(_prompt(1, 64, 4, 128, 6007), name="prompt_t6007"),
        # One answered token with the 20 alternatives that a user may ask for.
        dict(_logprobs(1, 32000, BF16, 1, 20), name="logprobs_n1"),
        # The four verified tokens of one sequence; each row is asked for its node's children.
        dict(_logprobs(4, 128000, BF16, 4, 2), name="logprobs_n4"),
        # The trees of a batch at a temperature, an odd vocabulary in fp32.
        dict(_logprobs(64, 150001, F32, 2, 8, scale=1.25), name="logprobs_n64_odd"),
        # Scoring a prompt: every token's log probability.
        dict(_logprobs(2048, 200000, BF16, 1, 5), name="logprobs_n2048"),
        # The accepted tokens of a step of four sequences.
        dict(_pages(4, 5, 9001, 64, 0.0), name="pages_b4"),
        # A busy server's step: many sequences, prompts among them, some ended.
        dict(_pages(256, 2003, 20011, 16, 0.25), name="pages_b256"),
        # The accepted tokens of four sequences, of all their drafts' rows.
        dict(_rows(64, 64, 0.3), name="rows_n64"),
        # The prompt of a new conversation.
        dict(_rows(15001, 64, 1.0), name="rows_n15001"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _any(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "logprobs", "logprobs", "logprobs", "pages", "rows"])
    if kind == "prompt":
        Hkv = rng.choice([1, 2, 4, 8])
        return _prompt(_log_int(rng, 1, 64), Hkv * rng.choice([1, 2, 4, 5, 8, 16]), Hkv, rng.choice([64, 128]), _log_int(rng, 1, 6000),
                       rng.choice([0, 0, _log_int(rng, 1, 20000)]))
    if kind == "logprobs":
        return _logprobs(_log_int(rng, 1, 2048), _log_int(rng, 500, 200000), rng.choice([BF16, F32]), rng.randint(0, 8),
                         rng.choice([0, 1, rng.randint(1, 20), rng.randint(1, 64)]), rng.choice([1.0, 1.0, rng.uniform(0.3, 3.0)]))
    if kind == "pages":
        return _pages(_log_int(rng, 1, 512), _log_int(rng, 1, 4000), _log_int(rng, 1, 60000), rng.choice([16, 32, 64, 128]),
                      rng.choice([0.0, rng.random()]), rng.choice([1.0, 1.0, rng.random()]))
    return _rows(_log_int(rng, 1, 30000), rng.choice([16, 32, 64, 128]), rng.choice([1.0, rng.random()]))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def _room(case):
    """Bytes of the largest intermediate of the plain form."""
    if case["kind"] == "prompt":
        t, n = _lens(case)
        return case["B"] * case["H"] * max(t) * max(n) * 4
    return case["N"] * case["V"] * 8 if case["kind"] == "logprobs" else 0


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _any(rng)
        if _room(c) < 14e9 and _cost(c) <= most:
            return c


# ----------------------------------------------------------------------------- lengths and inputs

def _rng(case):
    return random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))


def _lens(case):
    """(queries, keys) of each prompt: the first has the most of both, the others from a spread."""
    r, T, B, prefix = _rng(case), case["T"], case["B"], case["prefix"]
    t = [T] + [r.randint(max(1, T // 4), T) for _ in range(B - 1)]
    p = [prefix] + [r.choice([0, r.randint(0, prefix)]) for _ in range(B - 1)]
    return t, [a + b for a, b in zip(t, p)]


def _requests(case):
    """(cached, kept, new) tokens of each sequence: ended ones keep nothing, and half of them make room for a prompt."""
    r, T, L = _rng(case), case["T"], case["L"]
    out = [(L, L, T)]
    for _ in range(case["B"] - 1):
        n = r.randint(L // 5, L)
        if r.random() < case["turn"]:
            out.append((n, 0, r.choice([0, r.randint(1, T)])))
        else:
            out.append((n, n, r.randint(0, min(T, 8))))
    return out


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed << 32) | zlib.crc32(tag.encode()))
    return g


def _randn(g, *shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _offsets(t):
    o = [0]
    for n in t:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    kind = case["kind"]
    g = _gen(seed, kind)
    s = dict(case)
    if kind == "prompt":
        t, n = _lens(case)
        s.update(N=sum(t), most_t=max(t), most_n=max(n), offsets=_offsets(t), kv_offsets=_offsets(n))
        s["q"] = _randn(g, sum(t), case["H"], case["D"], std=1.3)
        kv = _randn(g, sum(n), 2, case["Hkv"], case["D"])  # keys and values side by side, as a cache of them lies
        kv[:, 0, :, ::37] *= 4.0  # keys have a few large channels
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        s["scale"] = 1.0 / math.sqrt(case["D"])
        return s
    if kind == "logprobs":
        N, V = case["N"], case["V"]
        x = _randn(g, N, V, std=2.5, dtype=torch.bfloat16 if case["type"] == BF16 else torch.float32)
        # Most rows of a trained model have a few tokens far above the others, and the last few tokens are never used.
        for row in (x[::2], x[1::3]):
            row.scatter_add_(1, torch.randint(0, V, (len(row), 3), generator=g, device=DEV), _randn(g, len(row), 3, std=9.0, dtype=x.dtype).abs())
        x[:, V - V // 500:] = -math.inf
        s["logits"] = x
        s["tokens"] = torch.randint(0, V, (N, case["M"]), generator=g, device=DEV, dtype=torch.int32)
        if case["M"] > 1:
            s["tokens"][:, -1] = -1  # a node with fewer children than others
        return s
    if kind == "pages":
        reqs = _requests(case)
        page, B = case["page"], case["B"]
        have = [-(-n // page) for n, _, _ in reqs]
        want = [-(-(k + m) // page) for _, k, m in reqs]
        back = sum(max(0, h - w) for h, w in zip(have, want))
        free = max(0, int(case["spare"] * sum(max(0, w - h) for h, w in zip(have, want))) - back) + 3
        total, blocks = sum(have) + free, max(max(have), max(want), 1) + 1
        order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        s["table"] = torch.zeros(B, blocks, dtype=torch.int32, device=DEV)
        at = 0
        for b, h in enumerate(have):
            s["table"][b, :h] = order[at:at + h]
            at += h
        s["free"] = torch.zeros(total, dtype=torch.int32, device=DEV)
        s["free"][:free] = order[at:]
        s["n_free"] = torch.tensor([free], dtype=torch.int32, device=DEV)
        s["N"] = max(1, sum(m for _, _, m in reqs)) + 5  # a step's buffers have room for a few more
        s["len"] = torch.tensor([n for n, _, _ in reqs], dtype=torch.int32, device=DEV)
        s["keep"] = torch.tensor([k for _, k, _ in reqs], dtype=torch.int32, device=DEV)
        s["offsets"] = _offsets([m for _, _, m in reqs])
        return s
    N, page = case["N"], case["page"]
    M = max(1, int(N * case["kept"]))
    pages = -(-M // page) + 3
    s["new"] = _randn(g, N, WIDTH)
    s["cache"] = _randn(g, pages, page, WIDTH)
    s["row_ids"] = torch.randperm(N, generator=g, device=DEV)[:M].sort().values.to(torch.int32) if M < N else None
    # Runs of slots in pages in any order; a few rows behind the last have none.
    s["slots"] = (torch.randperm(pages, generator=g, device=DEV)[:, None] * page + torch.arange(page, device=DEV)).flatten()[:M].contiguous()
    s["slots"][M - M // 20:] = -1
    return s


# ----------------------------------------------------------------------------- the plain forms

def _plain_prompt(s):
    B, H, Hkv, D, T, M = s["B"], s["H"], s["Hkv"], s["D"], s["most_t"], s["most_n"]
    G = H // Hkv

    def ragged(offsets, most):
        at = offsets[:-1, None].long() + torch.arange(most, device=DEV)
        return at.clamp(max=offsets[-1:].long() - 1), at < offsets[1:, None]

    q_at, has = ragged(s["offsets"], T)
    k_at, kept = ragged(s["kv_offsets"], M)
    q = (s["q"][q_at].float() * s["scale"]).view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    k, v = (s[x][k_at].float().transpose(1, 2).contiguous() for x in "kv")
    lens = s["offsets"][1:] - s["offsets"][:-1]
    prefix = (s["kv_offsets"][1:] - s["kv_offsets"][:-1]) - lens
    row = torch.arange(T, device=DEV)[None] + prefix[:, None]
    seen = (torch.arange(M, device=DEV) <= row[..., None]) & kept[:, None]
    seen = seen[:, None, :, None].expand(B, 1, T, G, M).reshape(B, 1, T * G, M)
    scores = (q @ k.transpose(2, 3)).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(base).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.where(total > 0, base + total.log(), torch.full_like(total, -math.inf))[..., 0]
    o = o.view(B, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, H, D)[has]
    lse = lse.view(B, Hkv, T, G).permute(0, 2, 1, 3).reshape(B, T, H)[has]
    return {"o": o.to(torch.bfloat16), "lse": lse}


def _plain_logprobs(s):
    x = s["logits"].float()
    N, V = x.shape
    out = {}
    if s["k"]:
        # One whole number for an element: its logit's order, then the lower index.
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
        at = (V - 1) - (((order << 24) | (V - 1 - torch.arange(V, device=DEV))).topk(s["k"], dim=1).values & 0xffffff)
        out["top_idx"] = at.to(torch.int32)
    x = x * s["scale"]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    out["lse"] = (top + log_total)[:, 0]
    out["entropy"] = (log_total - torch.where(e > 0, e * (x - top), torch.zeros_like(e)).sum(1, keepdim=True) / total)[:, 0]

    def of(tokens):
        p = (x.gather(1, tokens.clamp(0, V - 1).long()) - top) - log_total
        return torch.where((tokens >= 0) & (tokens < V), p, torch.full_like(p, -math.inf))

    if s["M"]:
        out["logprob"] = of(s["tokens"])
    if s["k"]:
        out["top_logprob"] = of(out["top_idx"])
    return out


def _plain_pages(s):
    page, N = s["page"], s["N"]
    table, free, n = s["table"], s["free"], s["n_free"].long()
    B, blocks = table.shape
    old, keep, off = s["len"].long(), s["keep"].long(), s["offsets"].long()
    size = off[1:] - off[:-1]
    have, want = (old + page - 1) // page, (keep + size + page - 1) // page
    fits = want <= blocks
    back = torch.where(fits, (have - want).clamp(min=0), torch.zeros_like(have))
    take = torch.where(fits, (want - have).clamp(min=0), torch.zeros_like(have))
    # The returned pages, in order, behind the free ones.
    col = torch.arange(blocks, device=DEV)
    gone = (col >= want[:, None]) & (col < have[:, None]) & fits[:, None]
    returned = table[gone]
    free[n + torch.arange(len(returned), device=DEV)] = returned
    n = n + len(returned)
    # Pages from the end, in order of the sequences.
    upto = take.cumsum(0)
    fits &= (take == 0) | (upto <= n)
    got = (col >= have[:, None]) & (col < want[:, None]) & (fits & (take > 0))[:, None]
    b, c = got.nonzero(as_tuple=True)
    table[b, c] = free[n - 1 - (upto[b] - take[b] + c - have[b])]
    n = n - (take * fits).sum()
    # The tokens.
    t = torch.arange(N, device=DEV)
    seq = torch.searchsorted(off[1:], t, right=True).clamp(max=B - 1)
    pos = keep[seq] + t - off[seq]
    ok = (t < off[-1]) & fits[seq]
    slot = table[seq, (pos // page).clamp(0, blocks - 1)].long() * page + pos % page
    none = torch.full_like(pos, -1)
    return {"len": torch.where(fits, keep + size, old).to(torch.int32), "n_free": n.to(torch.int32),
            "slots": torch.where(ok, slot, none), "positions": torch.where(ok, pos, none).to(torch.int32),
            "refused": (~fits).sum().to(torch.int32).view(1), "table": table, "free": free}


def _plain_rows(s):
    flat = s["cache"].view(-1, WIDTH)
    new = s["new"] if s["row_ids"] is None else s["new"][s["row_ids"].long()]
    ok = (s["slots"] >= 0) & (s["slots"] < len(flat))
    flat[s["slots"][ok]] = new[ok]
    return {"cache": s["cache"]}


# ----------------------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_2607_12696_amd as moe

    kind = s["kind"]
    if kind == "prompt":
        o, lse = moe.moe_grouped_prompt(s["q"], s["k"], s["v"], s["offsets"], s["kv_offsets"], s["scale"], max_tokens=s["most_t"])
        return {"o": o, "lse": lse}
    if kind == "logprobs":
        r = moe.moe_token_logprobs(s["logits"], s["tokens"] if s["M"] else None, k=s["k"], scale=s["scale"])
        out = {"lse": r.lse, "entropy": r.entropy}
        if s["k"]:
            out.update(top_idx=r.top_idx, top_logprob=r.top_logprob)
        if s["M"]:
            out["logprob"] = r.logprob
        return out
    if kind == "pages":
        r = moe.moe_pages_update(s["len"], s["offsets"], s["table"], s["free"], s["n_free"], s["page"], s["N"], keep_len=s["keep"])
        return {"len": r.new_len, "n_free": r.n_free, "slots": r.slots, "positions": r.positions, "refused": r.refused,
                "table": s["table"], "free": s["free"]}
    moe.moe_latent_append(s["new"], s["cache"], s["slots"], rows=s["row_ids"])
    return {"cache": s["cache"]}


_PLAIN = {"prompt": _plain_prompt, "logprobs": _plain_logprobs, "pages": _plain_pages, "rows": _plain_rows}


def run(state):
    return _own(state) if own else _PLAIN[state["kind"]](state)


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "prompt":
        t, n = _lens(case)
        N, H, D = sum(t), case["H"], case["D"]
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(t, n))
        return {"bytes": N * H * (4 * D + 4) + 4 * sum(n) * case["Hkv"] * D, "flops": 4 * H * pairs * D}
    if kind == "logprobs":
        N, V = case["N"], case["V"]
        return {"bytes": N * V * (2 if case["type"] == BF16 else 4) + 4 * N * (2 * case["M"] + 2 + 2 * case["k"]), "flops": N * V * 8}
    if kind == "pages":
        reqs, page = _requests(case), case["page"]
        moved = sum(abs(-(-n // page) - -(-(k + m) // page)) for n, k, m in reqs)
        return {"bytes": case["B"] * 16 + moved * 8 + sum(m for _, _, m in reqs) * 12 + 12, "flops": 0}
    M = max(1, int(case["N"] * case["kept"]))
    written = M - M // 20
    return {"bytes": written * WIDTH * 4 + M * 8 + (4 * M if M < case["N"] else 0), "flops": 0}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    kind = case["kind"]
    f64 = torch.float64
    if kind == "pages":
        return None  # whole numbers
    s = prepare(case, seed)
    if kind == "rows":
        cache = s["cache"].to(f64)
        ids = range(case["N"]) if s["row_ids"] is None else s["row_ids"].tolist()
        for slot, row in zip(s["slots"].tolist(), ids):
            if slot >= 0:
                cache[slot // case["page"], slot % case["page"]] = s["new"][row].to(f64)
        return {"cache": cache}
    if kind == "logprobs":
        V, k, parts = case["V"], case["k"], []
        for n in range(case["N"]):
            row = s["logits"][n].to(f64)
            z = row * case["scale"]
            lse = torch.logsumexp(z, 0)
            p = z - lse
            w = p.exp()
            out = {"lse": lse, "entropy": -(w[w > 0] * p[w > 0]).sum()}
            if k:
                best = p[torch.sort(row, descending=True, stable=True).indices[:k]]
                out.update(top_idx=None, top_logprob=best)
            if case["M"]:
                ids = s["tokens"][n].long()
                out["logprob"] = torch.where(ids < 0, torch.full((case["M"],), -math.inf, dtype=f64, device=DEV), p[ids % V])
            parts.append(out)
        return {x: None if parts[0][x] is None else torch.stack([o[x] for o in parts]) for x in parts[0]}
    t, n = _lens(case)
    G, at, key, o_all, lse_all = case["H"] // case["Hkv"], 0, 0, [], []
    for a, m in zip(t, n):
        late = torch.arange(m, device=DEV)[None] > torch.arange(m - a, m, device=DEV)[:, None]
        parts = []
        for h in range(case["H"]):
            k, v = (s[x][key:key + m, h // G].to(f64) for x in "kv")
            z = (s["q"][at:at + a, h].to(f64) @ k.t()) * s["scale"]
            z.masked_fill_(late, -math.inf)
            lse = torch.logsumexp(z, 1)
            parts.append(((z - lse[:, None]).exp() @ v, lse))
        o_all.append(torch.stack([p[0] for p in parts], 1))
        lse_all.append(torch.stack([p[1] for p in parts], 1))
        at, key = at + a, key + m
    return {"o": torch.cat(o_all), "lse": torch.cat(lse_all)}
