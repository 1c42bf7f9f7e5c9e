"""Performance cases of the operators around an MoE layer's verification pass: the norm before it and the attention.

A case is a dict of plain values.  `kind` names the operator:

  norm    residual addition and RMS norm of T rows of width d, with a bf16 and an 8-bit output (`q`: the 8-bit format)
  latent  latent attention in the absorbed form: the draft tokens of B sequences over a paged cache of one latent vector
          a token, and over each other through a tree mask
  prompt  latent attention in the expanded form: the prompts of B sequences, causal, with per-head keys and values
  append  accepted tokens into the paged 8-bit key/value cache, with one scale for a page and head
  cache   grouped-query attention of the draft tokens of B sequences over that cache, and over each other

Lengths of the sequences of a batch are drawn from the case alone, so a case's work does not depend on the seed.
Head counts and cache widths are those of the benchmark's three layers' models (128 heads on a 512 + 64 wide latent; 64
heads on 4 heads of 128; 64 heads on 8 heads of 64), their shares on several GPUs, and odd ones.
"""
import math
import random
import zlib

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
R, P = 512, 64         # latent and rotary width of a cached token
DN, DV = 128, 128      # per-head key width (without the rotary part) and value width of the expanded form
Q_NONE, Q_G128, Q_MX, Q_ROW = 0, 1, 2, 3


def _norm(T, d, q, y=True):
    return dict(kind="norm", T=T, d=d, q=q, y=y)


def _latent(B, H, T, L, page, tree=True):
    """T: most draft tokens of a sequence, L: longest cache; other sequences of the batch have fewer."""
    return dict(kind="latent", B=B, H=H, T=T, L=L, page=page, tree=tree)


def _prompt(B, H, T, prefix=0):
    return dict(kind="prompt", B=B, H=H, T=T, prefix=prefix)


def _append(B, Hkv, D, T, L, page):
    return dict(kind="append", B=B, Hkv=Hkv, D=D, T=T, L=L, page=page)


def _cache(B, H, Hkv, D, T, L, page, tree=True):
    return dict(kind="cache", B=B, H=H, Hkv=Hkv, D=D, T=T, L=L, page=page, tree=tree)


def listed():
    return [
        # The norm before the router in a verification step of four tokens, with the input of an 8-bit projection.
        dict(_norm(4, 7168, Q_G128), name="norm_t4_d7168"),
        # The same over a chunk of prompts, with MX blocks; a width of 22.5 groups of 128.
        dict(_norm(6001, 2880, Q_MX), name="norm_t6001_d2880_mx"),
        # Plain decoding of one token of one conversation, one GPU's 16 of 128 heads.
        dict(_latent(1, 16, 1, 4097, 64, tree=False), name="latent_b1_t1_h16"),
        # The paper's operating point: four verified tokens of one sequence, all heads.
        dict(_latent(1, 128, 4, 8191, 64), name="latent_b1_t4"),
        # A batch of draft trees with ragged trees and caches.
        dict(_latent(8, 128, 16, 20011, 64), name="latent_b8_t16"),
        # A batch of plain decoding.
        dict(_latent(48, 128, 1, 6007, 16, tree=False), name="latent_b48_t1"),
        # A batch of short prompts, one GPU's 16 heads, some of them behind a cached prefix.
        dict(_prompt(6, 16, 1201, prefix=300), name="prompt_b6_h16"),
        # One long prompt, all heads.
        dict(_prompt(1, 128, 5003), name="prompt_t5003"),
        # The accepted tokens of a verification step of four sequences.
        dict(_append(4, 8, 64, 5, 9001, 64), name="append_b4_t5"),
        # The prompt of a new conversation.
        dict(_append(1, 4, 128, 15001, 0, 64), name="append_t15001"),
        # Four verified tokens of one sequence on a Qwen layer's heads.
        dict(_cache(1, 64, 4, 128, 4, 16383, 64), name="cache_b1_t4"),
        # A batch of ragged trees on a GPT-OSS layer's heads.
        dict(_cache(16, 64, 8, 64, 8, 60013, 32), name="cache_b16_t8"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _any(rng):
    kind = rng.choice(["norm", "latent", "latent", "prompt", "append", "cache", "cache"])
    if kind == "norm":
        q = rng.choice([Q_NONE, Q_G128, Q_MX, Q_ROW])
        return _norm(_log_int(rng, 1, 8000), 32 * _log_int(rng, 4, 512), q, y=q == Q_NONE or rng.random() < 0.7)
    if kind == "prompt":
        return _prompt(_log_int(rng, 1, 12), _log_int(rng, 1, 128), _log_int(rng, 1, 5000), rng.choice([0, 0, rng.randint(1, 1500)]))
    B, T = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    page = rng.choice([16, 32, 64, 128])
    if kind == "latent":
        return _latent(B, rng.choice([1, 8, 16, 20, 32, 64, 128]), T, _log_int(rng, 1, 40000), page, rng.random() < 0.6)
    D = rng.choice([64, 128])
    if kind == "append":
        return _append(B, rng.choice([1, 2, 4, 8]), D, _log_int(rng, 1, 20000), rng.choice([0, _log_int(rng, 1, 5000)]), page)
    Hkv = rng.choice([1, 2, 4, 8])
    return _cache(B, Hkv * rng.choice([1, 2, 4, 5, 8, 16]), Hkv, D, T, _log_int(rng, 1, 100000), page, rng.random() < 0.6)


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def _room(case):
    """Bytes of the largest intermediate of the plain form and of the caches."""
    if case["kind"] == "norm":
        return case["T"] * case["d"] * 4
    t, n = _lens(case)
    if case["kind"] == "prompt":
        return case["B"] * case["H"] * max(t) * max(n) * 4
    if case["kind"] == "append":
        return case["B"] * (max(t) + 2 * case["page"]) * case["Hkv"] * case["D"] * 4
    width = R + P if case["kind"] == "latent" else case["Hkv"] * case["D"]
    return case["B"] * max(n) * 4 * (max(t) * case["H"] + 2 * width)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _any(rng)
        if _room(c) < 14e9 and _cost(c) <= most and 3072 not in c.values():
            return c


# ----------------------------------------------------------------------------- lengths and inputs

def _lens(case):
    """(new tokens, cached tokens) of each sequence: the first has the most of both, the others from a spread.  For a
    prompt the second is the number of keys."""
    r = random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    T, B = case["T"], case["B"]
    t = [T] + [r.randint(max(1, T // 4), T) for _ in range(B - 1)]
    if case["kind"] == "prompt":
        p = [case["prefix"]] + [r.choice([0, r.randint(0, case["prefix"])]) for _ in range(B - 1)]
        return t, [a + b for a, b in zip(t, p)]
    L = case["L"]
    return t, [L] + [r.randint(L // 5, L) for _ in range(B - 1)]


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed << 32) | zlib.crc32(tag.encode()))
    return g


def _randn(g, *shape, std=1.0):
    return torch.empty(*shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=g)


def _offsets(t):
    o = [0]
    for n in t:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def _tree_masks(t, seed, tree):
    """One int64 a draft token: bit j set where it attends to token j of its sequence (itself and its ancestors in a
    random tree; a chain where `tree` is false)."""
    r, out = random.Random(seed), []
    for n in t:
        m = []
        for i in range(n):
            up = (r.randrange(max(0, i - 6), i) if tree else i - 1) if i else -1
            m.append((m[up] if up >= 0 else 0) | 1 << i)
        out += [v - (1 << 64) if v >> 63 else v for v in m]
    return torch.tensor(out, dtype=torch.int64, device=DEV)


def _pages(case, lens, g):
    """Pages in random order for every sequence, and a few that nobody has."""
    page = case["page"]
    need = [max(1, -(-n // page)) for n in lens]
    most, total = max(need), sum(need) + 3
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(len(lens), most, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _codes(g, *shape):
    """8-bit codes of values that fill most of a page's range."""
    out = torch.empty(*shape, dtype=torch.uint8, device=DEV)
    flat = out.view(-1)
    step = 1 << 27
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_(_randn(g, part.numel(), std=60.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def prepare(case, seed):
    kind = case["kind"]
    g = _gen(seed, kind)
    s = dict(case)
    if kind == "norm":
        T, d = case["T"], case["d"]
        s["x"] = _randn(g, T, d)
        s["residual"] = _randn(g, T, d, std=2.0)
        s["residual"][:, :: max(1, d // 7)] *= 20.0  # the few large channels of a residual stream
        s["weight"] = (1.0 + 0.2 * _randn(g, d).float()).to(torch.bfloat16)
        return s
    t, n = _lens(case)
    N = sum(t)
    s.update(N=N, most_t=max(t), most_n=max(n), offsets=_offsets(t))
    if kind == "prompt":
        H, M = case["H"], sum(n)
        s["kv_offsets"] = _offsets(n)
        s["q"] = _randn(g, N, H, DN + P, std=1.5)
        s["kv"] = _randn(g, M, H, DN + DV)  # the output of the latent's expansion: keys and values side by side
        s["k_rope"] = _randn(g, M, P)
        s["scale"] = 1.0 / math.sqrt(DN + P)
        return s
    if kind != "append":
        s["mask"] = _tree_masks(t, seed, case["tree"])
        s["cache_len"] = torch.tensor(n, dtype=torch.int32, device=DEV)
        s["table"], pages = _pages(case, n, g)
    if kind == "latent":
        H = case["H"]
        s["q"] = _randn(g, N, H, R + P, std=0.8)
        s["kv_new"] = _randn(g, N, R + P)
        s["cache"] = _randn(g, pages, case["page"], R + P)
        s["scale"] = 1.0 / math.sqrt(DN + P)
        return s
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    s["k_new"] = _randn(g, N, Hkv, D)
    s["k_new"][..., ::37] *= 6.0  # keys have a few large channels
    s["v_new"] = _randn(g, N, Hkv, D)
    if kind == "append":
        # Only the pages that the new tokens reach matter; the table's other entries share one page.
        n = [v % page for v in n]
        s["cache_len"] = torch.tensor(n, dtype=torch.int32, device=DEV)
        s["table"], pages = _pages(case, [a + b for a, b in zip(n, t)], g)
    s["k_cache"] = _codes(g, pages, Hkv, page, D)
    s["v_cache"] = _codes(g, pages, Hkv, D, page)
    s["k_scale"] = torch.exp2(torch.randint(-8, -5, (pages, Hkv), generator=g, device=DEV).float())
    s["v_scale"] = torch.exp2(torch.randint(-8, -5, (pages, Hkv), generator=g, device=DEV).float())
    if kind == "cache":
        s["q"] = _randn(g, N, case["H"], D)
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# ----------------------------------------------------------------------------- the plain forms

def _ragged(offsets, most):
    """Row of the i-th token of each sequence [B, most], and whether the sequence has one."""
    at = offsets[:-1, None].long() + torch.arange(most, device=DEV)
    has = at < offsets[1:, None]
    return at.clamp(max=offsets[-1:].long() - 1), has


def _softmax_pv(scores, seen, values):
    """Softmax over the last axis where `seen`, times values: (output, log of the sum); a row that sees nothing gives
    zeros and -inf.  A list of score, mask and value blocks that stand side by side."""
    top = None
    for i in range(len(scores)):
        scores[i].masked_fill_(~seen[i], -math.inf)
        m = scores[i].amax(-1, keepdim=True)
        top = m if top is None else torch.maximum(top, m)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    total, out = 0.0, 0.0
    for i in range(len(scores)):
        p = scores[i].sub_(base).exp_()
        total = total + p.sum(-1, keepdim=True)
        out = out + p @ values[i]
    lse = torch.where(total > 0, base + total.log(), torch.full_like(total, -math.inf))
    return out / torch.where(total > 0, total, torch.ones_like(total)), lse[..., 0]


def _bits(mask, most):
    return (mask[..., None] >> torch.arange(most, device=DEV)) & 1 > 0


def _plain_norm(s):
    v = s["x"].float() + s["residual"].float()
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    out = {"sum": v.to(torch.bfloat16)}
    if s["y"]:
        out["y"] = y.to(torch.bfloat16)
    if s["q"] == Q_NONE:
        return out
    T, d = y.shape
    width = {Q_G128: 128, Q_MX: 32, Q_ROW: d}[s["q"]]
    groups = -(-d // width)
    padded = torch.zeros(T, groups * width, device=DEV)
    padded[:, :d] = y
    padded = padded.view(T, groups, width)
    top = padded.abs().amax(-1)
    if s["q"] == Q_MX:
        e = (torch.frexp(top).exponent - 1 - 8).clamp(-127, 127)
        e = torch.where(top == 0, torch.full_like(e, -127), e).float()
        out["scales"] = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
        unit = torch.exp2(e)
    else:
        unit = top.clamp(min=2.0 ** -100) / 448.0
        out["scales"] = unit
    code = (padded / unit[..., None]).clamp(-448, 448).view(T, -1)[:, :d]
    out["q"] = code.contiguous().to(torch.float8_e4m3fn)
    return out


def _plain_latent(s):
    B, H = s["B"], s["H"]
    at, has = _ragged(s["offsets"], s["most_t"])
    T = s["most_t"]
    blocks = -(-s["most_n"] // s["page"])
    kv = s["cache"][s["table"][:, :blocks].long()].view(B, -1, R + P).float()
    new = s["kv_new"][at].float()
    q = (s["q"][at].float() * s["scale"]).view(B, T * H, R + P)
    old = q @ kv.transpose(1, 2)
    fresh = q @ new.transpose(1, 2)
    see_old = (torch.arange(kv.shape[1], device=DEV) < s["cache_len"][:, None])[:, None, :]
    see_new = _bits(s["mask"][at], T) & has[:, :, None] & has[:, None, :]
    see_new = see_new[:, :, None, :].expand(B, T, H, T).reshape(B, T * H, T)
    o, lse = _softmax_pv([old, fresh], [see_old, see_new], [kv[..., :R], new[..., :R]])
    o, lse = o.view(B, T, H, R)[has], lse.view(B, T, H)[has]
    return {"o": o.to(torch.bfloat16), "lse": lse}


def _plain_prompt(s):
    q_at, has = _ragged(s["offsets"], s["most_t"])
    k_at, kept = _ragged(s["kv_offsets"], s["most_n"])
    q = (s["q"][q_at].float() * s["scale"]).transpose(1, 2)
    kv = s["kv"][k_at].float().transpose(1, 2)
    rope = s["k_rope"][k_at].float()[:, None].expand(-1, s["H"], -1, -1)
    k = torch.cat([kv[..., :DN], rope], -1)
    scores = q @ k.transpose(2, 3)
    lens = s["offsets"][1:] - s["offsets"][:-1]
    prefix = (s["kv_offsets"][1:] - s["kv_offsets"][:-1]) - lens
    row = torch.arange(s["most_t"], device=DEV)[None] + prefix[:, None]
    seen = (torch.arange(s["most_n"], device=DEV) <= row[..., None]) & kept[:, None]
    o, lse = _softmax_pv([scores], [seen[:, None]], [kv[..., DN:]])
    return {"o": o.transpose(1, 2)[has].to(torch.bfloat16), "lse": lse.transpose(1, 2)[has]}


def _plain_append(s):
    """Every touched page is decoded, gets its new tokens, and is coded again with the larger of its scale and the
    smallest power of two that holds the new values; a page that the first token of begins has no old scale."""
    B, Hkv, D, page = s["B"], s["Hkv"], s["D"], s["page"]
    most = -(-s["most_t"] // page) + 1
    first = s["cache_len"].long() // page
    lens = (s["offsets"][1:] - s["offsets"][:-1]).long()
    blk = first[:, None] + torch.arange(most, device=DEV)
    touched = (blk * page < (s["cache_len"] + lens)[:, None]) & (lens > 0)[:, None]
    which, col = touched.nonzero(as_tuple=True)
    blk = blk[which, col]
    ids = s["table"][which, blk].long()
    pos = blk[:, None] * page + torch.arange(page, device=DEV)
    row = pos - s["cache_len"][which, None]
    new = (row >= 0) & (row < lens[which, None])
    row = (row + s["offsets"][which, None]).clamp(0, s["N"] - 1).long()
    begun = (pos[:, 0] < s["cache_len"][which])[:, None]
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        old_scale = torch.where(begun, scale[ids], torch.zeros_like(scale[ids]))
        v = s[name + "_new"][row].float().transpose(1, 2)  # [pages, Hkv, page, D]
        keep = new[:, None, :, None]
        top = (v.abs() * keep).amax((2, 3))
        f, e = torch.frexp(top)
        need = torch.exp2(torch.where(f <= 0.875, e - 9, e - 8).clamp(min=-126).float())
        need = torch.where(top == 0, torch.full_like(need, 2.0 ** -126), need)
        unit = torch.maximum(old_scale, need)
        was = cache[ids].view(torch.float8_e4m3fn).float()
        was = was.transpose(2, 3) if name == "v" else was
        kept = was * (torch.where(begun, old_scale, unit) / unit)[..., None, None]
        code = torch.where(keep, v / unit[..., None, None], kept).to(torch.float8_e4m3fn).view(torch.uint8)
        cache[ids] = code.transpose(2, 3) if name == "v" else code
        scale[ids] = unit
    return _append_outputs(s)


def _append_outputs(s):
    return {"k": s["k_cache"].view(torch.float8_e4m3fn), "v": s["v_cache"].view(torch.float8_e4m3fn),
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_cache(s):
    B, H, Hkv, D, T = s["B"], s["H"], s["Hkv"], s["D"], s["most_t"]
    G = H // Hkv
    at, has = _ragged(s["offsets"], T)
    blocks = -(-s["most_n"] // s["page"])
    ids = s["table"][:, :blocks].long()
    k = s["k_cache"].view(torch.float8_e4m3fn)[ids].float() * s["k_scale"][ids][..., None, None]
    v = s["v_cache"].view(torch.float8_e4m3fn)[ids].float() * s["v_scale"][ids][..., None, None]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, -1, D)
    q = (s["q"][at].float() * s["scale"]).view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    kn = s["k_new"][at].float().transpose(1, 2)
    vn = s["v_new"][at].float().transpose(1, 2)
    old = q @ k.transpose(2, 3)
    fresh = q @ kn.transpose(2, 3)
    see_old = (torch.arange(k.shape[2], device=DEV) < s["cache_len"][:, None])[:, None, None, :]
    see_new = _bits(s["mask"][at], T) & has[:, :, None] & has[:, None, :]
    see_new = see_new[:, None, :, None, :].expand(B, Hkv, T, G, T).reshape(B, Hkv, T * G, T)
    o, lse = _softmax_pv([old, fresh], [see_old, see_new], [v, vn])
    o = o.view(B, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, H, D)[has]
    lse = lse.view(B, Hkv, T, G).permute(0, 2, 1, 3).reshape(B, T, H)[has]
    return {"o": o.to(torch.bfloat16), "lse": lse}


# ----------------------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_2607_12696_amd as moe

    kind = s["kind"]
    if kind == "norm":
        total, y, q, scales = moe.moe_add_rmsnorm(s["x"], s["weight"], EPS, residual=s["residual"], qfmt=s["q"], want_y=s["y"])
        out = {"sum": total}
        if s["y"]:
            out["y"] = y
        if s["q"] != Q_NONE:
            out["q"] = q.view(torch.float8_e4m3fn)
            out["scales"] = scales.view(torch.float8_e8m0fnu) if s["q"] == Q_MX else scales
        return out
    if kind == "latent":
        o, lse = moe.moe_latent_attn(s["q"], s["kv_new"], s["offsets"], s["cache"], s["table"], s["cache_len"], R, s["scale"],
                                     mask=s["mask"])
        return {"o": o, "lse": lse}
    if kind == "prompt":
        o, lse = moe.moe_latent_prompt(s["q"], s["kv"][..., :DN], s["k_rope"], s["kv"][..., DN:], s["offsets"], s["kv_offsets"],
                                       s["scale"], max_tokens=s["most_t"])
        return {"o": o, "lse": lse}
    if kind == "append":
        moe.moe_cache_append(s["k_new"], s["v_new"], s["offsets"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                             s["table"], s["cache_len"], max_tokens=s["most_t"])
        return _append_outputs(s)
    o, lse = moe.moe_cache_attn(s["q"], s["k_new"], s["v_new"], s["offsets"], s["k_cache"], s["v_cache"], s["k_scale"],
                                s["v_scale"], s["table"], s["cache_len"], s["scale"], mask=s["mask"])
    return {"o": o, "lse": lse}


_PLAIN = {"norm": _plain_norm, "latent": _plain_latent, "prompt": _plain_prompt, "append": _plain_append, "cache": _plain_cache}


def run(state):
    return _own(state) if own else _PLAIN[state["kind"]](state)


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "norm":
        T, d = case["T"], case["d"]
        n = T * d
        b = n * 6 + d * 2 + (n * 2 if case["y"] else 0)
        if case["q"] != Q_NONE:
            b += n + T * {Q_G128: -(-d // 128) * 4, Q_MX: d // 32, Q_ROW: 4}[case["q"]]
        return {"bytes": b, "flops": n * 5}
    t, n = _lens(case)
    N = sum(t)
    if kind == "prompt":
        H, M = case["H"], sum(n)
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(t, n))
        return {"bytes": N * H * (DN + P + DV) * 2 + N * H * 4 + M * H * (DN + DV) * 2 + M * P * 2,
                "flops": 2 * H * pairs * (DN + P + DV)}
    if kind == "latent":
        H = case["H"]
        pairs = sum(a * (b + a) for a, b in zip(t, n))
        return {"bytes": (sum(n) + N) * (R + P) * 2 + N * H * (R + P + R) * 2 + N * H * 4,
                "flops": 2 * H * pairs * (R + P + R)}
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    if kind == "append":
        # The new tokens in and out, and of a page begun before also the codes that it keeps, in case its scale grows.
        pages = sum(-(-(b % page + a) // page) for a, b in zip(t, n))
        return {"bytes": 2 * Hkv * (N * D * 3 + sum(b % page for b in n) * D * 2 + pages * 8), "flops": 2 * Hkv * N * D * 2}
    H = case["H"]
    pairs = sum(a * (b + a) for a, b in zip(t, n))
    pages = sum(-(-b // page) for b in n)
    return {"bytes": 2 * Hkv * (sum(n) * D + N * D * 2 + pages * 4) + N * H * (4 * D + 4), "flops": 4 * H * pairs * D}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def _exact_softmax(scores, values):
    """float64 softmax of a list of score rows [.., n] (masked: -inf) times values [n, w]; rows that see nothing: zeros."""
    top = scores.max(-1).values
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = (scores - top[..., None]).exp()
    den = e.sum(-1)
    o = torch.matmul(e, values) / torch.where(den == 0, torch.ones_like(den), den)[..., None]
    return o, torch.log(den) + top


def _exact_append(case, s, t):
    """The cache after the new tokens, page by page: the values that the codes round, and the scales."""
    f64, page = torch.float64, case["page"]
    codes = {x: s[x + "_cache"].view(torch.float8_e4m3fn).to(torch.float32).to(f64) for x in "kv"}
    codes["v"] = codes["v"].transpose(2, 3).contiguous()
    units = {x: s[x + "_scale"].to(f64) for x in "kv"}
    lens, row = s["cache_len"].tolist(), 0
    for b, a in enumerate(t):
        done = 0
        while done < a:
            at = lens[b] + done
            slot, pg = at % page, int(s["table"][b, at // page])
            m = min(page - slot, a - done)
            for x in "kv":
                v = s[x + "_new"][row + done:row + done + m].to(f64).transpose(0, 1)
                unit = torch.exp2(torch.ceil(torch.log2(v.abs().amax((1, 2)) / 448)))
                if slot:
                    unit = torch.maximum(unit, units[x][pg])
                    codes[x][pg] *= (units[x][pg] / unit)[:, None, None]
                codes[x][pg, :, slot:slot + m] = v / unit[:, None, None]
                units[x][pg] = unit
            done += m
        row += a
    return {"k": codes["k"], "v": codes["v"].transpose(2, 3), "k_scale": units["k"], "v_scale": units["v"]}


def exact(case, seed):
    kind = case["kind"]
    f64 = torch.float64
    s = prepare(case, seed)
    if kind == "norm":
        v = s["x"].to(f64) + s["residual"].to(f64)
        y = v / torch.sqrt((v * v).sum(1, keepdim=True) / case["d"] + EPS) * s["weight"].to(f64)
        out = {"sum": v}
        if case["y"]:
            out["y"] = y
        if case["q"] != Q_NONE:
            # The values that the codes round, and the scales.
            parts = y.split({Q_G128: 128, Q_MX: 32, Q_ROW: case["d"]}[case["q"]], 1)
            unit = torch.stack([p.abs().max(1).values for p in parts], 1) / 448
            if case["q"] == Q_MX:
                unit = torch.exp2(torch.floor(torch.log2(unit * 448)) - 8)
            out["scales"] = unit
            out["q"] = torch.cat([(p / unit[:, i:i + 1]).clamp(-448, 448) for i, p in enumerate(parts)], 1)
        return out
    t, n = _lens(case)
    if kind == "append":
        return _exact_append(case, s, t)
    o_all, lse_all = [], []
    at, key = 0, 0
    for b, (a, m) in enumerate(zip(t, n)):
        if kind == "prompt":
            k_all = torch.cat([s["kv"][key:key + m, :, :DN].to(f64), s["k_rope"][key:key + m, None].to(f64).expand(m, case["H"], P)], 2)
            late = torch.arange(m, device=DEV)[None] > torch.arange(m - a, m, device=DEV)[:, None]
            parts = []
            for h in range(case["H"]):
                sc = torch.matmul(s["q"][at:at + a, h].to(f64), k_all[:, h].t()) * s["scale"]
                parts.append(_exact_softmax(sc.masked_fill(late, -math.inf), s["kv"][key:key + m, h, DN:].to(f64)))
            o_all.append(torch.stack([p[0] for p in parts], 1))
            lse_all.append(torch.stack([p[1] for p in parts], 1))
            at, key = at + a, key + m
            continue
        page = case["page"]
        ids = s["table"][b, :-(-m // page)].long()
        hidden = torch.tensor([[not (int(w) >> j) & 1 for j in range(a)] for w in s["mask"][at:at + a].tolist()], device=DEV)
        if kind == "latent":
            rows = torch.cat([s["cache"][ids].reshape(-1, R + P)[:m], s["kv_new"][at:at + a]]).to(f64)
            sc = torch.matmul(s["q"][at:at + a].to(f64), rows.t()) * s["scale"]  # [a, H, m + a]
            sc[:, :, m:].masked_fill_(hidden[:, None], -math.inf)
            o, lse = _exact_softmax(sc, rows[:, :R])
        else:
            G, parts = case["H"] // case["Hkv"], []
            for h in range(case["Hkv"]):
                k8, v8 = (s[x][ids, h].view(torch.float8_e4m3fn).to(torch.float32).to(f64) for x in ("k_cache", "v_cache"))
                k8 = (k8 * s["k_scale"][ids, h].to(f64)[:, None, None]).reshape(-1, case["D"])[:m]
                v8 = (v8 * s["v_scale"][ids, h].to(f64)[:, None, None]).transpose(1, 2).reshape(-1, case["D"])[:m]
                k8 = torch.cat([k8, s["k_new"][at:at + a, h].to(f64)])
                v8 = torch.cat([v8, s["v_new"][at:at + a, h].to(f64)])
                sc = torch.matmul(s["q"][at:at + a, h * G:(h + 1) * G].to(f64), k8.t()) * s["scale"]
                sc[:, :, m:].masked_fill_(hidden[:, None], -math.inf)
                parts.append(_exact_softmax(sc, v8))
            o, lse = (torch.cat([p[i] for p in parts], 1) for i in (0, 1))
        o_all.append(o)
        lse_all.append(lse)
        at += a
    return {"o": torch.cat(o_all), "lse": torch.cat(lse_all)}
