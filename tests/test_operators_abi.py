"""Refusals of the norm, attention and cache entry points, on the host: no GPU is touched."""
import ctypes as C

import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import attention as ref

FAKE = 0x10000
BAD, UNS, WS, OK = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED, moe.MOE_ERR_WORKSPACE, moe.MOE_OK


def norm(x=FAKE, r=FAKE, w=FAKE, T=4, d=256, eps=1e-6, fmt=0, total=FAKE + 64, y=FAKE + 128, q=None, s=None):
    return moe.lib().moe_add_rmsnorm(x, r, w, T, d, eps, fmt, total, y, q, s, None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), BAD), (dict(w=None), BAD), (dict(T=0), BAD), (dict(d=0), BAD), (dict(d=48), UNS), (dict(d=16416), UNS),
    (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD), (dict(fmt=4), BAD), (dict(fmt=-1), BAD),
    (dict(fmt=1), BAD), (dict(fmt=1, q=FAKE), BAD), (dict(q=FAKE, s=FAKE), BAD), (dict(total=None, y=None), BAD),
    (dict(x=FAKE + 8), BAD), (dict(y=FAKE + 2), BAD), (dict(y=FAKE, r=FAKE), BAD), (dict(y=FAKE + 64), BAD),
    (dict(fmt=1, q=FAKE, s=FAKE + 4), BAD), (dict(fmt=1, q=FAKE + 256, s=FAKE + 2), BAD)])
def test_norm_rejects(change, status):
    assert norm(**change) == status


def latent_cache(**c):
    f = dict(r=512, p=64, n_pages=8, page=64, max_blocks=4, pages=FAKE, block_table=FAKE, cache_len=FAKE)
    f.update(c)
    return moe.moe_latent_cache_t(*(f[n] for n, _ in moe.moe_latent_cache_t._fields_))


def latent(cache=None, N=4, B=2, H=16, off=FAKE, q=FAKE, new=FAKE, o=FAKE + 256, scale=1.0, ws=FAKE, size=1 << 40):
    c, d = cache or latent_cache(), moe.moe_drafts_t(N, B, off, None)
    return moe.lib().moe_latent_attn(C.byref(c), C.byref(d), q, new, H, scale, o, None, ws, size, None)


CALLS = [dict(N=0), dict(B=0), dict(B=1025), dict(H=0), dict(H=1025), dict(N=1 << 22), dict(off=None), dict(q=None), dict(o=None),
         dict(ws=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=FAKE + 8), dict(o=FAKE + 2), dict(ws=FAKE + 16),
         dict(o=FAKE)]
PAGES = [(dict(n_pages=0), BAD), (dict(page=0), BAD), (dict(page=48), BAD), (dict(page=256), BAD), (dict(max_blocks=0), BAD),
         (dict(max_blocks=1 << 30), BAD), (dict(block_table=None), BAD), (dict(cache_len=None), BAD)]


@pytest.mark.parametrize("change", CALLS + [dict(new=None), dict(new=FAKE + 4)])
def test_latent_rejects_calls(change):
    assert latent(**change) == BAD


@pytest.mark.parametrize("change,status", PAGES + [(dict(pages=None), BAD), (dict(pages=FAKE + 8), BAD), (dict(r=0), BAD), (dict(r=256), UNS),
                                                   (dict(p=32), UNS)])
def test_latent_rejects_caches(change, status):
    assert latent(cache=latent_cache(**change)) == status
    n, c = C.c_size_t(), latent_cache(**change)
    assert moe.lib().moe_latent_attn_workspace_size(C.byref(c), 4, 2, 16, C.byref(n)) == status


def cache(**c):
    f = dict(Hkv=4, D=128, n_pages=8, page=64, max_blocks=4, k=FAKE, v=FAKE + 1024, k_scale=FAKE, v_scale=FAKE, block_table=FAKE,
             cache_len=FAKE)
    f.update(c)
    return moe.moe_cache_t(*(f[n] for n, _ in moe.moe_cache_t._fields_))


def attn(c=None, N=4, B=2, H=16, off=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE + 256, scale=1.0, ws=FAKE, size=1 << 40):
    c, d = c or cache(), moe.moe_drafts_t(N, B, off, None)
    return moe.lib().moe_cache_attn(C.byref(c), C.byref(d), q, k, v, H, scale, o, None, ws, size, None)


def append(c=None, k=FAKE, v=FAKE, n_rows=4, rows=None, N=4, B=2, off=FAKE, most=4):
    c = c or cache()
    return moe.lib().moe_cache_append(C.byref(c), k, v, n_rows, rows, N, B, off, most, None)


HEADS = [(dict(Hkv=0), BAD), (dict(Hkv=257), BAD), (dict(D=0), BAD), (dict(D=96), UNS), (dict(k=None), BAD), (dict(v=None), BAD),
         (dict(k_scale=None), BAD), (dict(v_scale=None), BAD), (dict(k=FAKE + 8), BAD), (dict(v=FAKE), BAD)]


@pytest.mark.parametrize("change", CALLS + [dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(H=18)])
def test_cache_attn_rejects_calls(change):
    assert attn(**change) == BAD


@pytest.mark.parametrize("change,status", PAGES + HEADS)
def test_cache_rejects_caches(change, status):
    assert attn(cache(**change)) == status
    assert append(cache(**change)) == status
    n, c = C.c_size_t(), cache(**change)
    assert moe.lib().moe_cache_attn_workspace_size(C.byref(c), 4, 2, 1028, C.byref(n)) == (BAD if status == BAD else status)


@pytest.mark.parametrize("change", [dict(k=None), dict(v=None), dict(off=None), dict(N=0), dict(n_rows=0), dict(n_rows=3), dict(B=0),
                                    dict(B=1025), dict(most=0), dict(k=FAKE + 4), dict(v=FAKE + 8)])
def test_append_rejects(change):
    assert append(**change) == BAD


def prompt(o=FAKE, **c):
    f = dict(N=4, M=4, B=1, H=2, dn=128, p=64, dv=128, max_tokens=4, q_offsets=FAKE, kv_offsets=FAKE, q=FAKE + 64, k=FAKE, k_rope=FAKE,
             v=FAKE, k_stride=512, k_head=256, v_stride=512, v_head=256, scale=1.0)
    f.update(c)
    a = moe.moe_prompt_t(*(f[n] for n, _ in moe.moe_prompt_t._fields_))
    return moe.lib().moe_latent_prompt(C.byref(a), o, None, None)


@pytest.mark.parametrize("change,status", [
    (dict(N=0), BAD), (dict(M=0), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(H=0), BAD), (dict(H=1025), BAD), (dict(dn=0), BAD),
    (dict(dn=64), UNS), (dict(p=32), UNS), (dict(dv=64), UNS), (dict(max_tokens=0), BAD), (dict(q_offsets=None), BAD),
    (dict(kv_offsets=None), BAD), (dict(q=None), BAD), (dict(k=None), BAD), (dict(k_rope=None), BAD), (dict(v=None), BAD),
    (dict(k_stride=4), BAD), (dict(v_head=12), BAD), (dict(k_head=-8), BAD), (dict(scale=float("nan")), BAD), (dict(k=FAKE + 8), BAD),
    (dict(o=None), BAD), (dict(o=FAKE + 64), BAD)])
def test_prompt_rejects(change, status):
    assert prompt(**change) == status


def test_launches_that_do_not_fit():
    """Sizes past what one launch or 32-bit offsets reach are refused, not cut."""
    assert norm(T=(1 << 21) + 1) == UNS
    big = dict(N=1 << 30, n_rows=1 << 30, most=1 << 30)
    assert append(cache(Hkv=256, D=128, page=16), **big) == UNS
    assert append(cache(Hkv=256, D=64, page=128), **big) == UNS
    assert prompt(k_stride=1 << 24) == UNS and prompt(v_stride=1 << 24) == UNS
    assert prompt(N=1 << 29, H=8, max_tokens=1) == UNS
    assert prompt(N=1 << 20, B=1024, H=8, max_tokens=1 << 20) == UNS


def test_short_workspaces():
    n, c = C.c_size_t(), latent_cache()
    assert moe.lib().moe_latent_attn_workspace_size(C.byref(c), 4, 2, 16, C.byref(n)) == OK and n.value > 0
    assert latent(size=n.value - 1) == WS
    c = cache()
    assert moe.lib().moe_cache_attn_workspace_size(C.byref(c), 4, 2, 16, C.byref(n)) == OK and n.value > 0
    assert attn(size=n.value - 1) == WS


def test_binding_refuses_wrong_tensors():
    """The Python entry points check types and shapes before the library is called."""
    f, h = torch.zeros(2, 64), torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        moe.moe_add_rmsnorm(f, h[0], 1e-6)
    with pytest.raises(ValueError):
        moe.moe_add_rmsnorm(h, h[0, :32], 1e-6)
    with pytest.raises(ValueError):
        moe.moe_add_rmsnorm(h, h[0], 1e-6)  # not on the device
    off, q = torch.zeros(2, dtype=torch.int32), torch.zeros(3, 4, 576, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        moe.moe_latent_attn(q, q[:, 0], off, torch.zeros(2, 16, 576, dtype=torch.bfloat16), off[None], off[:1], 512, 1.0,
                            mask=torch.zeros(3))
    with pytest.raises(ValueError):
        moe.moe_latent_prompt(q[..., :192], q[..., :128], q[:, 0, :64], q[..., :128], off, off, 1.0)


def test_oracle_e4m3_and_scales():
    """The oracle's own pins: codes against torch's conversion, power-of-two scales at their edges."""
    v = torch.linspace(-448, 448, 70001, dtype=torch.float32)
    assert (torch.from_numpy(ref.e4m3(v.numpy())) == v.to(torch.float8_e4m3fn).view(torch.uint8)).all()
    assert [ref.power_scale(x) for x in (448.0, 448.1, 224.0, 1.75, 1.76, 0.0, 1e-44)] == [1.0, 2.0, 0.5, 2.0 ** -8, 2.0 ** -7, 2.0 ** -126,
                                                                                      2.0 ** -126]
