"""Refusals of the 8-bit cache's append by slots, on the host: no GPU is touched."""
import ctypes as C

import pytest
import torch

import paper_2607_12696_amd as moe

FAKE = 0x10000
BAD, UNS = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED


def append(k_new=FAKE, v_new=FAKE, n_rows=4, rows=None, N=4, B=2, off=FAKE, most=4, slots=FAKE, **c):
    f = dict(Hkv=4, D=128, n_pages=8, page=64, max_blocks=4, k=FAKE, v=FAKE + 1024, k_scale=FAKE, v_scale=FAKE, block_table=FAKE,
             cache_len=FAKE)
    f.update(c)
    cache = moe.moe_cache_t(*(f[n] for n, _ in moe.moe_cache_t._fields_))
    return moe.lib().moe_cache_append_slots(C.byref(cache), k_new, v_new, n_rows, rows, N, B, off, most, slots, None)


@pytest.mark.parametrize("change,status", [
    (dict(slots=None), BAD), (dict(slots=FAKE + 4), BAD), (dict(k_new=None), BAD), (dict(v_new=None), BAD), (dict(off=None), BAD),
    (dict(N=0), BAD), (dict(n_rows=0), BAD), (dict(n_rows=3), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(most=0), BAD),
    (dict(k_new=FAKE + 4), BAD), (dict(v_new=FAKE + 8), BAD), (dict(k=None), BAD), (dict(v=FAKE), BAD), (dict(Hkv=0), BAD),
    (dict(page=24), BAD), (dict(n_pages=0), BAD), (dict(D=96), UNS), (dict(N=1 << 30, n_rows=1 << 30, most=1 << 30), UNS)])
def test_rejects(change, status):
    assert append(**change) == status


def test_binding_refuses_wrong_slots():
    """None of these is on the device, and the slots' type and length are checked before the library is called."""
    kv, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    k, v, s = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 64, 16, dtype=torch.uint8), torch.zeros(4, 2)
    for slots in (i, i.long(), i.long()[:2]):
        with pytest.raises(ValueError):
            moe.moe_cache_append(kv, kv, i, k, v, s, s, i[:2].view(2, 1), i[:2], slots=slots)
