"""Refusals of the page, latent append, grouped prompt and log probability entry points, on the host: no GPU is touched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2607_12696_amd as moe
from oracle import step as ref

FAKE = 0x10000
BAD, UNS, WS, OK = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED, moe.MOE_ERR_WORKSPACE, moe.MOE_OK


def pages(N=8, keep=None, off=FAKE, new_len=FAKE + 64, n_out=FAKE + 128, refused=FAKE + 192, slots=FAKE, pos=FAKE, **c):
    f = dict(B=2, n_pages=8, page=16, max_blocks=4, block_table=FAKE, cache_len=FAKE, free_pages=FAKE, n_free=FAKE)
    f.update(c)
    p = moe.moe_page_pool_t(*(f[n] for n, _ in moe.moe_page_pool_t._fields_))
    return moe.lib().moe_pages_update(C.byref(p), keep, off, N, new_len, n_out, refused, slots, pos, None)


@pytest.mark.parametrize("change", [
    dict(B=0), dict(B=1025), dict(n_pages=0), dict(page=0), dict(page=8), dict(page=24), dict(page=256), dict(max_blocks=0),
    dict(max_blocks=1 << 27), dict(N=0), dict(N=(1 << 30) + 1), dict(block_table=None), dict(cache_len=None), dict(free_pages=None),
    dict(n_free=None), dict(off=None), dict(new_len=None), dict(n_out=None), dict(refused=None), dict(slots=FAKE + 4),
    dict(new_len=FAKE), dict(n_out=FAKE), dict(keep=FAKE + 64), dict(refused=FAKE + 128)])
def test_pages_rejects(change):
    assert pages(**change) == BAD


def append(pages=FAKE, n_pages=4, page=16, r=512, p=64, new=FAKE + 4096, n_rows=8, rows=None, N=8, slots=FAKE):
    return moe.lib().moe_latent_append(pages, n_pages, page, r, p, new, n_rows, rows, N, slots, None)


@pytest.mark.parametrize("change,status", [
    (dict(pages=None), BAD), (dict(new=None), BAD), (dict(slots=None), BAD), (dict(n_pages=0), BAD), (dict(page=48), BAD), (dict(r=0), BAD),
    (dict(p=-1), BAD), (dict(N=0), BAD), (dict(n_rows=0), BAD), (dict(n_rows=7), BAD), (dict(new=FAKE), BAD), (dict(pages=FAKE + 8), BAD),
    (dict(new=FAKE + 2), BAD), (dict(slots=FAKE + 4), BAD), (dict(r=256), UNS), (dict(p=32), UNS),
    (dict(N=(1 << 24) + 1, n_rows=1 << 25), UNS)])
def test_latent_append_rejects(change, status):
    assert append(**change) == status


def prompt(o=FAKE, ws=FAKE, size=1 << 40, lse=None, **c):
    f = dict(N=4, M=4, B=1, H=4, Hkv=2, D=64, max_tokens=4, q_offsets=FAKE, kv_offsets=FAKE, q=FAKE + 64, k=FAKE + 128, v=FAKE + 192,
             q_stride=256, q_head=64, k_stride=128, k_head=64, v_stride=128, v_head=64, scale=1.0)
    f.update(c)
    a = moe.moe_grouped_prompt_t(*(f[n] for n, _ in moe.moe_grouped_prompt_t._fields_))
    return moe.lib().moe_grouped_prompt(C.byref(a), o, lse, ws, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(N=0), BAD), (dict(M=0), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(H=0), BAD), (dict(H=1026), BAD), (dict(Hkv=0), BAD),
    (dict(H=5), BAD), (dict(H=514, Hkv=257), BAD), (dict(D=0), BAD), (dict(D=96), UNS), (dict(D=256), UNS), (dict(max_tokens=0), BAD),
    (dict(q_offsets=None), BAD), (dict(kv_offsets=None), BAD), (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD),
    (dict(o=None), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 16), BAD), (dict(size=0), WS), (dict(lse=FAKE + 2), BAD),
    (dict(q_stride=4), BAD), (dict(q_head=-8), BAD), (dict(k_stride=12), BAD), (dict(v_head=2), BAD), (dict(scale=math.nan), BAD),
    (dict(scale=math.inf), BAD), (dict(k=FAKE + 8), BAD), (dict(o=FAKE + 64), BAD), (dict(o=FAKE + 128), BAD), (dict(o=FAKE + 192), BAD),
    (dict(k_stride=1 << 24), UNS), (dict(v_stride=1 << 24), UNS), (dict(N=1 << 29, max_tokens=1), UNS),
    (dict(N=1 << 20, B=1024, max_tokens=1 << 20), UNS)])
def test_grouped_prompt_rejects(change, status):
    assert prompt(**change) == status


def test_grouped_prompt_workspace():
    n, L = C.c_size_t(), moe.lib()
    for D in (64, 128):
        assert L.moe_grouped_prompt_workspace_size(D, C.byref(n)) == OK and n.value > 0
        assert prompt(D=D, size=n.value - 1) == WS
    assert L.moe_grouped_prompt_workspace_size(64, None) == BAD
    assert L.moe_grouped_prompt_workspace_size(0, C.byref(n)) == BAD
    assert L.moe_grouped_prompt_workspace_size(80, C.byref(n)) == UNS


def logprobs(logits=FAKE, dtype=0, stride=100, N=4, V=100, scale=1.0, tokens=FAKE, M=2, k=3, lp=FAKE, lse=FAKE, ent=FAKE, idx=FAKE, top=FAKE,
             ws=FAKE, size=1 << 40):
    return moe.lib().moe_token_logprobs(logits, dtype, stride, N, V, scale, tokens, M, k, lp, lse, ent, idx, top, ws, size, None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(ws=None), dict(ws=FAKE + 128), dict(N=0), dict(N=(1 << 22) + 1), dict(V=0), dict(V=(1 << 24) + 1, stride=1 << 30),
    dict(stride=99), dict(stride=0), dict(dtype=2), dict(dtype=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
    dict(scale=math.inf), dict(k=-1), dict(k=65), dict(V=2, stride=2), dict(M=-1), dict(M=0), dict(M=0, tokens=None), dict(M=0, lp=None),
    dict(tokens=None), dict(lp=None), dict(M=65537), dict(N=1 << 20, M=1 << 11), dict(idx=None), dict(k=0), dict(k=0, idx=None),
    dict(k=0, top=None), dict(M=0, tokens=None, lp=None, k=0, idx=None, top=None, lse=None, ent=None), dict(logits=FAKE + 2),
    dict(dtype=1, logits=FAKE + 1)])
def test_logprobs_rejects(change):
    assert logprobs(**change) == BAD


def test_logprobs_workspace_serves_fewer_rows():
    n, last = C.c_size_t(), 0
    for N in (1, 2, 3, 5, 17, 64, 100, 1000, 4095, 4096, 4097, 70000):
        assert moe.lib().moe_token_logprobs_workspace_size(N, C.byref(n)) == OK
        assert n.value >= last
        last = n.value
        assert logprobs(N=N, size=n.value - 1) == WS
    assert moe.lib().moe_token_logprobs_workspace_size(0, C.byref(n)) == BAD
    assert moe.lib().moe_token_logprobs_workspace_size(4, None) == BAD


@pytest.mark.parametrize("change", [
    dict(new_len=0x10004), dict(new_len=0x20004), dict(new_len=0x30004), dict(n_out=0x40000), dict(refused=0x50004),
    dict(slots=0x60000 - 8), dict(pos=0x70000 - 4 * 7), dict(block_table=0x10000), dict(free_pages=0x60000 - 4 * 7),
    dict(pos=0x50008 - 32), dict(refused=0x10000), dict(free_pages=0x60004)])
def test_pages_rejects_overlaps(change):
    """Two sequences, four blocks each, eight pages and tokens: a buffer moved so that its first or last element is another's."""
    at = dict(cache_len=0x10000, keep=0x20000, off=0x30000, n_free=0x40000, new_len=0x50000, n_out=0x50008, refused=0x5000c,
              block_table=0x60000, free_pages=0x70000, slots=0x80000, pos=0x90000)
    at.update(change)
    assert pages(**at) == BAD


@pytest.mark.parametrize("change", [dict(new=FAKE + 4 * 16 * 1152 - 16), dict(new=FAKE - 8 * 1152 + 16), dict(rows=FAKE + 8),
                                    dict(slots=FAKE - 56)])
def test_latent_append_rejects_overlaps(change):
    at = dict(new=FAKE << 8, slots=FAKE << 4)
    at.update(change)
    assert append(**at) == BAD


@pytest.mark.parametrize("change", [
    dict(o=0x20000 + 2 * (3 * 256 + 3 * 64 + 56)), dict(o=0x20000 - 2 * (4 * 4 * 64 - 8)), dict(o=0x30000 + 2 * (3 * 128 + 64 + 56)),
    dict(o=0x40000 + 64), dict(lse=0x20000 + 16), dict(lse=0x10000 + 16), dict(lse=0x50004), dict(ws=0x20000), dict(ws=0x10000 + 256),
    dict(lse=0x1000004)])
def test_grouped_prompt_rejects_overlaps(change):
    at = dict(o=0x10000, q=0x20000, k=0x30000, v=0x40000, q_offsets=0x50000, kv_offsets=0x60000, ws=0x1000000)
    at.update(change)
    assert prompt(**at) == BAD


@pytest.mark.parametrize("change", [
    dict(lp=0x10000 + 4 * (3 * 100 + 99)), dict(lse=0x10000 - 12), dict(ent=0x20000 + 28), dict(idx=0x40000 + 12), dict(top=0x60000 + 44),
    dict(top=0x10000), dict(ws=0x10000), dict(lse=0x1000010), dict(lp=0x20000)])
def test_logprobs_rejects_overlaps(change):
    at = dict(logits=0x10000, tokens=0x20000, lp=0x30000, lse=0x40000, ent=0x50000, idx=0x60000, top=0x70000, ws=0x1000000)
    at.update(change)
    assert logprobs(**at) == BAD


def test_binding_refuses_wrong_tensors():
    """The Python entry points check types and shapes before the library is called; none of these is on the device."""
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: moe.moe_pages_update(i[:2], i[:3], i.view(2, 2), i, i[:1], 16, 4),
                 lambda: moe.moe_pages_update(i[:2].long(), i[:3], i.view(2, 2), i, i[:1], 16, 4),
                 lambda: moe.moe_latent_append(torch.zeros(3, 576), torch.zeros(2, 16, 576), i),
                 lambda: moe.moe_latent_append(torch.zeros(3, 576), torch.zeros(2, 16, 576), i.long()),
                 lambda: moe.moe_grouped_prompt(x, x[:, :2], x[:, :2], i[:2], i[:2], 1.0),
                 lambda: moe.moe_token_logprobs(x[0], i),
                 lambda: moe.moe_token_logprobs(x, i),
                 lambda: moe.moe_token_logprobs(x[0].half(), i),
                 lambda: moe.moe_token_logprobs(x[0].t(), i)):
        with pytest.raises(ValueError):
            call()


class OnDevice:
    """Stands for a tensor of some device where there is none."""

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_binding_refuses_tensors_of_several_devices():
    moe._one_device(OnDevice(1), OnDevice(1), None, OnDevice(1))
    with pytest.raises(ValueError):
        moe._one_device(OnDevice(1), None, OnDevice(1), OnDevice(0))


@pytest.mark.parametrize("stream,current,entered", [(0, 0, []), (0, 1, [0]), (5, 0, []), (5, 1, [])])
def test_a_default_stream_makes_its_device_the_current_one(monkeypatch, stream, current, entered):
    calls, devices = [], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            devices.append(self.device)

        def __exit__(self, *_):
            devices.append("left")

    monkeypatch.setattr(moe, "_stream", lambda t: stream)
    monkeypatch.setattr(moe, "_several_devices", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    monkeypatch.setattr(torch.cuda, "device", Device)

    def fn(*args):
        calls.append((args, list(devices)))
        return OK

    moe._enqueue("fn", fn, OnDevice(0), 7, 8)
    assert calls == [((7, 8, stream), entered)] and devices == entered + ["left"] * len(entered)


# ----------------------------------------------------------------------------- the oracle's own pins

def test_oracle_pages():
    table, free = [[5, 6, 0], [7, 8, 9], [1, 0, 0]], [2, 3]
    got = ref.pages([20, 40, 16], [20, 0, 16], [13, 5, 17], table, free, 16)
    # Sequence 1 returns 8 and 9; sequence 0 takes a third page, sequence 2 two more.
    assert got[0] == [33, 5, 33] and got[1] == 0
    assert table == [[5, 6, 9], [7, 8, 9], [1, 8, 3]] and free == [2]
    assert got[2][0] == (6 * 16 + 4, 20) and got[2][12] == (9 * 16, 32) and got[2][13] == (7 * 16, 0) and got[2][-1] == (3 * 16, 32)
    table, free = [[5, 0, 0], [6, 0, 0], [7, 0, 0], [4, 0, 0]], [2, 3]
    got = ref.pages([16] * 4, [16] * 4, [1, 33, 17, 0], table, free, 16)  # 1 is past the table, 2 past the pages
    assert got[0] == [17, 16, 16, 16] and got[1] == 2 and free == [2] and table[0][:2] == [5, 3]


def test_oracle_logprobs():
    x = np.array([1.0, 3.0, 3.0, -np.inf, 0.0, -0.0, np.nan])
    assert ref.order(x).tolist() == [1, 2, 0, 4, 5, 3, 6]
    r = ref.logprobs(x[:6], 2.0)
    t = torch.from_numpy(x[:6]) * 2
    want = torch.log_softmax(t, 0).numpy()
    fin = np.isfinite(want)
    assert abs(r.lse - float(torch.logsumexp(t, 0))) < 1e-12 and np.allclose(r.p[fin], want[fin], atol=1e-12) and r.p[3] == -np.inf
    assert abs(r.entropy + (np.exp(want[fin]) * want[fin]).sum()) < 1e-12
    assert math.isnan(ref.logprobs(x, 1.0).lse) and ref.logprobs(x[3:4], 1.0).lse == -math.inf
