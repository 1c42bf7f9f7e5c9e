"""Limits of the attention entry points that can be seen on the host: no GPU is touched."""
import ctypes as C

import pytest

import paper_2607_12696_amd as moe

FAKE = 0x10000
BAD, OK = moe.MOE_ERR_INVALID_ARG, moe.MOE_OK
LATENT = moe.moe_latent_cache_t(512, 64, 8, 64, 4, FAKE, FAKE, FAKE)
GROUPED = moe.moe_cache_t(4, 128, 8, 64, 4, FAKE, FAKE + 1024, FAKE, FAKE, FAKE, FAKE)


def size(kind, N, B, H=16, cache=None):
    """(status, bytes) of the workspace query."""
    n, L = C.c_size_t(), moe.lib()
    f = L.moe_latent_attn_workspace_size if kind == "latent" else L.moe_cache_attn_workspace_size
    cache = cache or (LATENT if kind == "latent" else GROUPED)
    return f(C.byref(cache), N, B, H, C.byref(n)), n.value


def attend(kind, N, B, H=16):
    d, L = moe.moe_drafts_t(N, B, FAKE, None), moe.lib()
    if kind == "latent":
        return L.moe_latent_attn(C.byref(LATENT), C.byref(d), FAKE, FAKE, H, 1.0, FAKE + 256, None, FAKE, 1 << 40, None)
    return L.moe_cache_attn(C.byref(GROUPED), C.byref(d), FAKE, FAKE, FAKE, H, 1.0, FAKE + 256, None, FAKE, 1 << 40, None)


@pytest.mark.parametrize("kind", ["latent", "grouped"])
@pytest.mark.parametrize("N,B", [(65, 1), (1000, 1), (129, 2), (64 * 7 + 1, 7)])
def test_more_tokens_than_masks_have_bits(kind, N, B):
    """A token's mask has 64 bits, so B sequences have at most 64 B tokens: with more, some would not see themselves."""
    assert size(kind, N, B)[0] == BAD
    assert attend(kind, N, B) == BAD
    assert size(kind, 64 * B, B)[0] == OK


@pytest.mark.parametrize("H", [1, 5, 16, 33, 64, 128])
@pytest.mark.parametrize("kind,shape", [("latent", 4), ("latent", 4000), ("grouped", 64), ("grouped", 128)])
def test_workspace_of_the_largest_call_is_enough_for_smaller_ones(kind, shape, H):
    """The size asked for the most tokens and sequences bounds that of every call with no more of either."""
    if kind == "latent":
        c = moe.moe_latent_cache_t(512, 64, 8, 64, shape, FAKE, FAKE, FAKE)
    else:
        c = moe.moe_cache_t(1, shape, 8, 64, 4, FAKE, FAKE + 1024, FAKE, FAKE, FAKE, FAKE)
    steps = [1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 64, 100, 150, 300, 600, 1000]
    sizes = {}
    for N in steps:
        for B in steps:
            if N > 64 * B:
                continue
            status, sizes[N, B] = size(kind, N, B, H, c)
            assert status == OK
    for (N, B), n in sizes.items():
        for (N2, B2), m in sizes.items():
            assert N2 > N or B2 > B or m <= n, ((N2, B2, m), (N, B, n))
