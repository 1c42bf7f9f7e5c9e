"""The log probabilities' workspace, on the host: no GPU is touched."""
import ctypes as C

import pytest

import paper_2607_12696_amd as moe

FAKE = 0x10000


@pytest.mark.parametrize("N", [512, 4097, 150000, 1 << 22])
def test_many_rows_ask_for_no_more_than_few(N):
    """Only parts of few rows leave anything between two kernels: at most 4096, of 16 bytes and 64 entries each."""
    n = C.c_size_t()
    assert moe.lib().moe_token_logprobs_workspace_size(N, C.byref(n)) == moe.MOE_OK
    assert n.value <= 4096 * (16 + 64 * 8)
    assert n.value == moe.moe_token_logprobs_workspace_size(1)
