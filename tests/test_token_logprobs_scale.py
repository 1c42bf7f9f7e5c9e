"""The scale's limit, on the host: no GPU is touched."""
import pytest

import paper_2607_12696_amd as moe

FAKE = 0x10000


@pytest.mark.parametrize("scale", [2.0 ** 126 * (1 + 2.0 ** -23), 2.4e38, 3.4e38])
def test_a_scale_past_the_limit_is_refused(scale):
    at = [FAKE * n for n in range(1, 9)]
    assert moe.lib().moe_token_logprobs(at[0], 0, 100, 4, 100, scale, at[1], 2, 3, *at[2:7], 1 << 30, 1 << 40, None) == \
        moe.MOE_ERR_UNSUPPORTED
