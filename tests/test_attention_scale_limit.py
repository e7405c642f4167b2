"""The largest scale of the attention over caches and encoder states (no GPU: nothing is launched, the addresses are never read)."""
import pytest

import paper_2402_19481_amd as df

A = 1 << 20


def _cross(scale):
    return df.lib().df_cross_attn(A, 64, 64, A, 64, 64, A, 64, 64, None, None, A, 1, 1, 1, 1, 1, 64, scale, df.DF_BF16, A, 0, None)


def _cached(scale):
    return df.lib().df_attn_kv4(A, 64, 64, A, None, A, 1, 1, 1, 1, 1, 64, scale, df.DF_BF16, A, 0, None)


def _displaced(scale):
    return df.lib().df_attn_displaced_kv4(A, 64, 64, A, 64, 64, A, 64, 64, A, A, 1, 1, 1, 1, 1, 64, 0, 1, scale, df.DF_BF16, 0, A, 0, None)


@pytest.mark.parametrize("call", [_cross, _cached, _displaced])
@pytest.mark.parametrize("scale", [2.4e38, 3e38, -1.0])
def test_a_scale_whose_exponent_is_no_number(call, scale):
    """The kernels multiply by scale * log2(e): infinite above 2.35e38, and NaN for a score of 0, whose weight is 1."""
    assert call(scale) == -1
