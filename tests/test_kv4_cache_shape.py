"""A 4-bit cache as the package makes it: its shape says its sizes (no GPU)."""
import pytest

import paper_2402_19481_amd as df


@pytest.mark.parametrize("B,L,h,d", [(1, 1, 1, 64), (2, 65, 3, 64), (4, 64, 2, 128)])
def test_shape_and_bytes(B, L, h, d):
    cache = df.kv4_cache(B, L, h, d, device="cpu")
    assert tuple(cache.shape) == (d + 4, B, h, (L + 63) // 64 * 64) and cache.is_contiguous()
    assert cache.numel() == df.lib().df_kv4_bytes(B, L, h, d) and not cache.any()
