"""Sizes of 4-bit caches whose bytes 64 bits do not count (no GPU: nothing is launched, the addresses are never read)."""
import pytest

import paper_2402_19481_amd as df


@pytest.mark.parametrize("B,L,h,d", [(32768, 1 << 28, 32768, 128), (65535, (1 << 30) - 64, 65535, 128), (65535, (1 << 30) - 64, 65535, 64),
                                     (1 << 15, 1 << 29, 1 << 15, 64)])
def test_sizes_beyond_64_bits_are_not_taken(B, L, h, d):
    lib, A = df.lib(), 1 << 20
    assert lib.df_kv4_bytes(B, L, h, d) == 0
    assert lib.df_kv4_refresh(A, A, h * d, 0, A, h * d, 0, B, 1, L, h, d, 0, L, df.DF_BF16, 0, None) == -2
    assert lib.df_kv4_read(A, A, A, B, L, h, d, df.DF_BF16, None) == -2
    assert lib.df_attn_kv4(A, h * d, h * d, A, None, A, B, 1, L, h, h, d, 0.1, df.DF_BF16, A, 1 << 60, None) == -2
    assert lib.df_attn_kv4_workspace_bytes(B, 1, L, h, h, d, df.DF_BF16) == 0
    with pytest.raises(df.DfError):
        df.kv4_cache(B, L, h, d, device="cpu")


def test_large_caches_are_taken():
    assert df.lib().df_kv4_bytes(16, 1 << 20, 64, 128) == 16 * 64 * (1 << 20) * 132
