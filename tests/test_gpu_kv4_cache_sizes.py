"""A cache is taken for the sizes that it was made for; a caller's own memory by its number of bytes."""
import pytest
import torch

import paper_2402_19481_amd as df
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def test_a_cache_of_other_sizes_and_as_many_bytes():
    cache = df.kv4_cache(2, 64, 4, 64)                       # as many bytes as 4 items of 2 heads, and as half the rows of 8 heads
    x = torch.zeros(4, 64, 2, 64, dtype=torch.bfloat16, device=DEV)
    for call in (lambda: df.kv4_refresh(cache, x, x, 0, 1), lambda: df.kv4_read(cache, 4, 64, 2, 64), lambda: df.attn_kv4(x, cache, 64, 2),
                 lambda: df.attn_displaced_kv4(x[:, :32], x[:, :32], x[:, :32], cache, 0, 2), lambda: df.kv4_read(cache, 2, 128, 2, 64),
                 lambda: df.kv4_refresh_cols(cache, x, x, 8, 8, 0, 1), lambda: df.kv4_read(cache[:1], 1, 64, 4, 64), lambda: df.kv4_read(cache[:, :1], 1, 64, 4, 64)):
        with pytest.raises((ValueError, df.DfError)):
            call()


def test_memory_of_the_callers():
    B, L, h, d = 2, 70, 3, 64
    k, v = (torch.randn(B, L, h, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    made = df.kv4_cache(B, L, h, d)
    several = torch.stack([made, made])                      # one of several layers'
    own = torch.zeros(made.numel() + 256, dtype=torch.uint8, device=DEV)[256:]
    for c in (made, several[1], own):
        df.kv4_refresh(c, k, v, 0, 1)
    want = df.kv4_read(made, B, L, h, d)
    for c in (several[1], own):
        assert all(torch.equal(x, y) for x, y in zip(want, df.kv4_read(c, B, L, h, d)))
        assert torch.equal(df.attn_kv4(k, c, L, h), df.attn_kv4(k, made, L, h))
    assert not several[0].any()
