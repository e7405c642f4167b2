"""Keys and values held in 4 bits: refresh and read bit for bit, attention over them against the 64-bit form (bounds derived there)."""
import numpy as np
import pytest
import torch

import paper_2402_19481_amd as df
from oracle import block_ops as bo
from gpu_util import DEV, host

pytestmark = pytest.mark.gpu
TYPES = {True: torch.bfloat16, False: torch.float32}


def _rows(seed, *shape, bf16=True, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(TYPES[bf16]).to(DEV)


def _own(H, W, patch, N, cols):
    j = np.arange(H * W)
    return np.flatnonzero((j % W) // (W // N) == patch) if cols else j[patch * (H * W // N):(patch + 1) * (H * W // N)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,L,h,d", [(1, 1, 1, 64), (2, 63, 3, 64), (1, 64, 2, 128), (1, 65, 1, 128), (2, 300, 5, 64)])
def test_held_exactly(B, L, h, d, bf16):
    print("kv4", B, L, h, d, bf16, flush=True)
    k, v = _rows(L, B, L, h, d, bf16=bf16), _rows(L + 1, B, L, h, d, bf16=bf16)
    k[0, 0, 0] = torch.tensor([6, 0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5] * (d // 8), device=DEV).to(k.dtype)    # every tie
    v[0, -1, 0, :9] = torch.tensor([3e38, 1e38, -3e38, 1, 0, 2e38, -1e37, 6e37, 1e-38], device=DEV).to(v.dtype)
    v[-1, 0, -1] = 1e-31 * torch.arange(d, device=DEV)
    cache = df.kv4_cache(B, L, h, d)
    assert df.kv4_refresh(cache, k, v, 0, 1) is cache
    for dt in (torch.bfloat16, torch.float32):
        gk, gv = df.kv4_read(cache, B, L, h, d, dtype=dt)
        assert gk.dtype == dt and np.array_equal(host(gk), bo.held_in_4_bits(host(k))) and np.array_equal(host(gv), bo.held_in_4_bits(host(v)))


def test_rows_without_a_number():
    k, v = _rows(1, 1, 5, 1, 64), _rows(2, 1, 5, 1, 64)
    k[0, 1, 0, 3], v[0, 2, 0, 63], v[0, 4] = float("nan"), float("-inf"), 0.0
    cache = df.kv4_cache(1, 5, 1, 64)
    df.kv4_refresh(cache, k, v, 0, 1)
    gk, gv = df.kv4_read(cache, 1, 5, 1, 64)
    np.testing.assert_array_equal(host(gk), bo.held_in_4_bits(host(k)))
    np.testing.assert_array_equal(host(gv), bo.held_in_4_bits(host(v)))


@pytest.mark.parametrize("H,W,N,cols", [(1, 130, 2, False), (5, 13, 5, False), (1, 70, 70, False), (6, 15, 3, True), (9, 28, 4, True), (3, 200, 2, True)])
def test_a_patch_leaves_the_other_rows(H, W, N, cols):
    B, h, d = 2, 2, 64
    L = H * W
    k, v = _rows(5, B, L, h, d), _rows(6, B, L, h, d)
    cache = df.kv4_cache(B, L, h, d)
    df.kv4_refresh(cache, k, v, 0, 1)
    k, v = host(k), host(v)
    for patch in {0, N // 2, N - 1}:
        own = _own(H, W, patch, N, cols)
        fused = _rows(7 + patch, B, len(own), 2 * h * d, std=2.0)                      # one projection gives both
        fk, fv = fused[..., :h * d].unflatten(-1, (h, d)), fused[..., h * d:].unflatten(-1, (h, d))
        if cols:
            df.kv4_refresh_cols(cache, fk, fv, H, W, patch, N)
        else:
            df.kv4_refresh(cache, fk, fv, patch, N)
        k[:, own], v[:, own] = host(fk), host(fv)
        gk, gv = df.kv4_read(cache, B, L, h, d)
        assert np.array_equal(host(gk), bo.held_in_4_bits(k)) and np.array_equal(host(gv), bo.held_in_4_bits(v)), patch


def _check(got, q, k, v, bf16, valid=None, scale=None):
    d = q.shape[-1]
    ref, size, reach = bo.attention(host(q), k, v, d ** -0.5 if scale is None else scale, valid)
    off = np.abs(host(got) - ref)
    bound = bo.attention_bound(ref, size, reach, d, k.shape[1], bf16)
    assert (off <= bound).all(), (np.argwhere(~(off <= bound))[:4], off.max(), float((off / bound).max()))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,Lq,L,heads,kv,d", [
    (1, 1, 1, 1, 1, 64), (1, 1, 64, 2, 2, 64), (2, 1, 777, 8, 2, 64), (1, 3, 130, 4, 4, 128), (1, 16, 1000, 2, 2, 64), (2, 5, 333, 12, 3, 128),
    (1, 33, 65, 2, 1, 64), (1, 64, 260, 1, 1, 64), (1, 65, 200, 2, 2, 64), (2, 100, 511, 4, 2, 128), (1, 300, 70, 3, 3, 64), (1, 1, 9000, 1, 1, 64),
    (2, 200, 900, 8, 4, 64), (2, 1300, 1600, 4, 4, 64), (1, 700, 1500, 8, 4, 128),
])
def test_cached_attention(B, Lq, L, heads, kv, d, bf16):
    print("attn_kv4", B, Lq, L, heads, kv, d, bf16, flush=True)
    k, v, q = _rows(1, B, L, kv, d, bf16=bf16), _rows(2, B, L, kv, d, bf16=bf16), _rows(3, B, Lq, heads, d, bf16=bf16, std=1.5)
    cache = df.kv4_cache(B, L, kv, d)
    df.kv4_refresh(cache, k, v, 0, 1)
    hk, hv = bo.held_in_4_bits(host(k)), bo.held_in_4_bits(host(v))
    _check(df.attn_kv4(q, cache, L, kv), q, hk, hv, bf16)
    _check(df.attn_kv4(q, cache, L, kv, scale=2.0), q, hk, hv, bf16, scale=2.0)      # peaked: the running maximum moves
    # lengths; the rows behind hold no numbers, one item has none
    lens = torch.tensor([(L + 1) // 2, 0][:B] if L < 500 else [L - 65, 0][:B], dtype=torch.int32)
    valid = np.arange(L)[None] < lens.numpy()[:, None]
    k[~torch.from_numpy(valid).to(DEV)] = float("nan")
    v[~torch.from_numpy(valid).to(DEV)] = float("inf")
    df.kv4_refresh(cache, k, v, 0, 1)
    got = df.attn_kv4(q, cache, L, kv, lens=lens.to(DEV))
    _check(got, q, hk, hv, bf16, valid)
    assert B == 1 or not got[1].any()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,H,W,N,cols,heads,kv,d", [
    (1, 1, 64, 1, False, 2, 2, 64), (1, 4, 30, 2, False, 2, 2, 64), (2, 6, 50, 3, False, 4, 2, 64), (1, 8, 40, 8, False, 3, 3, 128), (1, 7, 36, 4, True, 2, 2, 64),
    (2, 10, 33, 3, True, 2, 1, 128), (1, 1, 16, 16, False, 2, 2, 64), (1, 20, 60, 2, True, 1, 1, 64),
    (1, 30, 100, 2, False, 4, 4, 64), (1, 30, 100, 2, True, 6, 3, 128), (2, 25, 90, 2, True, 4, 4, 64),
])
def test_displaced_attention(B, H, W, N, cols, heads, kv, d, bf16):
    print("displaced kv4", B, H, W, N, cols, heads, kv, d, bf16, flush=True)
    L, patch = H * W, N // 2
    own = _own(H, W, patch, N, cols)
    k, v = _rows(1, B, L, kv, d, bf16=bf16), _rows(2, B, L, kv, d, bf16=bf16)
    cache = df.kv4_cache(B, L, kv, d)
    df.kv4_refresh(cache, k, v, 0, 1)
    fused = _rows(4, B, len(own), (heads + 2 * kv) * d, bf16=bf16, std=1.5)
    q, fk, fv = (t.unflatten(-1, (-1, d)) for t in fused.split([heads * d, kv * d, kv * d], -1))
    hk, hv = bo.held_in_4_bits(host(k)), bo.held_in_4_bits(host(v))
    hk[:, own], hv[:, own] = host(fk), host(fv)
    if cols:
        got = df.attn_displaced_kv4_cols(q, fk, fv, cache, H, W, patch, N)
    else:
        got = df.attn_displaced_kv4(q, fk, fv, cache, patch, N)
    _check(got, q, hk, hv, bf16)


@pytest.mark.parametrize("bf16", [True, False])
def test_a_cache_beyond_32_bits(bf16):
    """64 heads of 2^20 rows, 4.5 GB: the last 1000 rows of the last heads, among zeros."""
    L, h, d, n = 1 << 20, 64, 64, 1 << 10
    cache = df.kv4_cache(1, L, h, d)
    assert cache.numel() * cache.element_size() > 1 << 32
    k, v, q = _rows(1, 1, n, h, d, bf16=bf16, std=3.0), _rows(2, 1, n, h, d, bf16=bf16), _rows(3, 1, 2, h, d, bf16=bf16, std=3.0)
    df.kv4_refresh(cache, k, v, L // n - 1, L // n)
    got = host(df.attn_kv4(q, cache, L, h))[:, :, -2:]
    hk, hv = bo.held_in_4_bits(host(k))[:, :, -2:], bo.held_in_4_bits(host(v))[:, :, -2:]
    hq = host(q)[:, :, -2:]
    s = np.einsum("bqhd,bkhd->bhqk", hq, hk) * d ** -0.5
    w = np.exp(s)
    whole = w.sum(-1) + (L - n)                              # the zero rows have weight e^0 each
    ref = np.einsum("bhqk,bkhd->bqhd", w / whole[..., None], hv)
    size = np.einsum("bhqk,bkhd->bqhd", w / whole[..., None], np.abs(hv))
    reach = np.abs(np.einsum("bqhd,bkhd->bhqk", np.abs(hq), np.abs(hk))).max() * d ** -0.5
    assert (np.abs(got - ref) <= bo.attention_bound(ref, size, reach, d, L, bf16)).all() and np.abs(got).max() > 0
