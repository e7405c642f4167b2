"""The pipelined attention where it is to be used: over a cache with fresh rows of the patch in one piece or in strips, over a cache with lengths,
over rows far apart, gathered rows and many batch items.  Its workspace tells it from the other forms: those take whole numbers of parts of all
rows.  Some rows are compared with the 64-bit form (bounds derived there); what a cache holds is read back from it (bit for bit tested elsewhere)."""
import numpy as np
import pytest
import torch

import paper_2402_19481_amd as df
from oracle import block_ops as bo
from gpu_util import DEV, host

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _large_blocks_go_back():
    """(Tests of what happens where memory is short count what torch holds.)"""
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _rows(seed, *shape, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(BF16).to(DEV)


def _check(got, q, k, v, valid=None, scale=None):
    d = q.shape[-1]
    if valid is not None:                                    # what lies where there is no key must not matter to the reference either
        k, v = np.where(valid[:, :, None, None], k, 0), np.where(valid[:, :, None, None], v, 0)
    ref, size, reach = bo.attention(host(q), k, v, d ** -0.5 if scale is None else scale, valid)
    off = np.abs(host(got) - ref)
    bound = bo.attention_bound(ref, size, reach, d, k.shape[1], True)
    assert (off <= bound).all(), (np.argwhere(~(off <= bound))[:4], off.max(), float((off / bound).max()))


def _pipelined(workspace, B, Lq, heads, d, copied):
    """`copied`: bytes of the rows that are written side by side first"""
    assert workspace >= copied and workspace % (B * Lq * heads * (d + 2) * 4) != 0, "another form: the sizes do not test the pipelined one"


def _own(H, W, patch, N, cols):
    j = np.arange(H * W)
    return np.flatnonzero((j % W) // (W // N) == patch) if cols else j[patch * (H * W // N):(patch + 1) * (H * W // N)]


def _displaced(q, fk, fv, cache, H, W, patch, N, cols, **kw):
    if cols:
        return df.attn_displaced_kv4_cols(q, fk, fv, cache, H, W, patch, N, **kw)
    return df.attn_displaced_kv4(q, fk, fv, cache, patch, N, **kw)


@pytest.mark.parametrize("B,H,W,N,patch,cols,heads,kv,d", [
    (2, 40, 80, 2, 0, False, 4, 4, 64), (2, 40, 80, 2, 1, False, 4, 4, 64), (1, 63, 120, 3, 0, False, 8, 4, 64), (1, 63, 120, 3, 1, False, 8, 4, 64),
    (1, 63, 120, 3, 2, False, 8, 4, 64), (1, 63, 120, 3, 1, True, 8, 4, 64), (1, 64, 100, 2, 1, False, 4, 4, 128), (1, 64, 100, 2, 0, True, 4, 4, 128),
    # blocks of 256 rows, cut between workgroups and whole ones
    (1, 120, 160, 4, 1, False, 8, 8, 64), (1, 120, 160, 4, 3, True, 8, 8, 64), (1, 160, 160, 4, 2, False, 10, 5, 64),
])
def test_a_patch_beside_its_cache(B, H, W, N, patch, cols, heads, kv, d):
    print("displaced", B, H, W, N, patch, cols, heads, kv, d, flush=True)
    L, Lq = H * W, H * W // N
    _pipelined(df.lib().df_attn_displaced_kv4_workspace_bytes(B, H, W, heads, kv, d, patch, N, df.DF_BF16, int(cols)), B, Lq, heads, d,
               B * kv * (L - Lq) * d * 4)
    own = _own(H, W, patch, N, cols)
    cache = df.kv4_cache(B, L, kv, d)
    df.kv4_refresh(cache, _rows(1, B, L, kv, d), _rows(2, B, L, kv, d), 0, 1)
    fused = _rows(4, B, Lq, (heads + 2 * kv) * d, std=1.5)
    q, fk, fv = (t.unflatten(-1, (-1, d)) for t in fused.split([heads * d, kv * d, kv * d], -1))
    k, v = (host(t) for t in df.kv4_read(cache, B, L, kv, d))
    k[:, own], v[:, own] = host(fk), host(fv)
    rows = torch.tensor([0, 127, 128, 255, 256, Lq // 2, Lq - 1])
    got = _displaced(q, fk, fv, cache, H, W, patch, N, cols)
    _check(got[:, rows], q[:, rows], k, v)
    assert torch.equal(got, _displaced(q, fk, fv, cache, H, W, patch, N, cols))
    _check(_displaced(q, fk, fv, cache, H, W, patch, N, cols, scale=2.0)[:, rows], q[:, rows], k, v, scale=2.0)      # the running maximum moves


def test_fresh_rows_far_above_the_cached_ones():
    """The fresh keys' scores exceed the cached ones' by hundreds: the tile is done again with its own maximum."""
    B, H, W, N, heads, d = 2, 40, 80, 2, 4, 64
    L, Lq = H * W, H * W // N
    _pipelined(df.lib().df_attn_displaced_kv4_workspace_bytes(B, H, W, heads, heads, d, 1, N, df.DF_BF16, 0), B, Lq, heads, d, B * heads * (L - Lq) * d * 4)
    cache = df.kv4_cache(B, L, heads, d)
    df.kv4_refresh(cache, _rows(1, B, L, heads, d, std=0.1), _rows(2, B, L, heads, d), 0, 1)
    q, fk, fv = _rows(3, B, Lq, heads, d, std=8.0), _rows(4, B, Lq, heads, d, std=8.0), _rows(5, B, Lq, heads, d)
    k, v = (host(t) for t in df.kv4_read(cache, B, L, heads, d))
    k[:, Lq:], v[:, Lq:] = host(fk), host(fv)
    rows = torch.tensor([0, 127, 128, Lq - 1])
    _check(df.attn_displaced_kv4(q, fk, fv, cache, 1, N)[:, rows], q[:, rows], k, v)


@pytest.mark.parametrize("B,Lq,L,heads,kv,d,lens", [
    (2, 2500, 2500, 8, 8, 64, [2435, 0]), (2, 2500, 2500, 8, 8, 64, [1, 130]), (3, 2500, 2500, 8, 4, 64, [2500, 1, 700]), (2, 9000, 9000, 4, 4, 64, [9000, 4001]),
    (2, 9000, 9000, 4, 4, 64, [0, 8999]),
])
def test_a_cache_with_lengths(B, Lq, L, heads, kv, d, lens):
    print("lengths", B, Lq, L, heads, kv, d, lens, flush=True)
    _pipelined(df.lib().df_attn_kv4_workspace_bytes(B, Lq, L, heads, kv, d, df.DF_BF16), B, Lq, heads, d, B * kv * L * d * 4)
    k, v, q = _rows(1, B, L, kv, d), _rows(2, B, L, kv, d), _rows(3, B, Lq, heads, d, std=1.5)
    cache = df.kv4_cache(B, L, kv, d)
    df.kv4_refresh(cache, k, v, 0, 1)
    hk, hv = (host(t) for t in df.kv4_read(cache, B, L, kv, d))
    rows = torch.tensor([0, 127, 128, 255, 256, Lq - 1])
    _check(df.attn_kv4(q, cache, L, kv)[:, rows], q[:, rows], hk, hv)
    valid = np.arange(L)[None] < np.array(lens)[:, None]     # the rows behind hold no numbers
    k[~torch.from_numpy(valid).to(DEV)] = float("nan")
    v[~torch.from_numpy(valid).to(DEV)] = float("inf")
    df.kv4_refresh(cache, k, v, 0, 1)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    got = df.attn_kv4(q, cache, L, kv, lens=n)
    assert got.isfinite().all() and torch.equal(got, df.attn_kv4(q, cache, L, kv, lens=n))
    _check(got[:, rows], q[:, rows], hk, hv, valid)
    for b in range(B):
        assert lens[b] or not got[b].any()


def test_a_replayed_graph():
    B, H, W, N, heads, d = 2, 40, 80, 2, 4, 64
    L, Lq = H * W, H * W // N
    cache = df.kv4_cache(B, L, heads, d)
    df.kv4_refresh(cache, _rows(1, B, L, heads, d), _rows(2, B, L, heads, d), 0, 1)
    q, fk, fv = (_rows(s, B, Lq, heads, d) for s in (3, 4, 5))
    text, mask = _rows(6, B, 1300, heads, d), torch.rand(B, 1300, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.5
    _pipelined(df.lib().df_cross_attn_workspace_bytes(B, 6 * Lq, 1300, heads, heads, d, 1, df.DF_BF16), B, 6 * Lq, heads, d, B * heads * 1300 * d * 4)

    def both():
        x = df.attn_displaced_kv4(q, fk, fv, cache, 0, N)
        return x, df.cross_attn(x.repeat(1, 6, 1, 1), text, text, key_mask=mask)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for step in range(3):                                    # replays with the program's own work between them
        q.copy_(_rows(10 + step, B, Lq, heads, d))
        mask.copy_(torch.rand(B, 1300, generator=torch.Generator().manual_seed(step)) < 0.2 + 0.3 * step)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, both()):
            assert torch.equal(x, y), step


@pytest.mark.parametrize("Lq,masked", [(6000, False), (12000, True)])
def test_rows_far_apart(Lq, masked):
    """Keys and values 2^20 values apart, 3000 of them: offsets beyond 32 bits."""
    print("far", Lq, masked, flush=True)
    Lk, heads, d = 3000, 2, 64
    _pipelined(df.lib().df_cross_attn_workspace_bytes(1, Lq, Lk, heads, heads, d, int(masked), df.DF_BF16), 1, Lq, heads, d, masked * heads * Lk * d * 4)
    wide = torch.empty(Lk, 1 << 20, dtype=BF16, device=DEV)
    k, v = (wide[None, :, i * heads * d:(i + 1) * heads * d].unflatten(-1, (heads, d)) for i in range(2))
    k.copy_(_rows(2, 1, Lk, heads, d)), v.copy_(_rows(3, 1, Lk, heads, d))
    q = _rows(1, 1, Lq, heads, d)
    valid = np.arange(Lk)[None] % 5 != 0 if masked else None
    out = df.cross_attn(q, k, v, key_mask=torch.from_numpy(valid).to(DEV) if masked else None)
    rows = torch.tensor([0, 1, Lq // 2, Lq - 1])
    _check(out[:, rows], q[:, rows], host(k), host(v), valid)


@pytest.mark.parametrize("masked", [True, False])
def test_hardly_any_keys_where_many_were_planned(masked):
    """Shares of 4000 keys, of which a batch item has one or none: most of them are left without work."""
    print("hardly any", masked, flush=True)
    B, Lq, Lk, heads, d = 2, 6000, 4000, 2, 64
    _pipelined(df.lib().df_cross_attn_workspace_bytes(B, Lq, Lk, heads, heads, d, int(masked), df.DF_BF16), B, Lq, heads, d, masked * B * heads * Lk * d * 4)
    q, k, v = _rows(1, B, Lq, heads, d), _rows(2, B, Lk, heads, d), _rows(3, B, Lk, heads, d)
    for n in ([0, 0], [0, 1], [1, 0], [65, 1]):
        valid = torch.arange(Lk)[None] < torch.tensor(n)[:, None]
        if masked:
            valid = valid.flip(1)
            got = df.cross_attn(q, k, v, key_mask=valid.to(DEV))
        else:
            got = df.cross_attn(q, k, v, lens=torch.tensor(n, dtype=torch.int32, device=DEV))
        rows = torch.tensor([0, 127, 128, Lq - 1])
        _check(got[:, rows], q[:, rows], host(k), host(v), valid.numpy())
        for b in range(B):
            if n[b] < 2:                                     # one key: its values; none: zeros
                at = Lk - 1 if masked else 0
                assert torch.equal(got[b], v[b, at].expand(Lq, heads, d) if n[b] else torch.zeros_like(got[b]))


def test_infinite_keys_of_no_weight_beside_padding():
    """d between the kernels' widths: rows copied with zeros behind their values; a key whose scores are all -inf has weight 0."""
    Lq, Lk, heads, d = 4000, 1500, 4, 72
    _pipelined(df.lib().df_cross_attn_workspace_bytes(1, Lq, Lk, heads, heads, d, 0, df.DF_BF16), 1, Lq, heads, d, heads * Lk * 128 * 4)
    q, k, v = _rows(1, 1, Lq, heads, d).abs() + 1, _rows(2, 1, Lk, heads, d), _rows(3, 1, Lk, heads, d)
    w = k.clone()
    w[:, 1::3, :, 2] = float("-inf")                         # (all queries are positive there)
    valid = np.broadcast_to(np.arange(Lk)[None] % 3 != 1, (1, Lk))
    rows = torch.tensor([0, 1, Lq // 2, Lq - 1])
    got = df.cross_attn(q, w, v)
    assert got.isfinite().all()
    _check(got[:, rows], q[:, rows], host(k), host(v), valid)


@pytest.mark.parametrize("masked", [True, False])
def test_more_than_a_thousand_batch_items(masked):
    """So many that the shares stay as planned; items without keys among them."""
    B, Lq, Lk, d = 1030, 300, 900, 64
    _pipelined(df.lib().df_cross_attn_workspace_bytes(B, Lq, Lk, 1, 1, d, int(masked), df.DF_BF16), B, Lq, 1, d, masked * B * Lk * d * 4)
    q, k, v = _rows(1, B, Lq, 1, d), _rows(2, B, Lk, 1, d), _rows(3, B, Lk, 1, d)
    n = torch.randint(0, Lk + 1, (B,), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
    n[0], n[1], n[7], n[1029] = 0, Lk, 1, 64
    valid = torch.arange(Lk)[None] < n[:, None]
    if masked:
        valid &= torch.arange(Lk)[None] % 3 != 0
    gone = ~valid.to(DEV)
    k[gone], v[gone] = float("nan"), float("nan")
    got = df.cross_attn(q, k, v, key_mask=valid.to(DEV) if masked else None, lens=n.to(DEV))
    assert got.isfinite().all() and not got[0].any()
    items, rows = [0, 1, 2, 7, 500, 1029], torch.tensor([0, 127, 128, Lq - 1])
    _check(got[items][:, rows], q[items][:, rows], host(k[items]), host(v[items]), valid[items].numpy())
