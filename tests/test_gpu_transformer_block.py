"""The operators of a transformer block together, as a user's denoising loop calls them: fused projection -> norm and rotation ->
displaced attention over a 4-bit cache -> refresh -> cross-attention to a padded prompt; eager, on another stream and as a replayed graph."""
import numpy as np
import pytest
import torch

import paper_2402_19481_amd as df
from oracle import block_ops as bo
from gpu_util import DEV, host

pytestmark = pytest.mark.gpu

B, H, W, N, HEADS, KV, D, LK = 2, 12, 21, 3, 4, 2, 64, 90
L, LQ = H * W, H * W // N


def _inputs(step, cols):
    g = torch.Generator().manual_seed(step)
    qkv = torch.randn(B, LQ, (HEADS + 2 * KV) * D, generator=g).to(torch.bfloat16)
    text = torch.randn(B, LK, 2 * KV * D, generator=g).to(torch.bfloat16)
    return qkv.to(DEV), text.to(DEV)


def _block(qkv, text, cache, consts, patch, cols, out=None):
    gq, gk, rot, mask = consts
    q, k, v = (t.unflatten(-1, (-1, D)) for t in qkv.split([HEADS * D, KV * D, KV * D], -1))
    q, k = df.qk_norm_rope(q, k, gq, gk, rot)
    if cols:
        x = df.attn_displaced_kv4_cols(q, k, v, cache, H, W, patch, N)
        df.kv4_refresh_cols(cache, k, v, H, W, patch, N)
    else:
        x = df.attn_displaced_kv4(q, k, v, cache, patch, N)
        df.kv4_refresh(cache, k, v, patch, N)
    tk, tv = (t.unflatten(-1, (KV, D)) for t in text.split(KV * D, -1))
    return q, k, x, df.cross_attn(x, tk, tv, key_mask=mask, out=out)


def _consts(patch, cols):
    g = torch.Generator().manual_seed(100)
    j = np.arange(L)
    own = np.flatnonzero((j % W) // (W // N) == patch) if cols else j[patch * LQ:(patch + 1) * LQ]
    a = own[:, None] * 100.0 ** (-np.arange(D // 2) / (D // 2))
    rot = torch.from_numpy(np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)).to(DEV)
    mask = torch.ones(B, LK, dtype=torch.bool)
    mask[0, 40:] = False
    mask[1, :3] = False
    return own, (1 + 0.1 * torch.randn(D, generator=g)).to(DEV), (1 + 0.1 * torch.randn(D, generator=g)).to(DEV), rot, mask.to(DEV)


@pytest.mark.parametrize("cols", [False, True])
def test_block_against_64_bits(cols):
    own, *consts = _consts(1, cols)
    g = torch.Generator().manual_seed(7)
    k0, v0 = (torch.randn(B, L, KV, D, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    cache = df.kv4_cache(B, L, KV, D)
    df.kv4_refresh(cache, k0, v0, 0, 1)
    hk, hv = bo.held_in_4_bits(host(k0)), bo.held_in_4_bits(host(v0))
    for step in range(2):                                    # the second step reads what the first refreshed
        qkv, text = _inputs(step, cols)
        q, k, x, y = _block(qkv, text, cache, consts, 1, cols)
        v = qkv[..., (HEADS + KV) * D:].unflatten(-1, (KV, D))
        for got, lo, n, gm in ((q, 0, HEADS, consts[0]), (k, HEADS, KV, consts[1])):
            ref, size = bo.qk_norm_rope(host(qkv)[..., lo * D:(lo + n) * D].reshape(B, LQ, n, D), host(gm), host(consts[2]))
            assert (np.abs(host(got) - ref) <= 2.0 ** -8 * np.abs(ref) + 32 * 2.0 ** -24 * size).all()
        sk, sv = hk.copy(), hv.copy()
        sk[:, own], sv[:, own] = host(k), host(v)
        ref, size, reach = bo.attention(host(q), sk, sv, D ** -0.5)
        assert (np.abs(host(x) - ref) <= bo.attention_bound(ref, size, reach, D, L, True)).all()
        hk[:, own], hv[:, own] = bo.held_in_4_bits(host(k)), bo.held_in_4_bits(host(v))
        gk, gv = df.kv4_read(cache, B, L, KV, D)
        assert np.array_equal(host(gk), hk) and np.array_equal(host(gv), hv)
        t = host(text)
        ref, size, reach = bo.attention(host(x), t[..., :KV * D].reshape(B, LK, KV, D), t[..., KV * D:].reshape(B, LK, KV, D), D ** -0.5, host(consts[3]) > 0)
        assert (np.abs(host(y) - ref) <= bo.attention_bound(ref, size, reach, D, LK, True)).all()


def test_block_as_a_graph_and_on_another_stream():
    own, *consts = _consts(1, False)
    g = torch.Generator().manual_seed(7)
    k0, v0 = (torch.randn(B, L, KV, D, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    caches = [df.kv4_cache(B, L, KV, D) for _ in range(3)]
    qkv, text = (t.clone() for t in _inputs(0, False))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph, got = torch.cuda.CUDAGraph(), None
    with torch.cuda.stream(stream):
        _block(qkv, text, caches[0], consts, 1, False)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = _block(qkv, text, caches[0], consts, 1, False)
    for c in caches:
        df.kv4_refresh(c, k0, v0, 0, 1)
    for step in range(4):                                    # replays with the program's own work between them
        a, t = _inputs(step, False)
        qkv.copy_(a)
        text.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        want = _block(a, t, caches[1], consts, 1, False)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            other = _block(a, t, caches[2], consts, 1, False)
        torch.cuda.current_stream().wait_stream(stream)
        for x, y, z in zip(got, want, other):
            assert torch.equal(x, y) and torch.equal(x, z), step
        assert torch.equal(caches[0], caches[1]) and torch.equal(caches[0], caches[2])


def test_what_the_binding_refuses_on_the_gpu():
    x = torch.zeros(2, 8, 4, 64, dtype=torch.bfloat16, device=DEV)
    cache = df.kv4_cache(2, 16, 4, 64)
    for call, error in [
        (lambda: df.cross_attn(x, x.float(), x.float()), df.DfError), (lambda: df.cross_attn(x, x, x[:, :7]), ValueError),
        (lambda: df.cross_attn(x, x[:1], x[:1]), ValueError), (lambda: df.cross_attn(x, x.cpu(), x.cpu()), df.DfError),
        (lambda: df.cross_attn(x, x, x, key_mask=torch.ones(2, 9, dtype=torch.bool, device=DEV)), ValueError),
        (lambda: df.cross_attn(x, x, x, key_mask=torch.ones(2, 8, device=DEV)), df.DfError),
        (lambda: df.cross_attn(x, x, x, lens=torch.ones(2, dtype=torch.int64, device=DEV)), df.DfError),
        (lambda: df.cross_attn(x, x, x, lens=torch.ones(2, dtype=torch.int32)), df.DfError),
        (lambda: df.cross_attn(x, x, x, out=x[:, :, :2]), ValueError), (lambda: df.cross_attn(x, x, x, out=x.float()), df.DfError),
        (lambda: df.cross_attn(x, x[:, :, :3], x[:, :, :3]), df.DfError), (lambda: df.cross_attn(x.half(), x.half(), x.half()), df.DfError),
        (lambda: df.cross_attn(x.transpose(1, 2), x, x), df.DfError),
        (lambda: df.attn_kv4(x, cache, 17, 4), None), (lambda: df.attn_kv4(x, cache, 65, 4), ValueError), (lambda: df.attn_kv4(x, cache, 16, 3), ValueError),
        (lambda: df.attn_kv4(x, cache.float(), 16, 4), df.DfError), (lambda: df.attn_displaced_kv4(x, x, x, cache, 2, 2), df.DfError),
        (lambda: df.attn_displaced_kv4_cols(x, x, x, cache, 4, 4, 0, 4), ValueError), (lambda: df.kv4_refresh(cache, x, x, 0, 20), ValueError),
        (lambda: df.kv4_refresh_cols(cache, x, x, 4, 4, 0, 3), ValueError), (lambda: df.kv4_read(cache, 2, 16, 4, 128), ValueError),
        (lambda: df.qk_norm_rope(x, x[:, :7]), ValueError), (lambda: df.qk_norm_rope(x, norm=False), df.DfError),
        (lambda: df.qk_norm_rope(x, q_gamma=torch.ones(63, device=DEV)), ValueError),
        (lambda: df.qk_norm_rope(x, rot=torch.zeros(7, 32, 2, device=DEV)), df.DfError), (lambda: df.qk_norm_rope(x, rot=torch.zeros(8, 32, 3, device=DEV)), ValueError),
        (lambda: df.qk_norm_rope(x, rot=torch.zeros(8, 32, 2, device=DEV), pos=torch.zeros(2, 7, dtype=torch.int32, device=DEV)), ValueError),
        (lambda: df.qk_norm_rope(x, q_out=x[:, :4]), ValueError), (lambda: df.qk_norm_rope(x, k_out=x), ValueError),
        (lambda: df.qk_norm_rope(x, q_out=x[:, :1].expand(2, 8, 4, 64)), df.DfError),
    ]:
        if error is None:
            call()                                           # (17 rows lie in as many bytes as 16)
        else:
            with pytest.raises(error):
                call()
