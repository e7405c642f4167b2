"""What the operators of a transformer block refuse, and how (no GPU: nothing is launched, the addresses are never read)."""
import pytest
import torch

import paper_2402_19481_amd as df

EINVAL, ESHAPE, ENOMEM = -1, -2, -4
A = 1 << 20                                                  # an aligned address
X = torch.zeros(2, 8, 4, 64)


@pytest.mark.parametrize("call,error", [
    (lambda: df.qk_norm_rope(X), df.DfError),                                                  # not on the GPU
    (lambda: df.kv4_refresh(X, X, X, 0, 1), df.DfError),
    (lambda: df.kv4_read(torch.zeros(10, dtype=torch.uint8), 1, 1, 1, 64), df.DfError),
    (lambda: df.attn_kv4(X, X, 8, 4), df.DfError),
    (lambda: df.attn_displaced_kv4(X, X, X, X, 0, 1), df.DfError),
    (lambda: df.cross_attn(X, X, X), df.DfError),
    (lambda: df.kv4_read(X, 1, 1, 1, 64, dtype=torch.float16), df.DfError),                    # type of the result
    (lambda: df.kv4_cache(1, 8, 4, 72, device="cpu"), df.DfError),                             # head size
    (lambda: df.kv4_cache(0, 8, 4, 64, device="cpu"), df.DfError),
    (lambda: df.qk_norm_rope(X[0]), ValueError),                                               # dimensions
    (lambda: df.cross_attn(X[0], X, X), ValueError),
    (lambda: df.attn_displaced_kv4(X[0], X, X, X, 0, 1), ValueError),
    (lambda: df.qk_norm_rope(3), TypeError),
    (lambda: df.kv4_refresh(X, 3, X, 0, 1), TypeError),
])
def test_binding(call, error):
    with pytest.raises(error):
        call()


def _rope(q=A, k=A, qo=A, ko=A, ld=256, bs=2048, old=256, obs=2048, qg=A, rot=A, pos=None, B=2, T=8, heads=4, kv=4, d=64, rot_dim=64, rows=8, norm=1,
          eps=1e-6, dt=df.DF_BF16):
    return df.lib().df_qk_norm_rope(q, ld, bs, k, ld, bs, qo, old, obs, ko, old, obs, qg, qg, rot, pos, B, T, heads, kv, d, rot_dim, rows, norm, eps, 1, dt, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(k=None), EINVAL), (dict(ko=None), EINVAL), (dict(dt=2), EINVAL),
    (dict(norm=0, rot=None), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(ld=-256), EINVAL),
    (dict(q=A + 4), EINVAL), (dict(ld=257), EINVAL), (dict(ld=258), EINVAL), (dict(dt=df.DF_F32, q=A + 8), EINVAL), (dict(dt=df.DF_F32, ld=258), EINVAL),
    (dict(qg=A + 4), EINVAL), (dict(rot=A + 8), EINVAL), (dict(pos=A + 2), EINVAL), (dict(old=0), EINVAL), (dict(obs=0), EINVAL),
    (dict(B=0), ESHAPE), (dict(T=0), ESHAPE), (dict(heads=0), ESHAPE), (dict(kv=0), ESHAPE), (dict(k=None, ko=None), ESHAPE), (dict(d=60), ESHAPE),
    (dict(d=264), ESHAPE), (dict(rot_dim=0), ESHAPE), (dict(rot_dim=12), ESHAPE), (dict(rot_dim=72), ESHAPE), (dict(rows=7), ESHAPE), (dict(rows=0), ESHAPE),
    (dict(T=1 << 30, B=4, rows=1 << 30, obs=1 << 40), ESHAPE), (dict(T=1 << 26, B=1, rows=1 << 26), ESHAPE),
])
def test_qk_norm_rope(kw, rc):
    assert _rope(**kw) == rc


def _refresh(c=A, k=A, v=A, ld=256, bs=2048, B=2, H=4, W=16, kv=4, d=64, patch=0, N=2, dt=df.DF_BF16, axis=0):
    return df.lib().df_kv4_refresh(c, k, ld, bs, v, ld, bs, B, H, W, kv, d, patch, N, dt, axis, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(c=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(c=A + 8), EINVAL), (dict(k=A + 8), EINVAL), (dict(ld=260), EINVAL),
    (dict(bs=-8), EINVAL), (dict(dt=3), EINVAL), (dict(axis=2), EINVAL), (dict(H=0), ESHAPE), (dict(N=0), ESHAPE), (dict(N=3), ESHAPE), (dict(patch=2), ESHAPE),
    (dict(patch=-1), ESHAPE), (dict(axis=1, N=3), ESHAPE), (dict(d=32), ESHAPE), (dict(B=0), ESHAPE), (dict(kv=0), ESHAPE), (dict(B=65536), ESHAPE),
    (dict(H=1 << 16, W=1 << 15), ESHAPE), (dict(H=1 << 15, W=1 << 15), ESHAPE),
])
def test_kv4_refresh(kw, rc):
    assert _refresh(**kw) == rc


def test_kv4_read_and_sizes():
    L = df.lib()
    assert L.df_kv4_bytes(2, 65, 3, 64) == 2 * 3 * 128 * 68 and L.df_kv4_bytes(1, 64, 1, 128) == 64 * 132
    assert L.df_kv4_bytes(1, 0, 1, 64) == L.df_kv4_bytes(1, 64, 1, 96) == 0
    assert L.df_kv4_read(None, A, A, 1, 64, 1, 64, 1, None) == L.df_kv4_read(A, A + 2, A, 1, 64, 1, 64, 1, None) == EINVAL
    assert L.df_kv4_read(A, A, A, 1, 64, 1, 64, 7, None) == EINVAL and L.df_kv4_read(A, A, A, 1, 64, 1, 80, 1, None) == ESHAPE


def _cross(q=A, k=A, v=A, ld=256, lens=None, out=A, B=2, Lq=8, Lk=4096, heads=4, kv=4, d=64, scale=0.1, dt=df.DF_BF16, w=A, wb=1 << 40):
    return df.lib().df_cross_attn(q, ld, 1 << 24, k, ld, 1 << 24, v, ld, 1 << 24, None, lens, out, B, Lq, Lk, heads, kv, d, scale, dt, w, wb, None)


def _cached(q=A, c=A, lens=None, out=A, B=2, Lq=8, Lk=4096, heads=4, kv=4, d=64, scale=0.1, dt=df.DF_BF16, w=A, wb=1 << 40):
    return df.lib().df_attn_kv4(q, 256, 1 << 24, c, lens, out, B, Lq, Lk, heads, kv, d, scale, dt, w, wb, None)


def _displaced(q=A, k=A, c=A, out=A, ld=256, B=2, H=8, W=512, heads=4, kv=4, d=64, patch=1, N=2, scale=0.1, dt=df.DF_BF16, axis=0, w=A, wb=1 << 40):
    return df.lib().df_attn_displaced_kv4(q, 256, 1 << 24, k, ld, 1 << 24, k, ld, 1 << 24, c, out, B, H, W, heads, kv, d, patch, N, scale, dt, axis, w, wb,
                                          None)


@pytest.mark.parametrize("call", [_cross, _cached, _displaced])
@pytest.mark.parametrize("kw,rc", [
    (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q=A + 8), EINVAL), (dict(out=A + 8), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(dt=2), EINVAL), (dict(w=A + 128), EINVAL), (dict(B=0), ESHAPE),
    (dict(heads=5), ESHAPE), (dict(heads=0), ESHAPE), (dict(kv=0), ESHAPE), (dict(d=136), ESHAPE), (dict(d=60), ESHAPE), (dict(w=None, wb=0), ENOMEM),
    (dict(wb=64), ENOMEM),
])
def test_attention(call, kw, rc):
    assert call(**kw) == rc


@pytest.mark.parametrize("got,rc", [
    (lambda: _cross(k=None), EINVAL), (lambda: _cross(k=A + 2), EINVAL), (lambda: _cross(ld=252), EINVAL), (lambda: _cross(lens=A + 1), EINVAL),
    (lambda: _cross(Lq=0), ESHAPE), (lambda: _cross(Lk=0), ESHAPE), (lambda: _cross(Lq=1 << 30, heads=1 << 10), ESHAPE), (lambda: _cached(c=None), EINVAL),
    (lambda: _cached(c=A + 4), EINVAL), (lambda: _cached(lens=A + 2), EINVAL), (lambda: _cached(d=96), ESHAPE), (lambda: _cached(Lk=0), ESHAPE),
    (lambda: _displaced(k=None), EINVAL), (lambda: _displaced(c=None), EINVAL), (lambda: _displaced(axis=2), EINVAL), (lambda: _displaced(patch=2), ESHAPE),
    (lambda: _cross(ld=(1 << 24) + 8), ESHAPE), (lambda: _displaced(ld=(1 << 24) + 8), ESHAPE),
    (lambda: _displaced(N=3), ESHAPE), (lambda: _displaced(axis=1, N=3), ESHAPE), (lambda: _displaced(d=32), ESHAPE),
])
def test_attention_each(got, rc):
    assert got() == rc


def test_workspace_of_sizes_that_are_not_taken():
    L = df.lib()
    assert L.df_cross_attn_workspace_bytes(1, 1, 64, 1, 1, 200, 0, 1) == 0
    assert L.df_attn_kv4_workspace_bytes(1, 1, 64, 1, 1, 96, 1) == 0
    assert L.df_attn_displaced_kv4_workspace_bytes(1, 8, 8, 1, 1, 64, 0, 5, 1, 0) == 0
    assert L.df_attn_kv4_workspace_bytes(1, 1, 57600, 1, 1, 64, 1) > 0
