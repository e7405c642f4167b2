"""Norm and rotation of queries and keys against the 64-bit form, value by value.

Tolerance: the result's rounding (2^-8 of it in bf16, 2^-24 in float32) and 32 roundings of the 32-bit arithmetic (at most 8 + 6 in the sum
of squares, halved by the root; root, mean, gamma, two products and a sum) of the terms a value is made of."""
import numpy as np
import pytest
import torch

import paper_2402_19481_amd as df
from oracle import block_ops as bo
from gpu_util import DEV, host

pytestmark = pytest.mark.gpu


def _table(rows, half, seed=5):
    a = np.random.default_rng(seed).uniform(-50, 50, (rows, half))
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def _near(got, ref, size, bf16):
    u = 2.0 ** -24
    ok = np.abs(host(got) - ref) <= (2.0 ** -8 if bf16 else u) * np.abs(ref) + 32 * u * size + 1e-37
    assert ok.all(), np.argwhere(~ok)[:3]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,T,hq,hk,d,rot,inter", [
    (1, 1, 1, 1, 8, 8, True), (1, 1, 20, 20, 64, 64, True), (2, 37, 10, 10, 64, 64, False), (1, 5, 5, 1, 72, 72, False), (2, 9, 3, 2, 72, 40, True),
    (1, 33, 16, 4, 128, 96, False), (1, 6, 7, 2, 256, 256, False), (1, 6, 7, 2, 256, 128, True), (3, 130, 4, 4, 40, 16, False), (1, 3, 130, 2, 16, 8, False),
])
def test_fused_projection(B, T, hq, hk, d, rot, inter, bf16):
    print("rope", B, T, hq, hk, d, rot, inter, bf16, flush=True)
    g = torch.Generator().manual_seed(T)
    qkv = (torch.randn(B, T, (hq + 2 * hk) * d, generator=g) * 3).to(torch.bfloat16 if bf16 else torch.float32)
    gq, gk = 1 + 0.1 * torch.randn(d, generator=g), 1 + 0.1 * torch.randn(d, generator=g)
    table = _table(T + 2, rot // 2)
    x = qkv.to(DEV)
    before = x.clone()
    q, k = x[..., :hq * d].unflatten(-1, (hq, d)), x[..., hq * d:(hq + hk) * d].unflatten(-1, (hk, d))
    qo, ko = df.qk_norm_rope(q, k, gq.to(DEV), gk.to(DEV), torch.from_numpy(table).to(DEV), eps=1e-5, interleaved=inter)
    for got, src, gm in ((qo, q, gq), (ko, k, gk)):
        ref, size = bo.qk_norm_rope(host(src), gm.numpy(), table, eps=1e-5, interleaved=inter)
        _near(got, ref, size, bf16)
    assert torch.equal(x, before)
    # in place, the keys into a patch's rows of a full buffer
    full = torch.full((B, 3 * T, hk, d), 7.0, dtype=x.dtype, device=DEV)
    qi, kf = df.qk_norm_rope(q, k, gq.to(DEV), gk.to(DEV), torch.from_numpy(table).to(DEV), eps=1e-5, interleaved=inter, q_out=q, k_out=full[:, T:2 * T])
    assert qi is q and torch.equal(q, qo) and torch.equal(full[:, T:2 * T], ko)
    assert (full[:, :T] == 7).all() and (full[:, 2 * T:] == 7).all() and torch.equal(x[..., hq * d:], before[..., hq * d:])


@pytest.mark.parametrize("bf16", [True, False])
def test_positions_and_parts(bf16):
    B, T, hq, d = 2, 21, 6, 64
    g = torch.Generator().manual_seed(3)
    x = torch.randn(B, T, hq, d, generator=g).to(torch.bfloat16 if bf16 else torch.float32).to(DEV)
    table = _table(9, 16)
    pos = torch.randint(-2, 9, (B, T), generator=g, dtype=torch.int32)
    pos[1, 4] = 9
    td, pd = torch.from_numpy(table).to(DEV), pos.to(DEV)
    for inter in (True, False):
        got, none = df.qk_norm_rope(x, rot=td, pos=pd, interleaved=inter)            # queries alone, no scale
        assert none is None
        ref, size = bo.qk_norm_rope(host(x), None, table, pos.numpy(), interleaved=inter)
        bad = np.zeros(ref.shape, bool)
        bad[1, 4, :, :32] = True
        assert np.isnan(host(got)[bad]).all()
        _near(torch.where(torch.from_numpy(bad).to(DEV), torch.zeros_like(got), got), np.where(bad, 0, ref), np.where(bad, 0, size), bf16)
        got, _ = df.qk_norm_rope(x, rot=td, pos=pd.clamp(max=8), norm=False, interleaved=inter)
        ref, size = bo.qk_norm_rope(host(x), None, table, pos.clamp(max=8).numpy(), norm=False, interleaved=inter)
        _near(got, ref, size, bf16)
    got, _ = df.qk_norm_rope(x, eps=0.0)
    ref, size = bo.qk_norm_rope(host(x), eps=0.0)
    _near(got, ref, size, bf16)


def test_odd_strides_and_alignment():
    """bf16 rows that 8-byte accesses take but 16-byte ones do not; tokens before batch items."""
    B, T, h, d = 3, 7, 2, 24
    base = torch.randn(T, B, h * d + 4, device=DEV).to(torch.bfloat16)
    x = base[..., 4:].unflatten(-1, (h, d)).transpose(0, 1)
    table = _table(T, 12)
    for inter in (True, False):
        got, _ = df.qk_norm_rope(x, rot=torch.from_numpy(table).to(DEV), interleaved=inter)
        ref, size = bo.qk_norm_rope(host(x), None, table, interleaved=inter)
        _near(got, ref, size, True)
    with pytest.raises(df.DfError):
        df.qk_norm_rope(torch.randn(1, 2, 1, 9, device=DEV)[..., 1:])               # 4-byte alignment


def test_zeros_infinities_and_large_offsets():
    x = torch.zeros(1, 3, 1, 64, device=DEV)
    x[0, 1, 0, 5] = float("inf")
    x[0, 2] = 1e-20
    got, _ = df.qk_norm_rope(x)
    assert not got[0, 0].any() and got[0, 1].isnan().any()
    _near(got[:, 2:], bo.qk_norm_rope(host(x[:, 2:]))[0], bo.qk_norm_rope(host(x[:, 2:]))[1], False)
    big = torch.zeros((1 << 31) + 4096, dtype=torch.bfloat16, device=DEV)           # batch items more than 2^31 elements apart
    y = big.as_strided((2, 2, 2, 64), (1 << 31, 128, 64, 1))
    y.copy_(torch.randn(2, 2, 2, 64, device=DEV))
    got, _ = df.qk_norm_rope(y)
    ref, size = bo.qk_norm_rope(host(y))
    _near(got, ref, size, True)
