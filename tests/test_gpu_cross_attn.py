"""Attention to an encoder's states of another length against the 64-bit form (bounds derived there)."""
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


def _check(got, q, k, v, bf16, valid=None, scale=None):
    d = q.shape[-1]
    if valid is not None:                                    # what lies in masked places must not matter to the reference either
        k, v = np.where(valid[:, :, None, None], k, 0), np.where(valid[:, :, None, None], v, 0)
    ref, size, reach = bo.attention(host(q), k, v, d ** -0.5 if scale is None else scale, valid)
    off = np.abs(host(got) - ref)
    bound = bo.attention_bound(ref, size, reach, d, k.shape[1], bf16)
    assert (off <= bound).all(), (np.argwhere(~(off <= bound))[:4], off.max(), float((off / bound).max()))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,Lq,Lk,heads,kv,d", [
    (1, 1, 1, 1, 1, 64), (1, 1, 77, 20, 20, 64), (2, 300, 77, 4, 4, 64), (1, 129, 64, 2, 2, 64), (2, 31, 300, 4, 2, 128), (1, 257, 130, 2, 2, 128),
    (1, 40, 65, 3, 3, 72), (1, 50, 200, 2, 1, 40), (1, 20, 33, 2, 2, 32), (1, 33, 500, 1, 1, 96), (1, 2, 3000, 2, 1, 64), (1, 9, 128, 1, 1, 8),
])
def test_lengths_and_masks(B, Lq, Lk, heads, kv, d, bf16):
    print("cross", B, Lq, Lk, heads, kv, d, bf16, flush=True)
    q = _rows(1, B, Lq, heads, d, bf16=bf16, std=1.5)
    fused = _rows(2, B, Lk, 2 * kv * d, bf16=bf16)
    k, v = fused[..., :kv * d].unflatten(-1, (kv, d)), fused[..., kv * d:].unflatten(-1, (kv, d))
    _check(df.cross_attn(q, k, v), q, host(k), host(v), bf16)
    _check(df.cross_attn(q, k, v, scale=2.5), q, host(k), host(v), bf16, scale=2.5)
    mask = torch.rand(B, Lk, generator=torch.Generator().manual_seed(9)) < 0.6
    mask[0, :70] = False                                     # a tile without a key in front (short prompts: none at all)
    lens = torch.tensor([Lk, max(1, Lk // 3)][:B], dtype=torch.int32)
    within = torch.arange(Lk)[None] < lens[:, None]
    for m, n in ((mask, None), (None, lens), (mask, lens)):
        valid = (m if m is not None else torch.ones(B, Lk, dtype=torch.bool)) & (within if n is not None else True)
        f = fused.clone()
        f[~valid.to(DEV)] = float("nan")
        k, v = f[..., :kv * d].unflatten(-1, (kv, d)), f[..., kv * d:].unflatten(-1, (kv, d))
        got = df.cross_attn(q, k, v, key_mask=None if m is None else m.to(DEV), lens=None if n is None else n.to(DEV))
        _check(got, q, host(k), host(v), bf16, valid.numpy())
        if not valid[0].any():
            assert not got[0].any()
    if m is not None:
        assert torch.equal(got, df.cross_attn(q, k, v, key_mask=m.to(torch.uint8).to(DEV) * 255, lens=lens.to(DEV)))


@pytest.mark.parametrize("bf16", [True, False])
def test_scores_far_apart_and_without_a_number(bf16):
    B, Lq, Lk, d = 1, 40, 400, 64
    q, k, v = _rows(1, B, Lq, 1, d, bf16=bf16, std=8.0), _rows(2, B, Lk, 1, d, bf16=bf16, std=8.0), _rows(3, B, Lk, 1, d, bf16=bf16)
    k = k * torch.linspace(0.1, 3, Lk, device=DEV)[None, :, None, None].to(k.dtype)    # the maximum climbs tile by tile
    got, kh = df.cross_attn(q, k, v), host(k)
    ref, size, reach = bo.attention(host(q), kh, host(v), d ** -0.5)
    assert reach > 300                                       # (the bound has the score's own error, which is not small here)
    assert (np.abs(host(got) - ref) <= bo.attention_bound(ref, size, reach, d, Lk, bf16)).all()
    lens = torch.tensor([7], dtype=torch.int32, device=DEV)
    w = k.clone()
    w[0, 3, 0, 0], w[0, 9] = float("nan"), float("nan")
    assert df.cross_attn(q, w, v, lens=lens).isnan().all()   # a key without a number counts, one behind the length does not
    w[0, 3] = k[0, 3]
    _check(df.cross_attn(q, w, v, lens=lens), q, kh, host(v), bf16, np.arange(Lk)[None] < 7)
    w[0, :7] = float("-inf")
    assert df.cross_attn(q.abs(), w, v, lens=lens).isnan().all()                       # every score -inf: the formula has no value


@pytest.mark.parametrize("Lq,Lk,heads,kv,d", [(130, 60, 600, 600, 64), (130, 130, 600, 600, 64), (70, 300, 600, 600, 64), (130, 1000, 600, 600, 64),
                                              (130, 1000, 700, 350, 64), (70, 200, 600, 600, 128), (20, 900, 600, 300, 72)])
def test_more_blocks_of_rows_than_workgroups(Lq, Lk, heads, kv, d):
    """Workgroups that go from block to block, and blocks that are cut between two of them."""
    print("blocks", Lq, Lk, heads, kv, d, flush=True)
    q, k, v = _rows(1, 1, Lq, heads, d), _rows(2, 1, Lk, kv, d), _rows(3, 1, Lk, kv, d)
    mask = torch.rand(1, Lk, generator=torch.Generator().manual_seed(5)) < 0.7
    mask[0, 64:128] = False
    out = df.cross_attn(q, k, v), df.cross_attn(q, k, v, key_mask=mask.to(DEV)), df.cross_attn(q, k, v, lens=torch.tensor([Lk - 7], dtype=torch.int32, device=DEV))
    valid = None, mask.numpy(), np.arange(Lk)[None] < Lk - 7
    g = heads // kv
    for h in (0, 1, kv // 2, kv - 2, kv - 1):                # some heads: the others are the same kernel's
        for got, ok in zip(out, valid):
            _check(got[:, :, h * g:(h + 1) * g], q[:, :, h * g:(h + 1) * g], host(k[:, :, h:h + 1]), host(v[:, :, h:h + 1]), True, ok)
    from_f32 = df.cross_attn(q[:, :, :g].float(), k[:, :, :1].float(), v[:, :, :1].float())
    assert torch.allclose(out[0][:, :, :g].float(), from_f32, rtol=0.05, atol=0.05)
    one = [torch.cat([df.cross_attn(q[:, :, h * g:(h + 1) * g].contiguous(), k[:, :, h:h + 1].contiguous(), v[:, :, h:h + 1].contiguous())]) for h in range(0, kv, 37)]
    for i, h in enumerate(range(0, kv, 37)):
        assert torch.allclose(out[0][:, :, h * g:(h + 1) * g].float(), one[i].float(), rtol=0.02, atol=0.02)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("Lq,Lk,heads", [(5, 3000, 1), (300, 5000, 2), (40, 130, 1)])
def test_parts_whose_scores_are_all_minus_infinity(Lq, Lk, heads, bf16):
    """Keys are split over workgroups: one that sees none but scores of -inf has no share in the others' result."""
    q, k, v = _rows(1, 1, Lq, heads, 64, bf16=bf16).abs(), _rows(2, 1, Lk, heads, 64, bf16=bf16), _rows(3, 1, Lk, heads, 64, bf16=bf16)
    w = k.clone()
    w[:, :Lk // 2] = float("-inf")
    valid = np.broadcast_to(np.arange(Lk)[None] >= Lk // 2, (1, Lk))
    _check(df.cross_attn(q, w, v), q, host(k), host(v), bf16, valid)
    assert df.cross_attn(q, torch.full_like(k, float("-inf")), v).isnan().all()


def test_the_same_bits_and_a_given_result():
    q, k, v = _rows(1, 2, 50, 4, 64), _rows(2, 2, 900, 2, 64), _rows(3, 2, 900, 2, 64)
    out = torch.empty_like(q)
    assert df.cross_attn(q, k, v, out=out) is out
    assert all(torch.equal(out, df.cross_attn(q, k, v)) for _ in range(3))


@pytest.mark.parametrize("masked,lengths", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("Lq,Lk,heads,kv,d", [(2000, 1300, 8, 4, 64), (1500, 900, 8, 8, 128), (1111, 1027, 5, 5, 72), (6000, 4099, 4, 4, 64),
                                              (6144, 6100, 4, 4, 64)])
def test_batch_items_with_different_numbers_of_keys(Lq, Lk, heads, kv, d, masked, lengths):
    """Long enough for the pipelined form: the work is shared by the keys there are; what is no key holds NaN."""
    print("numbers", Lq, Lk, heads, kv, d, masked, lengths, flush=True)
    B = 4
    q, fused = _rows(1, B, Lq, heads, d), _rows(2, B, Lk, 2 * kv * d)
    n = np.array([Lk, 517, 0, 65]) if lengths else np.full(B, Lk)
    valid = np.arange(Lk)[None] < n[:, None]
    mask = torch.rand(B, Lk, generator=torch.Generator().manual_seed(6)) < torch.tensor([0.9, 0.5, 1.0, 0.01])[:, None]
    if masked:
        mask[1, :200] = False
        valid = valid & mask.numpy()
    gone = torch.from_numpy(~valid).to(DEV)
    fused = torch.where(gone[..., None], torch.full_like(fused, float("nan")), fused)
    k, v = fused[..., :kv * d].unflatten(-1, (kv, d)), fused[..., kv * d:].unflatten(-1, (kv, d))
    rows = torch.tensor([0, 1, 127, 128, Lq // 2, Lq - 1])
    out = df.cross_attn(q, k, v, key_mask=mask.to(DEV) if masked else None, lens=torch.tensor(n, dtype=torch.int32, device=DEV) if lengths else None)
    assert out.isfinite().all()
    _check(out[:, rows], q[:, rows], host(k), host(v), True, valid)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("Lq,Lk,heads", [(5, 77, 2), (300, 1000, 2), (2000, 1500, 4)])
def test_infinite_keys_of_no_weight_beside_padding(Lq, Lk, heads, bf16):
    """d between the kernels' widths: a key whose scores are all -inf has weight 0, also where its infinities lie in the row's first values; and an
    infinite value under a key does not become NaN by way of keys that are none."""
    print("infinite", Lq, Lk, heads, bf16, flush=True)
    d = 72 if bf16 else 40
    q, k, v = _rows(1, 1, Lq, heads, d, bf16=bf16).abs() + 1, _rows(2, 1, Lk, heads, d, bf16=bf16), _rows(3, 1, Lk, heads, d, bf16=bf16)
    w = k.clone()
    w[:, 1::3, :, 2] = float("-inf")                         # (all queries are positive there)
    valid = np.broadcast_to(np.arange(Lk)[None] % 3 != 1, (1, Lk))
    rows = torch.tensor([0, 1, Lq // 2, Lq - 1])
    got = df.cross_attn(q, w, v)
    assert got.isfinite().all()
    _check(got[:, rows], q[:, rows], host(k), host(v), bf16, valid)


@pytest.mark.parametrize("Lq,bf16,masked", [(5, True, False), (2000, True, False), (2000, True, True), (300, False, False)])
def test_offsets_beyond_32_bits(Lq, bf16, masked):
    """Keys and values 2^20 values apart, 3000 of them."""
    print("far", Lq, bf16, masked, flush=True)
    Lk, heads, d = 3000, 2, 64
    wide = torch.empty(Lk, 1 << 20, dtype=TYPES[bf16], device=DEV)
    k, v = (wide[None, :, i * heads * d:(i + 1) * heads * d].unflatten(-1, (heads, d)) for i in range(2))
    k.copy_(_rows(2, 1, Lk, heads, d, bf16=bf16)), v.copy_(_rows(3, 1, Lk, heads, d, bf16=bf16))
    q = _rows(1, 1, Lq, heads, d, bf16=bf16)
    valid = np.arange(Lk)[None] % 5 != 0 if masked else None
    out = df.cross_attn(q, k, v, key_mask=torch.from_numpy(valid).to(DEV) if masked else None)
    rows = torch.tensor([0, 1, Lq // 2, Lq - 1])
    _check(out[:, rows], q[:, rows], host(k), host(v), bf16, valid)


@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_hardly_any_keys_where_many_were_planned(d, masked):
    """Workgroups for 4000 keys, of which a batch item has one or none: most of them are left without work."""
    print("hardly any", d, masked, flush=True)
    B, Lq, Lk, heads = 2, 2000, 4000, 2
    q, k, v = _rows(1, B, Lq, heads, d), _rows(2, B, Lk, heads, d), _rows(3, B, Lk, heads, d)
    for n in ([0, 0], [0, 1], [1, 0], [65, 1]):
        valid = torch.arange(Lk)[None] < torch.tensor(n)[:, None]
        if masked:
            valid = valid.flip(1)
            got = df.cross_attn(q, k, v, key_mask=valid.to(DEV))
        else:
            got = df.cross_attn(q, k, v, lens=torch.tensor(n, dtype=torch.int32, device=DEV))
        rows = torch.tensor([0, 127, 128, Lq - 1])
        _check(got[:, rows], q[:, rows], host(k), host(v), True, valid.numpy())
        for b in range(B):
            if n[b] < 2:                                     # one key: its values; none: zeros
                at = Lk - 1 if masked else 0
                assert torch.equal(got[b], v[b, at].expand(Lq, heads, d) if n[b] else torch.zeros_like(got[b]))
