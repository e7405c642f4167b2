"""Norm and rotation at the ends of float's range, and of tokens that are not rotated.  Tolerances as in test_gpu_qk_norm_rope.py."""
import numpy as np
import pytest
import torch

import paper_2402_19481_amd as df
from oracle import block_ops as bo
from gpu_util import DEV, host

pytestmark = pytest.mark.gpu
TYPES = {True: torch.bfloat16, False: torch.float32}


def _near(got, ref, size, bf16):
    u = 2.0 ** -24
    ok = np.abs(host(got) - ref) <= (2.0 ** -8 if bf16 else u) * np.abs(ref) + 32 * u * size + 1e-37
    assert ok.all(), np.argwhere(~ok)[:3]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-36, 1e-30, 1e-6])
@pytest.mark.parametrize("heads,d", [(5, 64), (3, 72), (2, 256), (9, 8)])
def test_small_rows(heads, d, eps, bf16):
    """Rows whose squares leave float's range below: the definition is of size 1 where eps is less than their mean square.  Rows of ordinary size share
    their waves."""
    print("small", heads, d, eps, bf16, flush=True)
    g = torch.Generator().manual_seed(d)
    eps = float(np.float32(eps))
    size = 10.0 ** torch.tensor([-16.0, -19.0, -20.0, -23.0, -30.0, 0.0, -37.0])
    x = (torch.randn(1, 7, heads, d, generator=g) * size[None, :, None, None]).to(TYPES[bf16]).to(DEV)
    x[0, 3, 0], x[0, 4, heads - 1] = 1.0, -3.0
    got, _ = df.qk_norm_rope(x, eps=eps)
    ref, terms = bo.qk_norm_rope(host(x), eps=eps)
    _near(got, ref, terms, bf16)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("heads,d", [(5, 64), (3, 72), (2, 256), (9, 8)])
def test_large_rows(heads, d, bf16):
    """Rows whose squares leave float's range above, with a value among them that is small beside theirs."""
    print("large", heads, d, bf16, flush=True)
    g = torch.Generator().manual_seed(d + 1)
    size = 10.0 ** torch.tensor([18.0, 19.0, 20.0, 30.0, 0.0, 37.5])
    x = torch.randn(1, 6, heads, d, generator=g).clamp(-3, 3) * size[None, :, None, None]
    x[..., 3] = 1e-6
    x = x.to(TYPES[bf16]).to(DEV)
    gamma = torch.linspace(0.5, 2, d)
    got, _ = df.qk_norm_rope(x, q_gamma=gamma.to(DEV))
    ref, terms = bo.qk_norm_rope(host(x), gamma.numpy())
    _near(got, ref, terms, bf16)


@pytest.mark.parametrize("bf16", [True, False])
def test_rows_of_denormal_numbers_and_of_zeros(bf16):
    x = torch.zeros(1, 3, 2, 64, dtype=TYPES[bf16])
    x[0, 0, :, :] = 2.0 ** -131                              # (a multiple of bf16's smallest number)
    x[0, 1, 0, 5] = -2.0 ** -133
    x = x.to(DEV)
    got, _ = df.qk_norm_rope(x, eps=0.0)
    assert torch.equal(got[0, 0], torch.ones_like(got[0, 0])) and got[0, 1, 0, 5] == -8 and got[0, 1, 0].count_nonzero() == 1
    assert got[0, 1, 1].isnan().all() and got[0, 2].isnan().all()                    # 0 / 0
    assert not df.qk_norm_rope(x, eps=1e-6)[0][0, 2].any()


@pytest.mark.parametrize("inter", [True, False])
@pytest.mark.parametrize("bf16", [True, False])
def test_a_token_that_is_not_rotated_keeps_its_bits(bf16, inter):
    """A negative position: no value depends on its partner, be that infinite or no number; zeros keep their sign."""
    d, rot = 64, 32
    x = torch.randn(1, 4, 3, d, generator=torch.Generator().manual_seed(2)).to(TYPES[bf16]).to(DEV)
    x[..., 3], x[..., 20], x[..., 6] = float("inf"), float("nan"), -0.0
    a = np.random.default_rng(1).uniform(0, 6, (2, rot // 2))
    table = torch.from_numpy(np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)).to(DEV)
    pos = torch.tensor([[-1, 1, -7, 2]], dtype=torch.int32, device=DEV)
    got, _ = df.qk_norm_rope(x, rot=table, pos=pos, norm=False, interleaved=inter)
    bits = torch.int16 if bf16 else torch.int32
    for t in (0, 2):
        number = ~x[0, t].isnan()                            # (what a NaN's bits are is nobody's promise)
        assert torch.equal(got[0, t].view(bits)[number], x[0, t].view(bits)[number]) and got[0, t][~number].isnan().all()
    assert got[0, 3, :, :rot].isnan().all() and not torch.equal(got[0, 1, :, :rot], x[0, 1, :, :rot])
    assert torch.equal(got[0, 3, :, rot:], x[0, 3, :, rot:])
