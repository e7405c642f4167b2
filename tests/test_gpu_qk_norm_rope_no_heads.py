"""Keys without a head are refused: None says that there are no keys."""
import pytest
import torch

import paper_2402_19481_amd as df
from gpu_util import DEV


@pytest.mark.gpu
def test_keys_without_heads():
    q = torch.ones(2, 3, 4, 64, device=DEV)
    with pytest.raises(ValueError):
        df.qk_norm_rope(q, q[:, :, :0])
    with pytest.raises(ValueError):
        df.qk_norm_rope(q, q[:, :, :0], k_out=q[:, :, :0])
    with pytest.raises(df.DfError):
        df.qk_norm_rope(q[:, :0])
    assert df.qk_norm_rope(q)[1] is None
