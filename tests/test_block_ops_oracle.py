"""The 64-bit forms of the block's operators against brute force and hand cases (no GPU)."""
import numpy as np
import pytest

from oracle import block_ops as bo


def test_rotation_turns_pairs_and_keeps_lengths():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((1, 3, 2, 8))
    a = rng.uniform(0, 6, (3, 4))
    rot = np.stack((np.cos(a), np.sin(a)), -1)
    for inter in (True, False):
        y, _ = bo.qk_norm_rope(x, rot=rot, norm=False, interleaved=inter)
        i = np.arange(4)
        f, s = (2 * i, 2 * i + 1) if inter else (i, i + 4)
        z = (x[..., f] + 1j * x[..., s]) * np.exp(1j * a)[None, :, None]
        np.testing.assert_allclose(y[..., f] + 1j * y[..., s], z, rtol=1e-13)
    y, _ = bo.qk_norm_rope(x, np.full(8, 2.0), eps=0.0)
    np.testing.assert_allclose((y * y).mean(-1), 4.0, rtol=1e-13)
    y, _ = bo.qk_norm_rope(x, rot=rot, pos=np.array([[-1, 0, 3]]), norm=False)
    assert np.array_equal(y[0, 0], x[0, 0]) and np.isnan(y[0, 2]).all()


@pytest.mark.parametrize("row,held", [
    ([6, 0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5], [6, 0, 1, 1, -2, 2, 4, 4]),        # scale 1: every tie
    ([0, 0, 0, 0], [0, 0, 0, 0]),
    ([7, 1, -1, 0], [6 * 37 / 32, 37 / 32, -37 / 32, 0]),                          # 7 / 6 = 37.33 / 32
])
def test_levels(row, held):
    assert bo.held_in_4_bits(np.array(row, float)).tolist() == held


def test_held_rows_are_exact_in_bf16_and_near():
    x = np.random.default_rng(1).standard_normal((50, 64)) * 10.0 ** np.random.default_rng(2).uniform(-20, 20, (50, 1))
    y = bo.held_in_4_bits(x)
    bits = y.astype(np.float32).view(np.uint32)
    assert np.array_equal(y.astype(np.float32).astype(np.float64), y) and not (bits & 0xffff).any()
    assert (np.abs(y - x) <= np.abs(x).max(-1, keepdims=True) * (1 / 6 + 1 / 32)).all()


def test_attention_is_a_mean_of_the_valid_values():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 3, 4, 8)), rng.standard_normal((2, 5, 2, 8)), rng.standard_normal((2, 5, 2, 8))
    valid = np.array([[1, 0, 1, 1, 0], [0, 0, 0, 0, 0]], bool)
    out, size, _ = bo.attention(q, k, v, 0.3, valid)
    assert not out[1].any()
    for i in range(3):
        for h in range(4):
            w = np.array([np.exp(0.3 * q[0, i, h] @ k[0, j, h // 2]) if valid[0, j] else 0.0 for j in range(5)])
            np.testing.assert_allclose(out[0, i, h], (w[:, None] * v[0, :, h // 2]).sum(0) / w.sum(), rtol=1e-12)
