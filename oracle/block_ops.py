"""64-bit forms of a transformer block's operators on a patch: norm and rotation of queries and keys, keys and values held in
4 bits, attention to rows of another length.  Written from the definitions, value by value where that decides anything."""
import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def qk_norm_rope(x, gamma=None, rot=None, pos=None, eps=1e-6, norm=True, interleaved=True):
    """x [B, T, heads, d]; rot [rows, n / 2, 2]; pos [B, T] or None.  Returns (y, size of the terms each value is made of)."""
    y = np.asarray(x, dtype=np.float64).copy()
    B, T, _, d = y.shape
    if norm:
        y /= np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if gamma is not None:
            y = y * np.asarray(gamma, dtype=np.float64)
    size = np.abs(y)
    if rot is not None:
        rot = np.asarray(rot, dtype=np.float64)
        n = 2 * rot.shape[1]
        i = np.arange(n // 2)
        first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + n // 2)
        out = y.copy()
        for b in range(B):
            for t in range(T):
                at = t if pos is None else int(pos[b, t])
                if at < 0:
                    continue
                cs = rot[at] if at < rot.shape[0] else np.full((n // 2, 2), np.nan)
                p, q = y[b, t][:, first], y[b, t][:, second]
                out[b, t][:, first] = p * cs[:, 0] - q * cs[:, 1]
                out[b, t][:, second] = q * cs[:, 0] + p * cs[:, 1]
                size[b, t][:, first] = size[b, t][:, second] = np.abs(p) + np.abs(q)
        y = out
    return y, size


def held_in_4_bits(x):
    """What a cache holds of rows x [..., d]."""
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros_like(x)
    for idx in np.ndindex(x.shape[:-1]):
        row = x[idx]
        if not np.isfinite(row).all():
            out[idx] = np.nan
            continue
        most = np.abs(row).max()
        if most < 2.0 ** -100:
            continue
        m, e = np.frexp(most / 6)                            # m in [1/2, 1): six significant bits are multiples of 1/64
        scale = min(np.ldexp(np.rint(m * 64) / 64, e), 1.3125 * 2.0 ** 125)
        off = np.abs(np.abs(row)[:, None] - LEVELS * scale)
        near = off == off.min(-1, keepdims=True)             # one level, or two: then the one with the even number
        code = np.where(near.sum(-1) == 1, near.argmax(-1), np.where(near[:, ::2].any(-1), 2 * near[:, ::2].argmax(-1), 0))
        out[idx] = np.copysign(LEVELS[code] * scale, row)
    return out


def attention(q, k, v, scale, valid=None):
    """q [B, Lq, heads, d], k, v [B, L, kv_heads, d], valid [B, L] or None.  Returns (out, sum of w |v|, largest sum of |q k| scale)."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    B, Lq, heads, d = q.shape
    group = heads // k.shape[2]
    out, size, reach = np.zeros_like(q), np.zeros_like(q), 0.0
    for b in range(B):
        keep = np.arange(k.shape[1]) if valid is None else np.flatnonzero(valid[b])
        if keep.size == 0:
            continue
        for h in range(heads):
            kk, vv = k[b, keep, h // group], v[b, keep, h // group]
            s = q[b, :, h] @ kk.T * scale
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[b, :, h], size[b, :, h] = w @ vv, w @ np.abs(vv)
            reach = max(reach, float((np.abs(q[b, :, h]) @ np.abs(kk).T).max()) * scale)
    return out, size, reach


def attention_bound(out, size, reach, d, keys, bf16):
    """Largest possible error of a kernel that multiplies and adds in 32 bits, value by value.  Scores: d products and sums, the scale and the
    exponential's argument, each off by 2^-24 of at most `reach`; a score off by x moves a weight by x of itself, and the weights' sum too;
    sums over the keys by 2^-24 a term.  bf16: a weight is rounded (2^-8), and the result."""
    u = 2.0 ** -24
    score = (d + 8) * u * reach
    terms = (2 * score + (keys + 16) * u + (2.0 ** -8 if bf16 else 0.0)) * size
    return terms + (2.0 ** -8 if bf16 else 4 * u) * (np.abs(out) + terms) + 1e-30
