"""Performance cases of the operators of a displaced-patch transformer block: what a user of the library calls between the projections.

A diffusion transformer's block on one patch normalises the queries and keys of its fused projection per head and rotates
them by position (`qk_norm_rope`), keeps the keys and values of the whole image in 4 bits between the steps (`kv4_refresh`,
`kv4_read`), attends to them with its own rows spliced in fresh (`attn_displaced_kv4`, `attn_kv4` where every row is in the
cache), and attends to the states of an encoder of another length, padded prompts among them (`cross_attn`).

Kinds of cases
  rope    norm and rotation of the queries and keys of a fused projection
  cache   refresh of a patch's rows of a 4-bit cache, and the cache read back
  attn4   attention over a 4-bit cache, or displaced attention with the patch's own rows fresh
  cross   attention to an encoder's states
"""
import math

import torch

own = False     # False: the plain form, elementary torch operations in 32 bits; True: the calls of the library

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token of a cached sequence: nothing but latency
        dict(name="rope_token", kind="rope", B=1, T=1, heads=20, kv_heads=20, d=64, rot=64, style="interleaved", norm=True, pos=False,
             dtype="bf16"),
        # the middle level's patch of a 1280x1920 image over 8 patches, both guidance branches
        dict(name="rope_patch", kind="rope", B=2, T=1200, heads=10, kv_heads=10, d=64, rot=64, style="halves", norm=True, pos=False, dtype="bf16"),
        # the coarsest level's tokens of a whole 3840x3840 image and one more, shared key heads, positions given (prompt tokens are not rotated), in
        # full precision
        dict(name="rope_long_f32", kind="rope", B=1, T=14401, heads=20, kv_heads=4, d=128, rot=96, style="interleaved", norm=True, pos=True,
             dtype="f32"),
        # the coarsest level's patch of a 1280x1920 image over 8 patches: 300 rows into a cache of 2400
        dict(name="cache_300_of_2400", kind="cache", B=1, H=30, W=80, N=8, patch=3, axis="rows", kv_heads=20, d=64, dtype="bf16"),
        # a vertical strip of a 2048x2048 image over 4 strips, odd edges, heads of 128
        dict(name="cache_strips", kind="cache", B=1, H=128, W=124, N=4, patch=1, axis="cols", kv_heads=10, d=128, dtype="bf16"),
        # one query per sequence against short caches, shared key heads: latency
        dict(name="attn4_token", kind="attn4", mode="cached", B=4, Lq=1, H=1, W=1037, heads=20, kv_heads=5, d=64, lens=True, dtype="bf16"),
        # one query against the longest cache: the cache's bytes
        dict(name="attn4_token_long", kind="attn4", mode="cached", B=4, Lq=1, H=1, W=57600, heads=20, kv_heads=20, d=64, lens=False, dtype="bf16"),
        # displaced self-attention of the benchmark's patch: 1280x1920 over 8 patches, middle level
        dict(name="attn4_1200_of_9600", kind="attn4", mode="displaced", B=1, H=80, W=120, N=8, patch=3, axis="rows", heads=10, kv_heads=10, d=64,
             dtype="bf16"),
        # the same of 3840x3840 over 8 patches, the largest image
        dict(name="attn4_7200_of_57600", kind="attn4", mode="displaced", B=1, H=240, W=240, N=8, patch=3, axis="rows", heads=10, kv_heads=10, d=64,
             dtype="bf16"),
        # a patch's cross-attention to two prompts of 77 tokens, padded
        dict(name="cross_300x77", kind="cross", B=2, Lq=300, Lk=77, heads=20, kv_heads=20, d=64, mask="lens", dtype="bf16"),
        # the tokens of a 2048x2048 image against a long prompt with holes, heads of 128 that share keys
        dict(name="cross_16384x512", kind="cross", B=1, Lq=16384, Lk=512, heads=16, kv_heads=8, d=128, mask="mask", dtype="bf16"),
        # full precision, a small network's heads
        dict(name="cross_f32", kind="cross", B=1, Lq=1200, Lk=333, heads=8, kv_heads=8, d=32, mask="none", dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["rope", "rope", "cache", "cache", "attn4", "attn4", "attn4", "cross", "cross", "cross"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 64, 128])
    kv_heads = rng.choice([2, 5, 8, 10, 20])
    heads = kv_heads * rng.choice([1, 1, 2, 4] if kv_heads < 10 else [1, 1, 2])
    B = rng.choice([1, 1, 2, 4])
    N = rng.choice([2, 4, 8])
    axis = rng.choice(["rows", "rows", "cols"])
    if kind == "rope":
        d = rng.choice([64, 64, 72, 96, 128])
        return dict(kind=kind, B=B, T=_log(rng, 1, 20000), heads=heads, kv_heads=kv_heads, d=d, rot=rng.choice([d, d, d // 2 // 8 * 8]),
                    style=rng.choice(["interleaved", "halves"]), norm=rng.random() < 0.8, pos=rng.random() < 0.3, dtype=dtype)
    if kind == "cache" or (kind == "attn4" and rng.random() < 0.5):
        part, other = _log(rng, 1, 40), _log(rng, 5, 240)
        H, W = (part * N, other) if axis == "rows" else (other, part * N)
        c = dict(kind=kind, B=B, H=H, W=W, N=N, patch=rng.randrange(N), axis=axis, kv_heads=kv_heads, d=d, dtype=dtype)
        return c if kind == "cache" else dict(c, mode="displaced", heads=heads)
    if kind == "attn4":
        return dict(kind=kind, mode="cached", B=B, Lq=rng.choice([1, 1, 1, 2, _log(rng, 2, 64), _log(rng, 64, 2048)]), H=1, W=_log(rng, 1, 60000), heads=heads,
                    kv_heads=kv_heads, d=d, lens=rng.random() < 0.5, dtype=dtype)
    return dict(kind=kind, B=B, Lq=rng.choice([1, _log(rng, 1, 20000), _log(rng, 64, 20000)]), Lk=_log(rng, 1, 4096), heads=heads, kv_heads=kv_heads,
                d=rng.choice([32, 40, 64, 64, 72, 128]), mask=rng.choice(["none", "lens", "mask"]), dtype=dtype)


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        # full precision runs at a tenth of the rate; nothing costs more than the largest listed case
        if w["flops"] * (10 if c["dtype"] == "f32" else 1) <= 1e12 and w["bytes"] <= 3.6e8:
            return c


def _tokens(c):
    """(queries, rows of the cache)"""
    L = c["H"] * c["W"]
    return (L // c["N"] if c.get("mode") != "cached" else c["Lq"]), L


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    B, d = c["B"], c["d"]
    if c["kind"] == "rope":
        n = B * c["T"] * (c["heads"] + c["kv_heads"]) * d
        return dict(bytes=2 * n * e + c["T"] * c["rot"] * 4 + (4 * B * c["T"] if c["pos"] else 0), flops=n * 8)
    if c["kind"] == "cache":
        T, L = _tokens(c)
        row = 2 * (d // 2 + 2)                               # codes and scale of a key and a value
        fresh, rows = B * T * c["kv_heads"], B * L * c["kv_heads"]
        return dict(bytes=fresh * (2 * d * e + row) + rows * (row + 2 * d * e), flops=fresh * d * 8 + rows * d * 2)
    if c["kind"] == "attn4":
        T, L = _tokens(c)
        io = 2 * B * T * c["heads"] * d * e
        seen = 0.75 * L if c.get("lens") else L
        fresh = T if c["mode"] == "displaced" else 0
        return dict(bytes=int(io + B * c["kv_heads"] * ((seen - fresh) * 2 * (d // 2 + 2) + fresh * 2 * d * e)),
                    flops=int(4 * B * c["heads"] * T * seen * d))
    seen = c["Lk"] * (1 if c["mask"] == "none" else 0.75)
    return dict(bytes=int(2 * B * c["Lq"] * c["heads"] * d * e + 2 * B * seen * c["kv_heads"] * d * e),
                flops=int(4 * B * c["heads"] * c["Lq"] * seen * d))


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=g, device=DEV) * std + mean


def _lengths(g, B, L):
    """Between half of the rows and all of them"""
    return (L - (torch.rand(B, generator=g, device=DEV) * (L / 2)).floor()).clamp(min=1).to(torch.int32)


def _angles(T, half):
    """Angles of T positions of a sequence, 64 bits"""
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / max(half, 1))
    return torch.arange(T, dtype=torch.float64, device=DEV)[:, None] * freq


def _inputs(case, seed):
    """The tensors of a case, as a user's program has them from its projections"""
    c, g, dt = case, _generator(seed), DTYPES[case["dtype"]]
    B, d = c["B"], c["d"]
    if c["kind"] == "rope":
        T, hq, hk = c["T"], c["heads"], c["kv_heads"]
        qkv = _normal(g, B, T, (hq + 2 * hk) * d, std=1.5).to(dt)
        s = dict(q=qkv[..., :hq * d].unflatten(-1, (hq, d)), k=qkv[..., hq * d:(hq + hk) * d].unflatten(-1, (hk, d)))
        if c["norm"]:
            s["q_gamma"], s["k_gamma"] = _normal(g, d, std=0.1, mean=1.0), _normal(g, d, std=0.1, mean=1.0)
        a = _angles(T, c["rot"] // 2)
        s["rot"] = torch.stack((a.cos(), a.sin()), -1).float().contiguous()
        if c["pos"]:                                         # the first tenth are prompt tokens, which are not rotated
            s["pos"] = torch.randint(T, (B, T), generator=g, device=DEV).to(torch.int32)
            s["pos"][:, :T // 10] = -1
        return s
    if c["kind"] == "cross":
        hq, hk = c["heads"], c["kv_heads"]
        kv = _normal(g, B, c["Lk"], 2 * hk * d).to(dt)       # one projection gives both
        s = dict(q=_normal(g, B, c["Lq"], hq, d, std=1.5).to(dt), k=kv[..., :hk * d].unflatten(-1, (hk, d)), v=kv[..., hk * d:].unflatten(-1, (hk, d)))
        if c["mask"] == "lens":
            s["lens"] = _lengths(g, B, c["Lk"])
        if c["mask"] == "mask":
            s["key_mask"] = torch.rand(B, c["Lk"], generator=g, device=DEV) < 0.75
        return s
    T, L = _tokens(c)
    hk = c["kv_heads"]
    spread = 0.5 + torch.rand(hk, d, generator=g, device=DEV)             # features of different size
    k, v = _normal(g, B, L, hk, d) * spread, _normal(g, B, L, hk, d)
    s = dict(k_all=k.to(dt), v_all=v.to(dt))
    if c["kind"] == "cache" or c["mode"] == "displaced":     # the patch's own rows a denoising step later
        rows = _own_rows(c)
        kf, vf = k[:, rows], v[:, rows]
        s["k_fresh"] = (kf + _normal(g, *kf.shape, std=0.02)).to(dt)
        s["v_fresh"] = (vf + _normal(g, *vf.shape, std=0.02)).to(dt)
    if c["kind"] == "attn4":
        s["q"] = _normal(g, B, T, c["heads"], d, std=1.5).to(dt)
        if c.get("lens"):
            s["lens"] = _lengths(g, B, L)
    return s


def _own_rows(c):
    """Rows of the cache that the patch owns, in its order"""
    j = torch.arange(c["H"] * c["W"], device=DEV)
    if c["axis"] == "rows":
        n = c["H"] * c["W"] // c["N"]
        return j[c["patch"] * n:(c["patch"] + 1) * n]
    w = c["W"] // c["N"]
    return j[(j % c["W"]) // w == c["patch"]]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] in ("cache", "attn4"):
        k, v = s.pop("k_all"), s.pop("v_all")
        if own:
            import paper_2402_19481_amd as df
            B, L, hk, d = k.shape
            s["cache"] = df.kv4_cache(B, L, hk, d, device=k.device)
            df.kv4_refresh(s["cache"], k, v, 0, 1)
        else:
            s["kq"], s["vq"] = _plain_quantise(k), _plain_quantise(v)
            if "N" in case:
                s["rows"] = _own_rows(case)
    return s


# ---- plain forms ----

def _plain_quantise(x):
    """x [..., d] -> two e2m1 codes per byte, and the scale of each row: a sixth of its largest magnitude to six significant bits.
    A quotient next to a border between two codes decides in 64 bits."""
    x = x.double()
    most = x.abs().amax(-1, keepdim=True)
    mant, ex = torch.frexp(most / 6)
    scale = torch.ldexp((mant * 64).round(), ex - 6).clamp(max=1.3125 * 2.0 ** 125)
    scale = torch.where(most < 2.0 ** -100, torch.zeros_like(scale), scale)
    scale = torch.where(most.isfinite(), scale, torch.full_like(scale, float("nan")))
    a = torch.where(scale > 0, x.abs() / scale, torch.zeros_like(x))
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = code | ((x < 0).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.float()


def _plain_values(q):
    """Codes and scales -> float"""
    code, scale = q
    both = torch.stack((code & 15, code >> 4), -1).flatten(-2).long()
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return level[both] * scale


def _plain_attention(q, k, v, valid, dtype):
    """q [B, Lq, heads, d], k, v [B, L, kv_heads, d] in 32 bits, valid [B, L] or None; a row without keys gives zeros"""
    B, Lq, hq, d = q.shape
    L, hk = k.shape[1], k.shape[2]
    out = torch.empty(B, Lq, hq, d, dtype=dtype, device=q.device)
    if valid is not None:
        k = torch.where(valid[:, :, None, None], k, torch.zeros_like(k))
        v = torch.where(valid[:, :, None, None], v, torch.zeros_like(v))
    per = max(1, min(hk, (1 << 28) // max(1, Lq * L * (hq // hk))))       # key heads at a time
    rows = max(1, min(Lq, (1 << 28) // max(1, per * L * (hq // hk))))
    for b in range(B):
        for h in range(0, hk, per):
            n = min(per, hk - h)
            kk, vv = k[b, :, h:h + n].permute(1, 2, 0).contiguous(), v[b, :, h:h + n].permute(1, 0, 2).contiguous()
            for r in range(0, Lq, rows):
                qq = q[b, r:r + rows, h * (hq // hk):(h + n) * (hq // hk)]
                m = qq.shape[0]
                qq = qq.unflatten(1, (n, hq // hk)).permute(1, 2, 0, 3).reshape(n, hq // hk * m, d).contiguous()
                s = torch.matmul(qq, kk) * d ** -0.5
                if valid is not None:
                    s = s.masked_fill(~valid[b], -math.inf)
                    top = s.amax(-1, keepdim=True)
                    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                else:
                    top = s.amax(-1, keepdim=True)
                p = torch.exp(s - top)
                o = torch.matmul(p, vv) / p.sum(-1, keepdim=True)
                if valid is not None:
                    o = torch.where(valid[b].any(), o, torch.zeros_like(o))
                out[b, r:r + rows, h * (hq // hk):(h + n) * (hq // hk)] = o.view(n, hq // hk, m, d).permute(2, 0, 1, 3).reshape(m, -1, d).to(dtype)
    return out


def _plain_rope(x, gamma, s, c):
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * gamma
    n, rot = c["rot"], s["rot"]
    if "pos" in s:
        t = rot[s["pos"].clamp(min=0).long()]
        t = torch.where((s["pos"] < 0)[..., None, None], torch.tensor([1.0, 0.0], device=t.device), t)[:, :, None]
    else:
        t = rot[None, :x.shape[1], None]
    cos, sin = t[..., 0], t[..., 1]
    r = y[..., :n]
    if c["style"] == "interleaved":
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = r[..., :n // 2], r[..., n // 2:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((r, y[..., n:]), -1).to(x.dtype)


def _valid(s, L):
    if "lens" in s:
        return torch.arange(L, device=DEV)[None, :] < s["lens"][:, None]
    return s.get("key_mask")


def _run_plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "rope":
        return _plain_rope(s["q"], s.get("q_gamma"), s, c), _plain_rope(s["k"], s.get("k_gamma"), s, c)
    if c["kind"] == "cross":
        return _plain_attention(s["q"].float(), s["k"].float(), s["v"].float(), _valid(s, c["Lk"]), dt)
    if c["kind"] == "cache":
        for name in "kv":
            code, scale = _plain_quantise(s[name + "_fresh"])
            s[name + "q"][0][:, s["rows"]] = code
            s[name + "q"][1][:, s["rows"]] = scale
        return _plain_values(s["kq"]).to(dt), _plain_values(s["vq"]).to(dt)
    k, v = _plain_values(s["kq"]), _plain_values(s["vq"])
    if c["mode"] == "displaced":
        k[:, s["rows"]] = s["k_fresh"].float()
        v[:, s["rows"]] = s["v_fresh"].float()
    return _plain_attention(s["q"].float(), k, v, _valid(s, k.shape[1]), dt)


# ---- the library's calls ----

def _run_own(s):
    import paper_2402_19481_amd as df
    c = s["case"]
    if c["kind"] == "rope":
        return df.qk_norm_rope(s["q"], s["k"], s.get("q_gamma"), s.get("k_gamma"), s["rot"], s.get("pos"), eps=1e-6, norm=c["norm"],
                               interleaved=c["style"] == "interleaved")
    if c["kind"] == "cross":
        return df.cross_attn(s["q"], s["k"], s["v"], key_mask=s.get("key_mask"), lens=s.get("lens"))
    if c["kind"] == "cache":
        if c["axis"] == "rows":
            df.kv4_refresh(s["cache"], s["k_fresh"], s["v_fresh"], c["patch"], c["N"])
        else:
            df.kv4_refresh_cols(s["cache"], s["k_fresh"], s["v_fresh"], c["H"], c["W"], c["patch"], c["N"])
        return df.kv4_read(s["cache"], c["B"], c["H"] * c["W"], c["kv_heads"], c["d"], dtype=DTYPES[c["dtype"]])
    if c["mode"] == "cached":
        return df.attn_kv4(s["q"], s["cache"], c["H"] * c["W"], c["kv_heads"], lens=s.get("lens"))
    if c["axis"] == "rows":
        return df.attn_displaced_kv4(s["q"], s["k_fresh"], s["v_fresh"], s["cache"], c["patch"], c["N"])
    return df.attn_displaced_kv4_cols(s["q"], s["k_fresh"], s["v_fresh"], s["cache"], c["H"], c["W"], c["patch"], c["N"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definition in 64 bits ----

def _exact_held(x):
    """What a cache holds of x [..., d]: the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 scales for each value (of two equally near ones the
    one whose number in this list is even), with its sign"""
    x = x.double()
    most = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(most / 6))
    step = torch.exp2(e - 5)                                 # six significant bits: 32 .. 63 steps
    n = torch.round(most / 6 / step)
    scale = torch.where(most > 0, n * step, torch.zeros_like(n))
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    best, held = torch.full_like(x, math.inf), torch.zeros_like(x)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                       # even numbers first: they keep a tie
        off = (x.abs() - level[i] * scale).abs()
        held = torch.where(off < best, level[i] * scale, held)
        best = torch.minimum(best, off)
    return held * torch.sign(x)


def _exact_attention(q, k, v, valid):
    q, out = q.double(), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    B, Lq, hq, d = q.shape
    group = hq // k.shape[2]
    step = max(1, (1 << 27) // max(1, k.shape[1]))
    for b in range(B):
        keep = slice(None) if valid is None else valid[b].nonzero()[:, 0]
        kb, vb = k[b, keep].double(), v[b, keep].double()
        if kb.shape[0] == 0:
            continue
        for h in range(hq):
            kh, vh = kb[:, h // group].t().contiguous(), vb[:, h // group].contiguous()
            for r in range(0, Lq, step):
                w = torch.softmax(torch.mm(q[b, r:r + step, h].contiguous(), kh) / math.sqrt(d), -1)
                out[b, r:r + step, h] = torch.mm(w, vh)
    return out


def _exact_rope(x, gamma, s, c):
    y = x.double()
    if c["norm"]:
        y = y / (y.pow(2).sum(-1, keepdim=True) / c["d"] + 1e-6).sqrt() * gamma.double()
    B, T = x.shape[:2]
    n = c["rot"] // 2
    table = s["rot"].double()
    p = s["pos"].long() if "pos" in s else torch.arange(T, device=x.device).expand(B, T)
    turn = torch.view_as_complex(table[p.clamp(min=0)].contiguous())
    turn = torch.where((p < 0)[..., None], torch.ones_like(turn), turn)[:, :, None]
    first = torch.arange(n, device=x.device) * (2 if c["style"] == "interleaved" else 1)
    second = first + (1 if c["style"] == "interleaved" else n)
    z = torch.complex(y[..., first], y[..., second]) * turn
    y = y.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "rope":
        return _exact_rope(s["q"], s.get("q_gamma"), s, c), _exact_rope(s["k"], s.get("k_gamma"), s, c)
    if c["kind"] == "cross":
        return _exact_attention(s["q"], s["k"], s["v"], _valid(s, c["Lk"]))
    k, v = _exact_held(s["k_all"]), _exact_held(s["v_all"])
    if c["kind"] == "cache":
        rows = _own_rows(c)
        k[:, rows], v[:, rows] = _exact_held(s["k_fresh"]), _exact_held(s["v_fresh"])
        return k, v
    if c["mode"] == "displaced":
        rows = _own_rows(c)
        k[:, rows], v[:, rows] = s["k_fresh"].double(), s["v_fresh"].double()
    return _exact_attention(s["q"], k, v, _valid(s, k.shape[1]))
