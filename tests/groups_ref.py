"""Plain forms of the operators on 4-bit groups, written from their formulas (tests only)."""
import math

import numpy as np
import torch

GROUP, TILE = 64, 16


def bf16_bits(x):
    """binary32 to bf16, half to even, as uint16 patterns."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7fc0), r)


def bf16_values(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


def quantise(bits, group):
    """uint16 bf16 patterns [..., n] to (codes uint8 [..., n], (scale, low) patterns uint16 [..., n / group, 2]): binary32 step by step."""
    with np.errstate(all="ignore"):
        x = bf16_values(bits)
        x = x.reshape(*x.shape[:-1], -1, group)
        low, top = x.min(-1) + np.float32(0), x.max(-1)
        span = (top - low).astype(np.float32)
        scale = bf16_values(bf16_bits((span / np.float32(15)).astype(np.float32)))
        scale = np.where(scale < np.float32(2.0 ** -120), np.float32(0), scale)
        inv = np.where(scale > 0, np.float32(1) / np.where(scale > 0, scale, np.float32(1)), np.float32(0)).astype(np.float32)
        t = ((x - low[..., None]).astype(np.float32) * inv[..., None]).astype(np.float32)
        bad = ~np.isfinite(span)
        q = np.where(bad[..., None], 0, np.minimum(np.rint(np.where(bad[..., None], 0, t)), 15)).astype(np.uint8)
        params = np.stack([bf16_bits(scale), bf16_bits(low)], -1)
        params[bad] = 0x7fc0
    return q.reshape(bits.shape), params


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def tile_half(codes, params):
    """Codes [16, D] and groups [16, D / 64, 2] of a tile's keys (or values) as bytes, one slot and element at a time."""
    D = codes.shape[1]
    out = np.zeros(9 * D, np.uint8)
    for s in range(TILE):
        for e in range(D):
            out[(e // 32) * 256 + s * 16 + (e % 32) // 2] |= codes[s, e] << (4 * (e % 2))
        for i in range(D // GROUP):
            out[8 * D + i * 64 + s * 4:8 * D + i * 64 + s * 4 + 4] = np.ascontiguousarray(params[s, i]).view(np.uint8)
    return out


def cache_bytes(k_bits, v_bits):
    """bf16 patterns [pages, heads, page, D] of keys and values to the cache's bytes [pages, heads, page / 16, 18 D]."""
    out = []
    for bits in (k_bits, v_bits):
        D = bits.shape[-1]
        c, p = quantise(bits, GROUP)
        c = pack(c).reshape(*c.shape[:2], -1, TILE, D // 32, 16)
        p = np.ascontiguousarray(p).view(np.uint8).reshape(*p.shape[:2], -1, TILE, D // GROUP, 4)
        out += [np.moveaxis(c, 4, 3).reshape(*c.shape[:3], 8 * D), np.moveaxis(p, 4, 3).reshape(*p.shape[:3], D)]
    return np.concatenate(out, -1)


def cache_values(tiles):
    """The cache's bytes to (k, v, middle of v's groups, 15 scale + |low| and low of k's) in 64 bits, [pages, heads, page, D] each; the middle of a group is low + 8 scale."""
    tiles = np.asarray(tiles)
    D = tiles.shape[-1] // 18
    out = []
    for at in (0, 9 * D):
        c = tiles[..., at:at + 8 * D].reshape(*tiles.shape[:3], D // 32, TILE, 16)
        c = np.stack([c & 15, c >> 4], -1).reshape(*tiles.shape[:3], D // 32, TILE, 32)
        c = np.moveaxis(c, 3, 4).reshape(*tiles.shape[:3], TILE, D).astype(np.float64)
        p = np.ascontiguousarray(tiles[..., at + 8 * D:at + 9 * D]).view(np.uint16).reshape(*tiles.shape[:3], D // GROUP, TILE, 2)
        p = np.repeat(np.moveaxis(bf16_values(p).astype(np.float64), 3, 4), GROUP, axis=4)
        shape = (*tiles.shape[:2], -1, D)
        with np.errstate(all="ignore"):
            out.append(((c * p[..., 0] + p[..., 1]).reshape(shape), (8 * p[..., 0] + p[..., 1]).reshape(shape), (15 * p[..., 0] + np.abs(p[..., 1])).reshape(shape),
                        np.broadcast_to(p[..., 1], c.shape).reshape(shape)))
    (k, _, k_size, k_low), (v, mid, _, _) = out
    return tuple(torch.from_numpy(np.ascontiguousarray(x)) for x in (k, v, mid, k_size, k_low))


def gemv(codes, params, x):
    """(y in 64 bits, bound on an fp32 result's error).  A product of the tensor cores is exact; each of the sums that follow (8 steps of 16 products in a group, the
    groups of a row, the join of warps, slots and CTAs) is off by 2^-23 of the terms' magnitudes at most: 2^-23 (8 + groups of a row + 40) of them."""
    group = codes.shape[1] // params.shape[1]
    s, low = (torch.from_numpy(bf16_values(params[..., i]).astype(np.float64)) for i in (0, 1))
    c = torch.from_numpy(codes.astype(np.float64)).unflatten(1, (-1, group))
    x = x.double().cpu()
    W = (c * s[..., None] + low[..., None]).flatten(1)
    size = (c * s[..., None] + low.abs()[..., None]).flatten(1)
    return x @ W.t(), 2.0 ** -23 * (48 + params.shape[1]) * (x.abs() @ size.t()) + 1e-37


def gemm(codes, params, x, bf16_out=False):
    """gemv's for the call for many tokens.  Products are exact: scale (code - 8) of 11 bits with x, (low + 8 scale) with the group's sum of x.  Sums in tensor memory are cut
    off: 2^-23 of the terms' magnitudes a step, twice that with what a step's sixteen products lose to one another, for 64 steps (1024 columns), or with bf16 outputs for all of the
    row's; eight more additions per group's sum, which is then held in 22 bits, and those of the segments.  Beside that, what is far below a row's largest group (2^-35 of it: a scale off by half a step of fp16, times 8) or a
    token's largest element (2^-31) is rounded to such a step."""
    group = codes.shape[1] // params.shape[1]
    K = codes.shape[1]
    s, low = (torch.from_numpy(bf16_values(params[..., i]).astype(np.float64)) for i in (0, 1))
    c = torch.from_numpy(codes.astype(np.float64)).unflatten(1, (-1, group))
    x = x.double().cpu()
    W = (c * s[..., None] + low[..., None]).flatten(1)
    size = ((c - 8).abs() * s[..., None] + low.abs()[..., None] + 8 * s[..., None]).flatten(1)
    terms = x.abs() @ size.t()
    steps = (K + 4 * params.shape[1]) / 16 + 8 if bf16_out else 72 + K / 1024
    top = torch.maximum(low.abs(), 8 * s).amax(1)
    small = 2.0 ** -35 * x.abs().sum(1)[:, None] * top[None] + 2.0 ** -31 * x.abs().amax(1)[:, None] * size.sum(1)[None]
    return x @ W.t(), (2.0 ** -22 * steps + 2.0 ** -20) * terms + small + 1e-37


def attn(q, tiles, table, cu, kv_len, scale, softcap=0.0, window=0, longest=None):
    """(out, bound) in 64 bits, one query row at a time over the keys it sees.  The output is rounded to 8 bits.  A score is off by 2^-20 of
    sum_d |q_d| (15 scale + |low|) at most (a few dozen fp32 steps) and, where queries are taken as 16-bit integers (calls of up to four rows: the longest sequence's bound times the heads of a group), by 2^-15 of the
    largest |q_d| times sum_d scale code_d, which moves weights by a factor.  p * scale is rounded to 8 bits beside code - 8 (2^-8 of sum_j p_j |v_j - middle_j|; with
    up to four rows to 16).  Calls of more than 16 rows may be served in fp16: queries, keys, values and weights are off by 2^-11 of themselves each; the larger of the two bounds
    is taken.  Sums in 32 bits add well under 2^-12 of their terms."""
    T, Hq, D = q.shape
    k_all, v_all, mid_all, size_all, low_all = cache_values(tiles)
    Hkv, ps = k_all.shape[1], k_all.shape[2]
    G = Hq // Hkv
    rows = (T if longest is None else longest) * G
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    tol = torch.zeros_like(out)
    q = q.cpu().double()
    for b in range(len(cu) - 1):
        n, L = cu[b + 1] - cu[b], kv_len[b]
        if n <= 0 or L <= 0:
            continue
        j = torch.arange(L)
        pages = table[b].cpu().long()[j // ps]
        k, v, mid, size, low = (t[pages, :, j % ps] for t in (k_all, v_all, mid_all, size_all, low_all))
        for i in range(n):
            p = L - n + i
            if p < 0:
                continue
            lo = max(0, p - window + 1) if window else 0
            qi = q[cu[b] + i].view(Hkv, G, D)
            s = torch.einsum("hgd,jhd->hgj", qi, k[lo:p + 1]) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            w = torch.softmax(s, -1)
            vs = v[lo:p + 1]
            o = torch.einsum("hgj,jhd->hgd", w, vs)
            spread = torch.einsum("hgj,jhd->hgd", w, vs.abs())
            moved = torch.einsum("hgj,jhd->hgd", w, vs.abs()) + o.abs()
            off = 2.0 ** -20 * scale * torch.einsum("hgd,jhd->hgj", qi.abs(), size[lo:p + 1]).amax(-1, keepdim=True)
            if rows <= 4:
                off = off + 2.0 ** -15 * scale * qi.abs().amax(-1, keepdim=True) * (k[lo:p + 1] - low[lo:p + 1]).sum(-1).amax(0)[:, None, None]
            if rows > 16:
                off = torch.maximum(off, 2.0 ** -10 * scale * torch.einsum("hgd,jhd->hgj", qi.abs(), k[lo:p + 1].abs()).amax(-1, keepdim=True))
            from_weights = 2.0 ** (-8 if rows <= 4 else 0) * torch.einsum("hgj,jhd->hgd", w, (vs - mid[lo:p + 1]).abs())
            if rows > 16:
                from_weights = torch.maximum(from_weights, 2.0 ** -2 * spread)
            bound = 2.0 ** -8 * o.abs() + 2.0 ** -8 * from_weights + 2.0 ** -12 * (spread + from_weights) + torch.expm1(2 * off) * moved + 1e-30
            out[cu[b] + i], tol[cu[b] + i] = o.reshape(Hq, D), bound.reshape(Hq, D)
    return out, tol


def make_cache(lens, Hkv, D, ps, seed, spare=3, fill=None):
    """Random pages for sequences of the given lengths: (k patterns, v patterns, table).  Slots past a sequence's end and spare pages hold ``fill`` (default: noise)."""
    rng = np.random.default_rng(seed)
    need = [math.ceil(L / ps) for L in lens]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    table = torch.full((len(lens), max(need + [1]) + 1), -7, dtype=torch.int32)
    k, v = (bf16_bits(rng.standard_normal((n_pages, Hkv, ps, D), dtype=np.float32)) for _ in range(2))
    used = np.zeros((n_pages, ps), bool)
    at = 0
    for b, L in enumerate(lens):
        for i in range(need[b]):
            page = int(order[at]); at += 1
            table[b, i] = page
            used[page, :min(ps, L - i * ps)] = True
    if fill is not None:
        for t in (k, v):
            np.moveaxis(t, 2, 1)[~used] = fill
    return k, v, table
