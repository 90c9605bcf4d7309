"""Plain 64-bit forms of the serving operators, written from their formulas (tests only)."""
import math

import numpy as np
import torch


def quantize_tokens(x_bits: np.ndarray):
    """x_bits: uint16 bf16 patterns [M, K].  The scale and the quotient are binary32 values by definition; a binary64 quotient of
    binary32 numbers rounded to binary32 is the correctly rounded binary32 quotient (53 >= 2 * 24 + 2)."""
    x = (x_bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    scale = np.maximum((np.abs(x).max(1) / 127.0).astype(np.float32), np.float32(2.0 ** -126))
    quot = (x / scale.astype(np.float64)[:, None]).astype(np.float32)
    xq = np.clip(np.rint(quot), -127, 127).astype(np.int8)
    return xq, scale, xq.astype(np.int64).sum(1).astype(np.int32)


def gemm_a8(xq, scale, q, alpha, zero, out_dtype):
    """(y in 64 bits, bound on a result's error).  The sum of products minus 128 * rowsum is an integer that is rounded to 24 bits once; the
    (z - 128) * rowsum term is rounded when z - 128 is formed, when it is multiplied and when it is subtracted; the two scales are
    multiplied and applied with one rounding each: at most six roundings of 2^-24 of the two terms' magnitudes, taken as 2^-21."""
    xd, qd = xq.double(), q.double()
    rs = xd.sum(1, keepdim=True)
    t = xd @ (qd - 128.0).t()
    u = (zero.double() - 128.0)[None, :] * rs
    f = scale.double()[:, None] * alpha.double()[None, :]
    y = f * (t - u)
    tol = 2.0 ** -21 * f.abs() * (t.abs() + u.abs())
    if out_dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * y.abs()                      # half a unit in the last of 8 bits
    return y, tol + 1e-37


def rotate(x, cos, sin, interleaved):
    """x: [T, H, D] double; cos, sin: [T, rot / 2] double."""
    half = cos.shape[1]
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y = x.clone()
    y[..., a] = x[..., a] * cos[:, None] - x[..., b] * sin[:, None]
    y[..., b] = x[..., b] * cos[:, None] + x[..., a] * sin[:, None]
    return y


def attn(q, kc, vc, table, cu, kv_len, scale, softcap=0.0, window=0):
    """(out, bound) in 64 bits, one query row at a time over the keys it sees, so that what it does not see cannot matter.  The weights and the
    result are rounded to 8 bits (2^-8 of each at most); scores and sums in 32 bits add well under 2^-12 of sum_j p_j |v_j|."""
    T, Hq, D = q.shape
    Hkv, ps = kc.shape[1], kc.shape[2]
    G = Hq // Hkv
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    tol = torch.zeros_like(out)
    q, kc, vc = q.cpu().double(), kc.cpu().double(), vc.cpu().double()
    for b in range(len(cu) - 1):
        n, L = cu[b + 1] - cu[b], kv_len[b]
        if n <= 0 or L <= 0:
            continue
        j = torch.arange(L)
        pages = table[b].cpu().long()[j // ps]
        k, v = kc[pages, :, j % ps], vc[pages, :, j % ps]    # [L, Hkv, D]
        for i in range(n):
            p = L - n + i
            if p < 0:
                continue
            lo = max(0, p - window + 1) if window else 0
            s = torch.einsum("hgd,jhd->hgj", q[cu[b] + i].view(Hkv, G, D), k[lo:p + 1]) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            w = torch.softmax(s, -1)
            o = torch.einsum("hgj,jhd->hgd", w, v[lo:p + 1])
            out[cu[b] + i] = o.reshape(Hq, D)
            spread = torch.einsum("hgj,jhd->hgd", w, v[lo:p + 1].abs()).reshape(Hq, D)
            tol[cu[b] + i] = 2.0 ** -8 * o.reshape(Hq, D).abs() + (2.0 ** -8 + 2.0 ** -12) * spread + 1e-30
    return out, tol


def make_cache(lens, Hkv, D, ps, seed, spare=3, fill=None):
    """Random pages for sequences of the given lengths: (k, v, table, page count).  Slots past a sequence's end and spare pages hold ``fill`` (default: noise)."""
    g = torch.Generator().manual_seed(seed)
    need = [math.ceil(L / ps) for L in lens]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g)
    table = torch.full((len(lens), max(need + [1]) + 1), -7, dtype=torch.int32)
    kc = torch.randn(n_pages, Hkv, ps, D, generator=g)
    vc = torch.randn(n_pages, Hkv, ps, D, generator=g)
    used = torch.zeros(n_pages, ps, dtype=torch.bool)
    at = 0
    for b, L in enumerate(lens):
        for i in range(need[b]):
            page = int(order[at]); at += 1
            table[b, i] = page
            used[page, :min(ps, L - i * ps)] = True
    if fill is not None:
        kc.permute(0, 2, 1, 3)[~used] = fill
        vc.permute(0, 2, 1, 3)[~used] = fill
    return kc.to(torch.bfloat16), vc.to(torch.bfloat16), table
