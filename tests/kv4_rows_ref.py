"""Attention over a cache in 4-bit groups for many rows at once: groups_ref.attn's formula in 64 bits with whole matrices (tests only)."""
import torch

from tests import groups_ref as gr


def attn(q, tiles, table, cu, kv_len, scale, softcap=0.0, window=0, device="cuda"):
    """(out, bound) of a call that unpacks its sequences of more than 16 rows.

    Those: queries, keys, values and weights are held in fp16, each off by 2^-11 of itself at most; beside that queries by 2^-39 of their row's largest element, keys and
    values by 2^-39 of the largest of their sequence and head, weights by 2^-29 of their row's largest.  The others: p * scale is rounded to bf16 beside code - 8, 2^-8 of
    sum_j p_j |v_j - middle_j|.  Both: a score is off by 2^-20 of sum_d |q_d| (15 scale + |low|) (fp32 steps), with a cap by 2.6e-6 of itself more; sums in 32 bits by well
    under 2^-12 of their terms; the output is rounded to bf16."""
    T, Hq, D = q.shape
    k_all, v_all, mid_all, size_all, _ = gr.cache_values(tiles)
    Hkv, ps = k_all.shape[1], k_all.shape[2]
    G = Hq // Hkv
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    tol = torch.zeros_like(out)
    q = q.cpu().double()
    for b in range(len(cu) - 1):
        n, L = int(cu[b + 1] - cu[b]), int(kv_len[b])
        if n <= 0 or L <= 0:
            continue
        j = torch.arange(L)
        pages = table[b].cpu().long()[j // ps]
        k, v, mid, size = (t[pages, :, j % ps].to(device) for t in (k_all, v_all, mid_all, size_all))
        pos = torch.arange(L - n, L, device=device)
        at = torch.arange(L, device=device)
        seen = at[None] <= pos[:, None]
        if window:
            seen &= at[None] > pos[:, None] - window
        some = (pos >= 0).double()[None, :, None]
        for h in range(Hkv):
            qh = q[cu[b]:cu[b + 1], h * G:(h + 1) * G].to(device).transpose(0, 1)          # [G, n, D]
            kh, vh = k[:, h], v[:, h].nan_to_num(0)
            lost = seen.double() @ v[:, h].isnan().double() > 0                            # a value that is not a number reaches the rows that see it
            largest = kh.nan_to_num(0).abs().max()
            s = qh @ kh.t() * scale
            off = 2.0 ** -20 * scale * (qh.abs() @ size[:, h].t())
            if n * G > 16:
                off = off + scale * (2.0 ** -10 * (qh.abs() @ kh.abs().t()) + 2.0 ** -39 * (qh.abs().sum(-1, keepdim=True) * largest
                                                                                            + qh.abs().amax(-1, keepdim=True) * kh.abs().sum(-1)))
            if softcap:
                s = softcap * torch.tanh(s / softcap)
                off = off + 2.6e-6 * s.abs()
            s = s.masked_fill(~seen, float("-inf"))
            off = off.masked_fill(~seen, 0).amax(-1, keepdim=True)
            w = torch.softmax(s, -1)
            w = torch.where(seen.any(-1, keepdim=True), w, 0)
            o, spread = (w @ vh).masked_fill(lost, float("nan")), w @ vh.abs()
            if n * G > 16:
                from_rounding = 2.0 ** -10 * spread + 2.0 ** -29 * w.amax(-1, keepdim=True) * (seen.double() @ vh.abs()) + 2.0 ** -39 * vh.abs().max()
            else:
                from_rounding = 2.0 ** -8 * torch.einsum("gnj,jd->gnd", w, (vh - mid[:, h].nan_to_num(0)).abs())
            bound = 2.0 ** -8 * o.abs() + from_rounding + 2.0 ** -12 * (spread + from_rounding) + torch.expm1(2 * off) * (spread + o.abs()) + 1e-30
            rows = slice(cu[b], cu[b + 1])
            out[rows, h * G:(h + 1) * G] = (o * some).transpose(0, 1).cpu()
            tol[rows, h * G:(h + 1) * G] = (bound * some).transpose(0, 1).cpu()
    return out, tol


def check(got, want, tol):
    bad = ~((got.double().cpu() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double().cpu() - want).abs() / tol)[bad].max()), bad.nonzero()[0].tolist())
