"""The operators that serve a chunk of new tokens next to the nested weight planes, and what is measured of them.

Three operators stand between the quantised linear layers of a decoder:

``linear``   a linear layer on 8-bit codes with 8-bit activations: the tokens are quantised with one scale each, multiplied
             with the codes (or a slice of them) in integers, and alpha, z and the token's scale are applied afterwards;
``append``   the new keys and values go into a paged cache, keys and queries rotated by their positions on the way;
``attend``   the new tokens' queries attend to the cache: single tokens, a few drafted tokens, whole chunks.

``own`` selects between the plain form (elementary torch operations in 32 bits) and the library's own calls.
"""
import math
import random

import torch

own = False

# ------------------------------------------------------------------ cases

def listed():
    return [
        # one token through the gate projection of a Gemma-2-2B MLP: what a call costs when there is next to nothing to do
        dict(name="linear_1_token", op="linear", M=1, N=9216, K=2304, r=8, out="f32"),
        # a ragged handful of tokens through the down projection
        dict(name="linear_37_tokens", op="linear", M=37, N=2304, K=9216, r=8, out="bf16"),
        # a chunk that fills no whole tile, on the int4 slice of the codes (Gemma-2-9B up projection)
        dict(name="linear_chunk_509_int4", op="linear", M=509, N=14336, K=3584, r=4, out="bf16"),
        # a long prompt through the Mistral-7B matrix
        dict(name="linear_prompt_4096", op="linear", M=4096, N=14336, K=4096, r=8, out="bf16"),
        # a decode step of 64 sequences: one new key and value each
        dict(name="append_64_sequences", op="append", B=64, new_min=1, new_max=1, ctx_min=1, ctx_max=4096, Hq=32, Hkv=8, D=128,
             page=16, rot=128, interleaved=False, lens_seed=1),
        # short drafts on a small model whose heads are rotated in part, neighbouring elements being the pairs
        dict(name="append_drafts_part_rotated", op="append", B=7, new_min=1, new_max=33, ctx_min=0, ctx_max=700, Hq=12, Hkv=4, D=64,
             page=32, rot=32, interleaved=True, lens_seed=2),
        # the prompts of three requests with Gemma-2-9B's heads
        dict(name="append_prompts_d256", op="append", B=3, new_min=1500, new_max=4000, ctx_min=0, ctx_max=3000, Hq=16, Hkv=8, D=256,
             page=64, rot=256, interleaved=False, lens_seed=3),
        # one long conversation, one new token
        dict(name="attend_1_token_32k", op="attend", B=1, new_min=1, new_max=1, ctx_min=32767, ctx_max=32767, Hq=32, Hkv=8, D=128,
             page=16, softcap=0.0, window=0, lens_seed=4),
        # a decode step of 64 sequences of very different lengths, Gemma-2-9B's heads and its cap on the scores
        dict(name="attend_64_tokens_ragged_d256", op="attend", B=64, new_min=1, new_max=1, ctx_min=5, ctx_max=8000, Hq=16, Hkv=8, D=256,
             page=32, softcap=50.0, window=0, lens_seed=5),
        # drafted tokens of 16 sequences are verified, each key reaching 4096 tokens back
        dict(name="attend_drafts_window", op="attend", B=16, new_min=2, new_max=6, ctx_min=100, ctx_max=9000, Hq=32, Hkv=8, D=128,
             page=16, softcap=0.0, window=4096, lens_seed=6),
        # a short chunk over a cache with Gemma-2-9B's heads, cap and window
        dict(name="attend_chunk_500_d256", op="attend", B=1, new_min=500, new_max=500, ctx_min=6011, ctx_max=6011, Hq=16, Hkv=8, D=256,
             page=64, softcap=50.0, window=4096, lens_seed=7),
        # the second half of a long prompt
        dict(name="attend_chunk_8192_over_8192", op="attend", B=1, new_min=8192, new_max=8192, ctx_min=8192, ctx_max=8192, Hq=32, Hkv=8,
             D=128, page=64, softcap=0.0, window=0, lens_seed=8),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        b, f = largest.get(c["op"], (0, 0))
        largest[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    op = rng.choice(["linear", "linear", "append", "attend", "attend", "attend"])
    while True:
        if op == "linear":
            case = dict(op=op, M=_log_int(rng, 1, 4096), N=_log_int(rng, 200, 16384), K=16 * _log_int(rng, 16, 896),
                        r=rng.choice([8, 8, 4, 2]), out=rng.choice(["f32", "bf16"]))
        else:
            D = rng.choice([64, 128, 128, 256])
            Hkv = rng.choice([1, 2, 4, 8])
            G = rng.choice([1, 2, 3, 4, 5, 8])
            B = _log_int(rng, 1, 64)
            new_max = rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 16, 8192)])
            ctx_max = _log_int(rng, 16, 32768)
            case = dict(op=op, B=B, new_min=rng.randint(1, new_max), new_max=new_max, ctx_min=rng.randint(0, ctx_max), ctx_max=ctx_max,
                        Hq=Hkv * G, Hkv=Hkv, D=D, page=rng.choice([16, 32, 64, 128]), lens_seed=rng.randint(0, 1 << 30))
            if op == "append":
                case.update(rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.5)
            else:
                case.update(softcap=rng.choice([0.0, 0.0, 50.0]), window=rng.choice([0, 0, _log_int(rng, 64, 8192)]))
        w = work(case)
        b, f = largest[op]
        cached = 0 if op == "linear" else sum(n + c for n, c in _lengths(case)) * case["Hkv"] * case["D"] * 4
        if w["bytes"] <= b and w["flops"] <= f and cached <= 1.5e9:
            return case


def _lengths(case):
    """(new tokens, tokens cached before) of every sequence; the longest values are always among them."""
    rng = random.Random(case["lens_seed"])
    out = [(rng.randint(case["new_min"], case["new_max"]), rng.randint(case["ctx_min"], case["ctx_max"])) for _ in range(case["B"])]
    out[rng.randrange(case["B"])] = (case["new_max"], case["ctx_max"])
    return out


def _keys(new, ctx, window):
    """Pairs of query and key that are multiplied, and keys that at least one query reads."""
    L = new + ctx
    if not window or window >= L:
        return new * ctx + new * (new + 1) // 2, L
    pairs = sum(min(window, ctx + i + 1) for i in range(new))
    return pairs, L - max(0, ctx + 1 - window)


def work(case):
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 8 * N + M * K + 8 * M + M * N * (4 if case["out"] == "f32" else 2), "flops": 2 * M * N * K}
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "append":
        return {"bytes": T * (2 * 2 * D * (Hq + 2 * Hkv) + 4 * case["rot"]), "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    pairs = sum(_keys(n, c, case["window"])[0] for n, c in lens)
    read = sum(_keys(n, c, case["window"])[1] for n, c in lens)
    return {"bytes": read * Hkv * D * 4 + 2 * T * Hq * D * 2, "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ inputs

def _slice(q, r):
    """S(q, r): the r leading bits of an 8-bit code, rounded, on the 8-bit grid."""
    if r == 8:
        return q
    sh = 8 - r
    return (((q.int() + (1 << (sh - 1))) >> sh).clamp(max=(1 << r) - 1) << sh).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    st = dict(case=case)
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        # a few input features are an order of magnitude larger than the rest, as in a decoder's residual stream
        gain = torch.ones(K, device="cuda")
        gain[torch.randint(0, K, (max(1, K // 512),), generator=g, device="cuda")] = 8.0
        st["x"] = (normal(M, K) * gain).to(torch.bfloat16)
        W = (normal(N, K) * 0.02).to(torch.bfloat16).float()
        lo, hi = W.amin(1), W.amax(1)
        alpha = (hi - lo) / torch.full_like(hi, 255.0)
        zero = -lo / alpha
        codes = torch.floor(W / alpha[:, None] + zero[:, None] + 0.5).clamp(0, 255).to(torch.uint8)
        st.update(alpha=alpha, zero=zero, codes=_slice(codes, case["r"]),
                  out_dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16)
        if own:
            st["y"] = torch.empty(M, N, dtype=st["out_dtype"], device="cuda")
            st["xq"] = torch.empty(M, K, dtype=torch.int8, device="cuda")
            st["scale"] = torch.empty(M, dtype=torch.float32, device="cuda")
            st["rowsum"] = torch.empty(M, dtype=torch.int32, device="cuda")
        return st

    lens = _lengths(case)
    B, Hq, Hkv, D, ps = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    T = sum(n for n, _ in lens)
    total = [n + c for n, c in lens]
    pages = [-(-t // ps) for t in total]
    n_pages = sum(pages) + 5
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((B, max(pages) + 2), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    st.update(lens=lens, cu=cu, page_table=table.cuda(), cu_q=torch.tensor(cu, dtype=torch.int32, device="cuda"),
              kv_len=torch.tensor(total, dtype=torch.int32, device="cuda"), max_q=max(n for n, _ in lens), max_kv=max(total))
    st["k_cache"] = normal(n_pages, Hkv, ps, D).to(torch.bfloat16)
    st["v_cache"] = normal(n_pages, Hkv, ps, D).to(torch.bfloat16)
    if case["op"] == "append":
        qkv = normal(T, (Hq + 2 * Hkv) * D).to(torch.bfloat16)       # the three projections of a token stand side by side
        st["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        st["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        st["v"] = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        half = case["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(max(total), device="cuda", dtype=torch.float64)[:, None] * freq
        st["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        st["q_out"] = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda")
        # where every new token goes, as a serving loop that plans on the host knows it
        pos = torch.cat([torch.arange(c, c + n) for n, c in lens])
        seq = torch.cat([torch.full((n,), b, dtype=torch.int64) for b, (n, _) in enumerate(lens)])
        st["pos"] = pos.cuda()
        st["page_of"] = table[seq, pos // ps].long().cuda()
        st["slot_of"] = (pos % ps).cuda()
    else:
        st["q"] = (normal(T, Hq, D) * 1.5).to(torch.bfloat16)
        st["scale"] = D ** -0.5
        if own:
            from paper_2502_06786_b200 import binding as mq
            st["out"] = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda")
            st["workspace"] = torch.empty(mq.attn_paged_workspace_bytes(T, B, Hq, Hkv, D, st["max_q"], st["max_kv"], case["window"]),
                                          dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    op = st["case"]["op"]
    if own:
        return {"linear": _linear_own, "append": _append_own, "attend": _attend_own}[op](st)
    return {"linear": _linear_plain, "append": _append_plain, "attend": _attend_plain}[op](st)


def _linear_own(st):
    from paper_2502_06786_b200 import binding as mq
    mq.quantize_tokens(st["x"], xq=st["xq"], scale=st["scale"], rowsum=st["rowsum"])
    mq.gemm_a8(st["xq"], st["scale"], st["rowsum"], st["codes"], st["alpha"], st["zero"], y=st["y"],
               flags=mq.GEMV_PDL)                                       # the call before writes no weights
    return st["xq"], st["scale"], st["y"]


def _linear_plain(st):
    x = st["x"].float()
    top = x.abs().amax(1)
    scale = (top / torch.full_like(top, 127.0)).clamp(min=2.0 ** -126)
    xq = torch.round(x / scale[:, None]).clamp(-127, 127)
    # z lies near 128: taking 128 off the codes first keeps the two sums that are subtracted small
    acc = xq @ (st["codes"].float() - 128.0).t() - (st["zero"] - 128.0)[None, :] * xq.sum(1, keepdim=True)
    y = (scale[:, None] * st["alpha"][None, :]) * acc
    return xq.to(torch.int8), scale, y.to(st["out_dtype"])


def _append_own(st):
    from paper_2502_06786_b200 import binding as mq
    mq.kv_append(st["k_cache"], st["v_cache"], st["page_table"], st["cu_q"], st["kv_len"], st["k"], st["v"], cos_sin=st["cos_sin"],
                 q=st["q"], q_out=st["q_out"], interleaved=st["case"]["interleaved"])
    return st["q_out"], st["k_cache"], st["v_cache"]


def _rotate_plain(x, cos, sin, rot, interleaved):
    x = x.float()
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    c, s = cos[:, None, :], sin[:, None, :]
    ra, rb = a * c - b * s, b * c + a * s
    done = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([done, x[..., rot:]], -1).to(torch.bfloat16)


def _append_plain(st):
    rot, inter = st["case"]["rot"], st["case"]["interleaved"]
    cs = st["cos_sin"][st["pos"]]
    cos, sin = cs[:, :rot // 2], cs[:, rot // 2:]
    st["q_out"].copy_(_rotate_plain(st["q"], cos, sin, rot, inter))
    st["k_cache"][st["page_of"], :, st["slot_of"]] = _rotate_plain(st["k"], cos, sin, rot, inter)
    st["v_cache"][st["page_of"], :, st["slot_of"]] = st["v"]
    return st["q_out"], st["k_cache"], st["v_cache"]


def _attend_own(st):
    from paper_2502_06786_b200 import binding as mq
    mq.attn_paged(st["q"], st["k_cache"], st["v_cache"], st["page_table"], st["cu_q"], st["kv_len"], st["max_q"], st["max_kv"],
                  scale=st["scale"], softcap=st["case"]["softcap"], window=st["case"]["window"], out=st["out"], workspace=st["workspace"])
    return st["out"]


def _attend_plain(st):
    case = st["case"]
    Hq, Hkv, D, cap, window = case["Hq"], case["Hkv"], case["D"], case["softcap"], case["window"]
    G = Hq // Hkv
    out = torch.empty_like(st["q"])
    for b, (n, ctx) in enumerate(st["lens"]):
        L = n + ctx
        pages = st["page_table"][b, :-(-L // case["page"])].long()
        q = st["q"][st["cu"][b]:st["cu"][b + 1]].float().view(n, Hkv, G, D).permute(1, 2, 0, 3)     # [Hkv, G, n, D]
        pos = torch.arange(ctx, L, device="cuda")[:, None]
        key = torch.arange(L, device="cuda")[None, :]
        seen = key <= pos
        if window:
            seen &= key > pos - window
        step = Hkv if n * L * Hq <= 1 << 29 else 1                    # long chunks: one key head at a time
        for h in range(0, Hkv, step):
            k = st["k_cache"][pages, h:h + step].permute(1, 0, 2, 3).reshape(step, 1, -1, D)[:, :, :L].float()
            v = st["v_cache"][pages, h:h + step].permute(1, 0, 2, 3).reshape(step, 1, -1, D)[:, :, :L].float()
            s = (q[h:h + step] @ k.transpose(-1, -2)) * st["scale"]
            if cap:
                s = torch.tanh(s / cap) * cap
            s.masked_fill_(~seen, -math.inf)
            s -= s.amax(-1, keepdim=True)
            s.exp_()
            o = (s @ v) / s.sum(-1, keepdim=True)
            out[st["cu"][b]:st["cu"][b + 1], h * G:(h + step) * G] = o.permute(2, 0, 1, 3).reshape(n, step * G, D).to(torch.bfloat16)
    return out


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "linear":
        # the scale and the quotient are binary32 values by definition; a binary64 quotient rounded to binary32 is that quotient
        x = st["x"].to(f64)
        scale = (x.abs().max(1).values / 127.0).float().clamp(min=2.0 ** -126)
        xq = (x / scale.to(f64).unsqueeze(1)).float().round().clamp(-127, 127)
        weight = st["alpha"].to(f64).unsqueeze(1) * (st["codes"].to(f64) - st["zero"].to(f64).unsqueeze(1))
        y = torch.matmul(xq.to(f64) * scale.to(f64).unsqueeze(1), weight.t())
        return xq.to(torch.int8), scale, y
    ps, D, Hq, Hkv = case["page"], case["D"], case["Hq"], case["Hkv"]
    table = st["page_table"].long()
    if case["op"] == "append":
        half = case["rot"] // 2
        q_out = st["q"].to(f64).clone()
        kc, vc = st["k_cache"].to(f64), st["v_cache"].to(f64)
        k_new = st["k"].to(f64).clone()
        first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)
        for b, (n, ctx) in enumerate(st["lens"]):
            rows = slice(st["cu"][b], st["cu"][b + 1])
            p = torch.arange(ctx, ctx + n, device="cuda")
            c = st["cos_sin"][p, :half].to(f64).unsqueeze(1)
            s = st["cos_sin"][p, half:].to(f64).unsqueeze(1)
            for t in (q_out, k_new):
                u, w = t[rows][..., first].clone(), t[rows][..., second].clone()
                block = t[rows]
                block[..., first] = u * c - w * s
                block[..., second] = u * s + w * c
            for i in range(-(-(ctx + n) // ps)):                         # page by page
                lo, hi = max(i * ps, ctx), min((i + 1) * ps, ctx + n)
                if lo < hi:
                    src = slice(st["cu"][b] + lo - ctx, st["cu"][b] + hi - ctx)
                    page = int(table[b, i])
                    kc[page, :, lo - i * ps:hi - i * ps] = k_new[src].transpose(0, 1)
                    vc[page, :, lo - i * ps:hi - i * ps] = st["v"][src].to(f64).transpose(0, 1)
        return q_out, kc, vc
    out = torch.zeros(st["q"].shape, dtype=f64, device="cuda")
    G = Hq // Hkv
    for b, (n, ctx) in enumerate(st["lens"]):
        L = n + ctx
        where = torch.arange(L, device="cuda")
        page, slot = table[b][where // ps], where % ps
        for h in range(Hkv):
            k, v = st["k_cache"][page, h, slot].to(f64), st["v_cache"][page, h, slot].to(f64)
            for lo in range(0, n, 2048):                                 # a block of queries, so that the scores fit
                hi = min(n, lo + 2048)
                at = ctx + torch.arange(lo, hi, device="cuda").unsqueeze(1)
                hidden = where.unsqueeze(0) > at
                if case["window"]:
                    hidden = hidden | (at - where.unsqueeze(0) >= case["window"])
                for head in range(h * G, (h + 1) * G):
                    rows = slice(st["cu"][b] + lo, st["cu"][b] + hi)
                    logits = st["q"][rows, head].to(f64) @ k.t() * st["scale"]
                    if case["softcap"]:
                        logits = case["softcap"] * torch.tanh(logits / case["softcap"])
                    weights = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
                    out[rows, head] = weights @ v
    return out
