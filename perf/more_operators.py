"""Decoding at four bits with a scale per group: the operators for it, and what is measured of them.

A group is a run of consecutive values that shares a scale and a low end: 4-bit codes q stand for ``scale * q + low``.  Four operators use it:

``quantize``  a weight matrix to codes and groups (32, 64 or 128 weights of a row each);
``linear``    a decode step's product of a few tokens with such a matrix;
``append``    new keys and values, rotated by their positions, into a paged cache held in 4-bit groups of 64;
``attend``    the new tokens' queries attend to that cache: single tokens, drafts, chunks.

``own`` selects between the plain form (elementary torch operations in 32 bits) and the library's own calls.
"""
import math
import random

import torch

own = False

# ------------------------------------------------------------------ cases

def listed():
    return [
        # a gate projection of Gemma-2-2B, as it is quantised when a model is loaded
        dict(name="quantize_9216x2304_g64", op="quantize", N=9216, K=2304, group=64),
        # the largest matrix of a Mistral-7B layer
        dict(name="quantize_14336x4096_g128", op="quantize", N=14336, K=4096, group=128),
        # one token through the gate projection: what a call costs when there is little to do
        dict(name="linear_1_token", op="linear", M=1, N=9216, K=2304, group=128, out="bf16"),
        # five drafted tokens, a matrix that fills no whole tile, the smallest groups
        dict(name="linear_5_tokens_odd_g32", op="linear", M=5, N=1001, K=4064, group=32, out="f32"),
        # a batch of 16 through the down projection of Gemma-2-9B
        dict(name="linear_16_tokens", op="linear", M=16, N=3584, K=14336, group=128, out="bf16"),
        # one token through a matrix of many rows, as an output head has them
        dict(name="linear_1_token_65536_rows", op="linear", M=1, N=65536, K=2304, group=64, out="f32"),
        # a decode step of 64 sequences: one new key and value each
        dict(name="append_64_sequences", op="append", B=64, new_min=1, new_max=1, ctx_min=1, ctx_max=4096, Hq=32, Hkv=8, D=128,
             page=16, rot=128, interleaved=False, lens_seed=11),
        # the prompts of three requests with Gemma-2-9B's heads
        dict(name="append_prompts_d256", op="append", B=3, new_min=1500, new_max=4000, ctx_min=0, ctx_max=3000, Hq=16, Hkv=8, D=256,
             page=64, rot=256, interleaved=False, lens_seed=13),
        # one long conversation, one new token
        dict(name="attend_1_token_32k", op="attend", B=1, new_min=1, new_max=1, ctx_min=32767, ctx_max=32767, Hq=32, Hkv=8, D=128,
             page=16, softcap=0.0, window=0, lens_seed=14),
        # a decode step of 64 sequences of very different lengths, Gemma-2-9B's heads and its cap on the scores
        dict(name="attend_64_tokens_ragged_d256", op="attend", B=64, new_min=1, new_max=1, ctx_min=5, ctx_max=8000, Hq=16, Hkv=8, D=256,
             page=32, softcap=50.0, window=0, lens_seed=15),
        # drafted tokens of 16 sequences are verified, each key reaching 4096 tokens back
        dict(name="attend_drafts_window", op="attend", B=16, new_min=2, new_max=6, ctx_min=100, ctx_max=9000, Hq=32, Hkv=8, D=128,
             page=16, softcap=0.0, window=4096, lens_seed=16),
        # the second half of a long prompt
        dict(name="attend_chunk_4096_over_4096", op="attend", B=1, new_min=4096, new_max=4096, ctx_min=4096, ctx_max=4096, Hq=32, Hkv=8,
             D=128, page=64, softcap=0.0, window=0, lens_seed=18),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        b, f = largest.get(c["op"], (0, 0))
        largest[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    op = rng.choice(["quantize", "linear", "linear", "append", "attend", "attend", "attend"])
    while True:
        if op in ("quantize", "linear"):
            group = rng.choice([32, 64, 128])
            case = dict(op=op, N=_log_int(rng, 200, 65536), K=group * _log_int(rng, 4, 14336 // group), group=group)
            if op == "linear":
                case.update(M=rng.choice([1, 1, _log_int(rng, 2, 64)]), out=rng.choice(["f32", "bf16"]))
        else:
            Hkv = rng.choice([1, 2, 4, 8])
            new_max = rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 16, 4096)])
            ctx_max = _log_int(rng, 16, 32768)
            case = dict(op=op, B=_log_int(rng, 1, 64), new_min=rng.randint(1, new_max), new_max=new_max, ctx_min=rng.randint(0, ctx_max),
                        ctx_max=ctx_max, Hq=Hkv * rng.choice([1, 2, 3, 4, 5, 8]), Hkv=Hkv, D=rng.choice([64, 128, 128, 256]),
                        page=rng.choice([16, 32, 64, 128]), lens_seed=rng.randint(0, 1 << 30))
            if op == "append":
                case.update(rot=rng.choice([case["D"], case["D"], case["D"] // 2]), interleaved=rng.random() < 0.5)
            else:
                case.update(softcap=rng.choice([0.0, 0.0, 50.0]), window=rng.choice([0, 0, _log_int(rng, 64, 8192)]))
        w = work(case)
        b, f = largest[op]
        fits = w["bytes"] <= b and w["flops"] <= f
        if op in ("append", "attend"):
            # what the plain form lays out in 32 bits: padded keys and values, and the scores
            longest = case["new_max"] + case["ctx_max"]
            fits = fits and case["B"] * longest * case["Hkv"] * case["D"] <= 1.1e9
            fits = fits and case["B"] * longest * case["Hq"] * (case["new_max"] if op == "attend" else 1) <= 1.1e9
        if fits:
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
    if case["op"] in ("quantize", "linear"):
        N, K = case["N"], case["K"]
        held = N * K // 2 + 4 * N * K // case["group"]
        if case["op"] == "quantize":
            return {"bytes": 2 * N * K + held, "flops": 5 * N * K}
        M = case["M"]
        return {"bytes": held + 2 * M * K + M * N * (4 if case["out"] == "f32" else 2), "flops": 2 * M * N * K}
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    key = 2 * Hkv * (D // 2 + D // 16)                                # a key and a value: codes, and 4 bytes per 64 of them
    if case["op"] == "append":
        return {"bytes": T * (2 * D * (2 * Hq + 2 * Hkv) + key + 4 * case["rot"]), "flops": T * (3 * (Hq + Hkv) * case["rot"] + 10 * Hkv * D)}
    pairs = sum(_keys(n, c, case["window"])[0] for n, c in lens)
    read = sum(_keys(n, c, case["window"])[1] for n, c in lens)
    return {"bytes": read * key + 2 * T * Hq * D * 2, "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ the 4-bit group

GROUP = 64                                                             # of the cache, along the head
TILE = 16                                                              # keys whose codes and groups stand together


def _to_groups(x, group):
    """Codes (one byte each) and (scale, low) of the groups along the last axis; every step is one binary32 operation."""
    v = x.float().unflatten(-1, (-1, group))
    low, top = v.aminmax(dim=-1)
    scale = ((top - low) / torch.full_like(low, 15.0)).to(torch.bfloat16).float()
    scale = torch.where(scale < 2.0 ** -120, 0.0, scale)
    inverse = torch.where(scale > 0, torch.ones_like(scale) / scale, 0.0)
    code = torch.round((v - low.unsqueeze(-1)) * inverse.unsqueeze(-1)).clamp(max=15).flatten(-2).to(torch.uint8)
    return code, torch.stack([scale, low + 0.0], -1).to(torch.bfloat16)


def _pack(code):
    """Element 2j in the low half of byte j."""
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


def _tiles(code, params):
    """A page's keys (or values) as the cache holds them: [..., page, D] codes and [..., page, D / 64, 2] groups to [..., page / 16, 9 D] bytes.
    The codes of 32 elements stand together for 16 keys, then the next 32; behind them the groups, likewise."""
    c = _pack(code).unflatten(-2, (-1, TILE)).unflatten(-1, (-1, 16)).transpose(-3, -2).flatten(-3)
    p = params.contiguous().view(torch.uint8).unflatten(-3, (-1, TILE)).flatten(-2).unflatten(-1, (-1, 4)).transpose(-3, -2).flatten(-3)
    return torch.cat([c, p], -1)


def _values(tiles, D):
    """The reverse of _tiles, in values: [..., page / 16, 9 D] bytes to [..., page, D]."""
    code = _unpack(tiles[..., :8 * D].unflatten(-1, (D // 32, TILE, 16)).transpose(-3, -2).flatten(-2))            # [..., page / 16, 16, D]
    params = tiles[..., 8 * D:].unflatten(-1, (D // GROUP, TILE, 4)).transpose(-3, -2).contiguous().view(torch.bfloat16).float()
    v = code.unflatten(-1, (-1, GROUP)).float() * params[..., :1] + params[..., 1:]
    return v.flatten(-2).flatten(-3, -2)


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    st = dict(case=case)
    if case["op"] in ("quantize", "linear"):
        N, K, group = case["N"], case["K"], case["group"]
        W = (normal(N, K) * 0.02).to(torch.bfloat16)
        if case["op"] == "quantize":
            st["W"] = W
            st["packed"] = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
            st["params"] = torch.empty(N, K // group, 2, dtype=torch.bfloat16, device="cuda")
            return st
        # a few input features are an order of magnitude larger than the rest, as in a decoder's residual stream
        gain = torch.ones(K, device="cuda")
        gain[torch.randint(0, K, (max(1, K // 512),), generator=g, device="cuda")] = 8.0
        st["x"] = (normal(case["M"], K) * gain).to(torch.bfloat16)
        code, st["params"] = _to_groups(W, group)
        st["packed"] = _pack(code)
        st["y"] = torch.empty(case["M"], N, dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")
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
    # where every new token stands, as a serving loop that plans on the host knows it
    seq = torch.cat([torch.full((n,), b, dtype=torch.int64) for b, (n, _) in enumerate(lens)])
    pos = torch.cat([torch.arange(c, c + n) for n, c in lens])
    st.update(seq=seq.cuda(), pos=pos.cuda(), row=torch.cat([torch.arange(n) for n, _ in lens]).cuda())
    # keys have a few channels that are larger than the rest in all tokens, values have none
    gain = 1.0 + 3.0 * (torch.rand(Hkv, 1, D, generator=g, device="cuda") < 0.03)
    st["cache"] = torch.empty(n_pages, Hkv, ps // TILE, 18 * D, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (Hkv * ps * D))
    for lo in range(0, n_pages, step):
        part = st["cache"][lo:lo + step]
        part[..., :9 * D] = _tiles(*_to_groups((normal(len(part), Hkv, ps, D) * gain).to(torch.bfloat16), GROUP))
        part[..., 9 * D:] = _tiles(*_to_groups(normal(len(part), Hkv, ps, D).to(torch.bfloat16), GROUP))
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
        st["page_of"] = table[seq, pos // ps].long().cuda()
        st["slot_of"] = (pos % ps).cuda()
    else:
        st["q"] = (normal(T, Hq, D) * 1.5).to(torch.bfloat16)
        st["scale"] = D ** -0.5
        st["out"] = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda")
        if own:
            from paper_2502_06786_b200 import binding as mq
            st["workspace"] = torch.empty(mq.attn_paged4_workspace_bytes(T, B, Hq, Hkv, D, st["max_q"], st["max_kv"], case["window"]),
                                          dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    op = st["case"]["op"]
    if own:
        return {"quantize": _quantize_own, "linear": _linear_own, "append": _append_own, "attend": _attend_own}[op](st)
    return {"quantize": _quantize_plain, "linear": _linear_plain, "append": _append_plain, "attend": _attend_plain}[op](st)


def _quantize_own(st):
    from paper_2502_06786_b200 import binding as mq
    # the codes are defined bit for bit: the bytes that hold them are whole numbers
    return mq.quantize_groups(st["W"], st["case"]["group"], packed=st["packed"], params=st["params"])


def _quantize_plain(st):
    code, params = _to_groups(st["W"], st["case"]["group"])
    return _pack(code), params


def _linear_own(st):
    from paper_2502_06786_b200 import binding as mq
    return mq.gemv_groups(st["packed"], st["params"], st["x"], y=st["y"], flags=mq.GEMV_PDL)           # the call before writes no weights


def _linear_plain(st):
    group, params = st["case"]["group"], st["params"].float()
    W = _unpack(st["packed"]).float().unflatten(-1, (-1, group)) * params[..., :1] + params[..., 1:]
    return (st["x"].float() @ W.flatten(1).t()).to(st["y"].dtype)


def _append_own(st):
    from paper_2502_06786_b200 import binding as mq
    mq.kv4_append(st["cache"], st["page_table"], st["cu_q"], st["kv_len"], st["k"], st["v"], cos_sin=st["cos_sin"], q=st["q"],
                  q_out=st["q_out"], interleaved=st["case"]["interleaved"])
    return st["q_out"], st["cache"]


def _rotate_plain(x, cos, sin, rot, interleaved):
    x = x.float()
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    c, s = cos[:, None, :], sin[:, None, :]
    ra, rb = a * c - b * s, b * c + a * s
    done = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([done, x[..., rot:]], -1).to(torch.bfloat16)


def _store_plain(tiles, D, page, slot, x):
    """Rows x [T, heads, D] into a cache's keys (or values) [pages, heads, page / 16, 9 D]."""
    code, params = _to_groups(x, GROUP)
    tile, key = slot // TILE, slot % TILE
    tiles[..., :8 * D].unflatten(-1, (D // 32, TILE, 16))[page, :, tile, :, key] = _pack(code).unflatten(-1, (-1, 16))
    tiles[..., 8 * D:].unflatten(-1, (D // GROUP, TILE, 4))[page, :, tile, :, key] = params.contiguous().view(torch.uint8).flatten(-2).unflatten(-1, (-1, 4))


def _append_plain(st):
    rot, inter, D = st["case"]["rot"], st["case"]["interleaved"], st["case"]["D"]
    cs = st["cos_sin"][st["pos"]]
    cos, sin = cs[:, :rot // 2], cs[:, rot // 2:]
    st["q_out"].copy_(_rotate_plain(st["q"], cos, sin, rot, inter))
    _store_plain(st["cache"][..., :9 * D], D, st["page_of"], st["slot_of"], _rotate_plain(st["k"], cos, sin, rot, inter))
    _store_plain(st["cache"][..., 9 * D:], D, st["page_of"], st["slot_of"], st["v"])
    return st["q_out"], st["cache"]


def _attend_own(st):
    from paper_2502_06786_b200 import binding as mq
    return mq.attn_paged4(st["q"], st["cache"], st["page_table"], st["cu_q"], st["kv_len"], st["max_q"], st["max_kv"], scale=st["scale"],
                          softcap=st["case"]["softcap"], window=st["case"]["window"], out=st["out"], workspace=st["workspace"])


def _attend_plain(st):
    case = st["case"]
    B, Hq, Hkv, D, cap, window = case["B"], case["Hq"], case["Hkv"], case["D"], case["softcap"], case["window"]
    n, L, ps = st["max_q"], st["max_kv"], case["page"]
    pages = st["page_table"][:, :-(-L // ps)].clamp(min=0).long()
    tiles = st["cache"][pages].transpose(1, 2).flatten(2, 3)                                            # [B, Hkv, keys / 16, 18 D]
    k, v = _values(tiles[..., :9 * D], D)[:, :, None, :L], _values(tiles[..., 9 * D:], D)[:, :, None, :L]
    seq, row = st["seq"], st["row"]
    q = torch.zeros(B, n, Hq, D, device="cuda")
    q[seq, row] = st["q"].float()
    pos = torch.full((B, n), L, dtype=torch.int64, device="cuda")
    pos[seq, row] = st["pos"]
    key = torch.arange(L, device="cuda")
    hidden = key > pos.unsqueeze(-1)
    if window:
        hidden |= key <= pos.unsqueeze(-1) - window
    s = (q.view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4) @ k.transpose(-1, -2)).mul_(st["scale"])    # [B, Hkv, heads of a group, n, L]
    if cap:
        s = s.div_(cap).tanh_().mul_(cap)
    s.masked_fill_(hidden[:, None, None], -math.inf)
    s -= s.amax(-1, keepdim=True)
    s.exp_()
    o = (s @ v) / s.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[seq, row].to(torch.bfloat16)


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "quantize":
        W = st["W"].to(f64).reshape(case["N"], -1, case["group"])
        low, top = W.min(-1).values, W.max(-1).values
        return None, torch.stack([(top - low) / 15.0, low], -1)        # the codes are whole numbers by definition
    if case["op"] == "linear":
        N, K = case["N"], case["K"]
        W = torch.empty(N, K, dtype=f64, device="cuda")
        W[:, 0::2] = (st["packed"] % 16).to(f64)
        W[:, 1::2] = (st["packed"] // 16).to(f64)
        scale, low = st["params"][..., 0].to(f64), st["params"][..., 1].to(f64)
        W = torch.addcmul(low.unsqueeze(-1), W.reshape(N, -1, case["group"]), scale.unsqueeze(-1)).reshape(N, K)
        return torch.matmul(st["x"].to(f64), W.t())
    ps, D, Hq, Hkv = case["page"], case["D"], case["Hq"], case["Hkv"]
    table = st["page_table"].long()
    if case["op"] == "append":
        half = case["rot"] // 2
        q_out = st["q"].to(f64).clone()
        first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)
        for b, (n, ctx) in enumerate(st["lens"]):
            block = q_out[st["cu"][b]:st["cu"][b + 1]]
            p = torch.arange(ctx, ctx + n, device="cuda")
            c, s = st["cos_sin"][p, :half].to(f64).unsqueeze(1), st["cos_sin"][p, half:].to(f64).unsqueeze(1)
            u, w = block[..., first].clone(), block[..., second].clone()
            block[..., first] = u * c - w * s
            block[..., second] = u * s + w * c
        return q_out, None                                               # bytes: whole numbers by definition

    def cached(page, slot, h, at):
        """Keys (at = 0) or values (at = 9 D) of one head, [keys, D]."""
        out = torch.empty(len(page), D, dtype=f64, device="cuda")
        tile = st["cache"][page, h, slot // TILE]
        key = slot % TILE
        every = torch.arange(len(page), device="cuda")
        for d in range(0, D, GROUP):
            p = torch.stack([tile[every, at + 8 * D + d + 4 * key + i] for i in range(4)], -1).view(torch.bfloat16).to(f64)
            for j in range(GROUP // 2):
                e = d + 2 * j
                byte = tile[every, at + 256 * (e // 32) + 16 * key + (e % 32) // 2]
                out[:, e] = (byte % 16).to(f64) * p[:, 0] + p[:, 1]
                out[:, e + 1] = (byte // 16).to(f64) * p[:, 0] + p[:, 1]
        return out

    out = torch.zeros(st["q"].shape, dtype=f64, device="cuda")
    G = Hq // Hkv
    for b, (n, ctx) in enumerate(st["lens"]):
        L = n + ctx
        where = torch.arange(L, device="cuda")
        page, slot = table[b][where // ps], where % ps
        for h in range(Hkv):
            k, v = cached(page, slot, h, 0), cached(page, slot, h, 9 * D)
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
                    out[rows, head] = torch.softmax(logits.masked_fill(hidden, -math.inf), -1) @ v
    return out
