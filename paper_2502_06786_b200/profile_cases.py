"""Small, self-contained invocations of each kernel for profilers (ncu wants short runs with few launches).

    python -m paper_2502_06786_b200.profile_cases quantize|slice4|slice2ep|gemv4|gemv2|gemv2b8|gemv4t|gemv2t|stream8|stream4|stream2|group4|group2|batch4|batch8|gemm|linear|attend|groups|attend4

(gemv4 / gemv2: the library's own choice at B = 1, the integer tensor kernel; a trailing t: the bf16 tensor kernel.)

Every case touches a few hundred MB of distinct buffers (more than the L2 holds) and launches each kernel 16-24 times.
"""
from __future__ import annotations

import sys

import torch

from . import binding as mq
from . import synth


def _planes(n, N, K, r):
    return [torch.randint(0, 256, (N, K * r // 8), dtype=torch.uint8, device="cuda") for _ in range(n)]


def main(which: str) -> None:
    N, K = 9216, 2304                       # a Gemma-2-2B gate / up matrix
    n = 12
    if which == "quantize":
        Ws = [torch.randn(N, K, device="cuda").mul_(0.02).to(torch.bfloat16) for _ in range(n)]
        outs = [(torch.empty(N, K, dtype=torch.uint8, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")) for _ in range(n)]
        for _ in range(2):
            for W, (q, a, z) in zip(Ws, outs):
                mq.quantize(W, q=q, alpha=a, zero=z)
    elif which in ("slice4", "slice2ep"):
        qs = [torch.from_numpy(synth.skewed_codes((N, K), 0.005, 224, 10 + i)).cuda() for i in range(n)]
        for _ in range(2):
            for q in qs:
                if which == "slice4":
                    mq.slice_pack(q, 4)
                else:
                    mq.slice_pack(q, 2, extra_precision=True, ovf_capacity=N * K // 16)
    elif which in ("gemv4", "gemv2", "gemv2b8", "gemv4t", "gemv2t"):
        r = 4 if which.startswith("gemv4") else 2
        flags = mq.GEMV_TENSOR if which.endswith("t") else mq.GEMV_AUTO
        B = 8 if which.endswith("b8") else 1
        n = 24
        P = _planes(n, N, K, r)
        X = [torch.randn(B, K, device="cuda").to(torch.bfloat16) for _ in range(n)]
        Y = [torch.empty(B, N, device="cuda") for _ in range(n)]
        a = torch.ones(N, device="cuda")
        for _ in range(2):
            for i in range(n):
                mq.gemv(P[i], K, r, a, a, X[i], y=Y[i], flags=flags)
    elif which in ("stream8", "stream4", "stream2"):
        # the persistent kernel on a plane large enough for its steady state: 65536 x 2304, one problem per launch
        r = int(which[-1])
        N3 = 65536
        P = _planes(4, N3, K, r)
        X = [torch.randn(1, K, device="cuda").to(torch.bfloat16) for _ in range(4)]
        Y = [torch.empty(1, N3, device="cuda") for _ in range(4)]
        a = torch.ones(N3, device="cuda")
        for _ in range(2):
            for i in range(4):
                mq.gemv(P[i], K, r, a, a, X[i], y=Y[i], flags=mq.GEMV_STREAM)
    elif which in ("group4", "group2"):
        # twelve matrices of the Gemma-2-2B MLP stack (4 layers) in one matq_gemv_grouped call
        r = int(which[-1])
        shapes = [(9216, 2304), (9216, 2304), (2304, 9216)] * 4
        P = [torch.randint(0, 256, (n_, k_ * r // 8), dtype=torch.uint8, device="cuda") for n_, k_ in shapes]
        X = [torch.randn(k_, device="cuda").to(torch.bfloat16) for n_, k_ in shapes]
        Y = [torch.empty(n_, device="cuda") for n_, k_ in shapes]
        a = torch.ones(9216, device="cuda")
        g = mq.gemv_group([(P[i], shapes[i][1], r, a[:shapes[i][0]], a[:shapes[i][0]], X[i], Y[i]) for i in range(len(shapes))])
        for _ in range(3):
            mq.gemv_grouped(g)
    elif which in ("batch4", "batch8"):
        # twelve matrices of the Gemma-2-2B MLP stack at r = 4 with 4 or 8 activation vectors each, one matq_gemv_grouped call
        B = int(which[-1])
        shapes = [(9216, 2304), (9216, 2304), (2304, 9216)] * 4
        P = [torch.randint(0, 256, (n_, k_ // 2), dtype=torch.uint8, device="cuda") for n_, k_ in shapes]
        X = [torch.randn(B, k_, device="cuda").to(torch.bfloat16) for n_, k_ in shapes]
        Y = [torch.empty(B, n_, device="cuda") for n_, k_ in shapes]
        a = torch.ones(9216, device="cuda")
        g = mq.gemv_group([(P[i], shapes[i][1], 4, a[:shapes[i][0]], a[:shapes[i][0]], X[i], Y[i]) for i in range(len(shapes))])
        for _ in range(3):
            mq.gemv_grouped(g)
    elif which == "gemm":
        N2, K2, M2 = 14336, 4096, 1024      # the Mistral-7B matrix with a quarter of the tokens
        q = torch.randint(0, 256, (N2, K2), dtype=torch.uint8, device="cuda")
        X = torch.randn(M2, K2, device="cuda").to(torch.bfloat16)
        a = torch.full((N2,), 1e-3, device="cuda")
        Ys = [torch.empty(M2, N2, device="cuda") for _ in range(3)]
        ws = torch.empty(mq.gemm_multi_workspace_bytes(mq.SRC_CODES8, M2, N2, K2, 3), dtype=torch.uint8, device="cuda")
        for _ in range(3):
            mq.gemm_multi(mq.SRC_CODES8, q, K2, X, alpha=a, zero=a, Ys=Ys, workspace=ws)
    elif which == "linear":
        # the linear layer on the codes themselves: one token, 64 and 1024 tokens (split kernel with tiles of 16 and 64 tokens, pair kernel)
        N2, K2 = 14336, 4096
        qs = [torch.randint(0, 256, (N2, K2), dtype=torch.uint8, device="cuda") for _ in range(4)]
        a = torch.full((N2,), 1e-3, device="cuda")
        z = torch.full((N2,), 128.0, device="cuda")
        for M in (1, 64, 1024):
            X = torch.randn(M, K2, device="cuda").to(torch.bfloat16)
            Y = torch.empty(M, N2, dtype=torch.bfloat16, device="cuda")
            for q in qs:
                mq.gemm_a8(*mq.quantize_tokens(X), q, a, z, y=Y)
    elif which == "attend":
        # append and attention over a paged cache: one token over 32768 keys of 8 heads of 128, 500 over 6500 of 8 heads of 256, 2048 over 4096 of 8 heads of 128
        for new, keys, D, Hq, Hkv in ((1, 32768, 128, 32, 8), (500, 6500, 256, 16, 8), (2048, 4096, 128, 32, 8)):
            pages = 3 * (keys + 63) // 64
            kc = torch.randn(pages, Hkv, 64, D, device="cuda").to(torch.bfloat16)
            vc = torch.randn_like(kc)
            table = torch.randperm(pages, device="cuda").to(torch.int32)[: (keys + 63) // 64].unsqueeze(0)
            cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
            lens = torch.tensor([keys], dtype=torch.int32, device="cuda")
            q = torch.randn(new, Hq, D, device="cuda").to(torch.bfloat16)
            k, v = (torch.randn(new, Hkv, D, device="cuda").to(torch.bfloat16) for _ in range(2))
            ang = torch.rand(keys, D, device="cuda")
            for _ in range(3):
                mq.kv_append(kc, vc, table, cu, lens, k, v, cos_sin=ang, q=q, q_out=q)
                mq.attn_paged(q, kc, vc, table, cu, lens, new, keys)
    elif which == "groups":
        # weights in 4-bit groups of 128: the quantiser, one token, 16, 64 and 1024 through a Gemma-2-2B gate matrix
        Ws = [torch.randn(N, K, device="cuda").mul_(0.02).to(torch.bfloat16) for _ in range(n)]
        held = [mq.quantize_groups(W, 128) for W in Ws]
        for M in (1, 16, 64, 1024):
            X = torch.randn(M, K, device="cuda").to(torch.bfloat16)
            Y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
            for packed, params in held:
                mq.gemv_groups(packed, params, X, y=Y)
    elif which == "attend4":
        # append to and attention over a 4-bit paged cache: 16 single tokens over 8192 keys of 8 heads of 128, 6 drafted tokens each, 2048 tokens over 4096
        for batch, new, keys in ((16, 1, 8192), (16, 6, 8192), (1, 2048, 4096)):
            pages = batch * keys // 64
            cache = torch.randint(0, 64, (pages, 8, 4, mq.kv4_tile_bytes(128)), dtype=torch.uint8, device="cuda")
            table = torch.randperm(pages, device="cuda").to(torch.int32).view(batch, -1)
            cu = torch.arange(batch + 1, device="cuda").to(torch.int32) * new
            lens = torch.full((batch,), keys, dtype=torch.int32, device="cuda")
            q = torch.randn(batch * new, 32, 128, device="cuda").to(torch.bfloat16)
            k, v = (torch.randn(batch * new, 8, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
            ang = torch.rand(keys, 128, device="cuda")
            for _ in range(3):
                mq.kv4_append(cache, table, cu, lens, k, v, cos_sin=ang, q=q, q_out=q)
                mq.attn_paged4(q, cache, table, cu, lens, new, keys)
    else:
        raise SystemExit(__doc__)
    torch.cuda.synchronize()
    print("ok", which)


if __name__ == "__main__":
    main(sys.argv[1] if len(sys.argv) > 1 else "")
