"""Refusals of the serving entry points: found on the host, before anything is launched (no GPU needed)."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2502_06786_b200 import binding as mq

lib = mq._lib
P = 0x10000              # never dereferenced: validation fails first
NULL = None


def test_status_strings():
    assert mq.status_string(mq.ERR_PAGE) not in ("ok", "unknown status")


def test_quantize_tokens_refusals():
    def call(X=P, M=4, K=64, ldx=64, xq=P, ldq=64, scale=P, rowsum=P):
        return lib.matq_quantize_tokens(X, M, K, ldx, xq, ldq, scale, rowsum, NULL, NULL)
    for kw in (dict(X=NULL), dict(xq=NULL), dict(scale=NULL), dict(rowsum=NULL), dict(M=-1), dict(K=0)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for kw in (dict(K=60), dict(K=65552, ldx=65552, ldq=65552), dict(ldx=56), dict(ldx=68), dict(ldq=48), dict(ldq=72), dict(M=1 << 31)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    assert call(X=P + 8) == mq.ERR_ALIGNMENT and call(xq=P + 8) == mq.ERR_ALIGNMENT
    assert call(M=0, X=NULL) == mq.OK


def test_gemm_a8_refusals():
    def call(xq=P, M=4, K=64, ldx=64, xs=P, xsum=P, q=P, N=8, ldw=64, c=8, a=P, z=P, out=mq.OUT_F32, Y=P, ldy=8, flags=0):
        return lib.matq_gemm_a8(xq, M, K, ldx, xs, xsum, q, N, ldw, c, a, z, out, Y, ldy, flags, NULL, NULL)
    for kw in (dict(xq=NULL), dict(xs=NULL), dict(xsum=NULL), dict(q=NULL), dict(a=NULL), dict(z=NULL), dict(Y=NULL), dict(M=-1), dict(N=-1), dict(K=0),
               dict(out=2), dict(flags=1), dict(flags=0x200)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    assert call(c=4) == mq.ERR_UNSUPPORTED
    for kw in (dict(K=72, ldx=80, ldw=80), dict(K=65552, ldx=65552, ldw=65552), dict(ldx=48), dict(ldx=72), dict(ldw=48), dict(ldw=72), dict(ldy=7), dict(M=1 << 31), dict(N=1 << 31, ldy=1 << 31)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    assert call(xq=P + 8) == mq.ERR_ALIGNMENT and call(q=P + 4) == mq.ERR_ALIGNMENT
    assert call(M=0, xq=NULL) == mq.OK and call(N=0, ldy=0, q=NULL) == mq.OK


def _cache(**kw):
    c = mq.PagedKv(P, P, 10, 16, 2, 64, 3, P, 8, 8, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_kv_append_refusals():
    def call(T=5, q=P, qh=4, ldq=256, k=P, ldk=128, v=P, ldv=128, cs=P, max_pos=100, rot=64, inter=0, qo=P + 0x1000, ldqo=256, **kw):
        c = _cache(**kw)
        return lib.matq_kv_append(C.byref(c), T, q, qh, ldq, k, ldk, v, ldv, cs, max_pos, rot, inter, qo, ldqo, NULL, NULL)
    assert lib.matq_kv_append(None, 1, P, 4, 256, P, 128, P, 128, P, 9, 64, 0, P, 256, NULL, NULL) == mq.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(q=NULL), dict(qo=NULL), dict(k=NULL), dict(v=NULL), dict(cs=NULL), dict(rot=-16), dict(qh=-1), dict(max_pos=-1), dict(page_size=0),
               dict(kv_heads=0), dict(head_dim=0), dict(batch=-1), dict(n_pages=-1), dict(table_width=-1), dict(table_stride=7), dict(page_table=None), dict(cu_q=None),
               dict(kv_len=None), dict(qo=P, ldqo=264)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for kw in (dict(rot=8), dict(rot=80), dict(head_dim=60), dict(ldk=120), dict(ldk=132), dict(ldv=127), dict(ldq=248), dict(ldqo=260), dict(T=1 << 31)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(q=P + 8), dict(qo=P + 0x1008), dict(k=P + 2), dict(v=P + 8), dict(cs=P + 4)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(T=0) == mq.OK and call(batch=0) == mq.OK


def test_attn_paged_refusals():
    def call(T=5, q=P, qh=4, ldq=256, scale=0.1, cap=0.0, window=0, max_q=5, max_kv=100, out=P, ldo=256, ws=P, ws_bytes=1 << 30, **kw):
        c = _cache(**kw)
        return lib.matq_attn_paged(C.byref(c), T, q, qh, ldq, scale, cap, window, max_q, max_kv, out, ldo, ws, ws_bytes, NULL, NULL)
    nan = float("nan")
    for kw in (dict(T=-1), dict(q=NULL), dict(out=NULL), dict(qh=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(cap=-1.0), dict(cap=nan), dict(window=-1),
               dict(max_q=-1), dict(max_kv=-1), dict(kv_heads=0), dict(n_pages=0), dict(table_width=-1), dict(table_stride=7), dict(page_table=None), dict(cu_q=None), dict(kv_len=None)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=96, ldq=384, ldo=384), dict(page_size=8), dict(page_size=48), dict(qh=5, ldq=320, ldo=320), dict(qh=130, ldq=130 * 64, ldo=130 * 64)):
        assert call(**kw) == mq.ERR_UNSUPPORTED, kw
    for kw in (dict(ldq=248), dict(ldq=260), dict(ldo=248), dict(ldo=258), dict(T=1 << 31), dict(n_pages=1 << 27)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(q=P + 8), dict(out=P + 8), dict(ws=P + 8)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(max_kv=100000, ws=NULL, ws_bytes=0) == mq.ERR_WORKSPACE
    assert call(T=0) == mq.OK and call(batch=0) == mq.OK


def test_attn_paged_workspace():
    f = mq.attn_paged_workspace_bytes
    assert f(0, 1, 8, 2, 128, 1, 1000) == 0 and f(4, 0, 8, 2, 128, 1, 1000) == 0 and f(4, 1, 8, 3, 128, 1, 1000) == 0
    assert f(1, 1, 32, 8, 128, 1, 32768) > 0                   # one long sequence is split
    assert f(1, 1, 32, 8, 128, 1, 64) == 0                     # a short one is not
    assert f(8192, 1, 32, 8, 128, 8192, 16384) == 0            # nor a chunk that fills the GPU by itself


def test_attn_paged_sizes_past_every_range():
    """Products of sizes that pass 32 and 64 bits are refused before anything is launched; hints of any size choose some plan."""
    def call(T=5, qh=4, ldq=256, window=0, max_q=5, max_kv=100, ws_bytes=0, **kw):
        c = _cache(**kw)
        return lib.matq_attn_paged(C.byref(c), T, P, qh, ldq, 0.1, 0.0, window, max_q, max_kv, P, ldq, NULL, ws_bytes, NULL, NULL)
    big = (1 << 31) - 1
    assert call(kv_heads=1 << 30, qh=1 << 30, ldq=1 << 36, page_size=256, n_pages=1 << 30) == mq.ERR_SHAPE       # pages * heads * slots = 2^68
    assert call(kv_heads=1 << 22, qh=1 << 22, ldq=1 << 28, n_pages=32, batch=big, T=big) == mq.ERR_SHAPE         # a grid of 2^53
    assert call(batch=1, table_width=1, max_q=(1 << 63) - 1, max_kv=(1 << 63) - 1, window=(1 << 63) - 1) == mq.ERR_WORKSPACE      # a long range is split
    f = mq.attn_paged_workspace_bytes
    huge = (1 << 63) - 1
    assert f(4, 1, 8, 2, 128, huge, 32768) == f(4, 1, 8, 2, 128, 4, 32768) > 0
    assert f(4, 1, 8, 2, 128, 4, huge) == f(4, 1, 8, 2, 128, 4, big) > 0
    assert f(4, 1, 8, 2, 128, 4, 32768, huge) == f(4, 1, 8, 2, 128, 4, 32768)


def test_binding_refuses_host_tensors_and_wrong_types():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        mq.quantize_tokens(x)
    with pytest.raises(TypeError):
        mq.gemm_a8(x, x, x, x, x, x)
    kc = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    t = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(TypeError):
        mq.kv_append(kc, kc, t, t[0], t[0], x, x)
    with pytest.raises(TypeError):
        mq.attn_paged(torch.zeros(4, 2, 64, dtype=torch.bfloat16), kc, kc, t, t[0], t[0], 1, 1)
    with pytest.raises(TypeError):
        mq._serving.gemm_a8(1, 2)


def test_gemm_a8_has_a_kernel_for_every_size_it_accepts():
    """The choice of kernel and tile is host arithmetic: every accepted size has one, up to the limits of M and N."""
    big = (1 << 31) - 1
    sizes = [1, 2, 8, 9, 16, 17, 32, 33, 64, 100, 128, 129, 509, 1024, 1025, 4096, 65535, 128 * 65535, 128 * 65535 + 1, 9000000, 1 << 30, big - 1, big]
    for M in sizes:
        for N in sizes:
            for K in (16, 144, 4096, 65536):
                tiles = -(-M // 256) * -(-N // 256)
                try:
                    kernel, tokens, parts = mq.gemm_a8_plan(M, N, K)
                except mq.MatqError as e:
                    assert e.status == mq.ERR_SHAPE and tiles >= 1 << 30, (M, N, K)
                    continue
                if kernel == mq.GEMM_A8_FEW:
                    assert M <= tokens == 8 and parts == 1
                elif kernel == mq.GEMM_A8_SPLIT:
                    assert tokens in (16, 32, 64, 128) and parts in (1, 2, 4, 8) and -(-M // tokens) <= 65535, (M, N, K)
                    assert parts <= -(-K // 256) and -(-N // 128) * parts < 1 << 31
                else:
                    assert kernel == mq.GEMM_A8_PAIRS and tokens in range(64, 257, 32) and parts == 1
                    assert -(-M // tokens) * -(-N // 256) < 1 << 30
    assert mq.gemm_a8_plan(128 * 65535 + 1, 256, 256)[0] == mq.GEMM_A8_PAIRS
    for M, N, K, st in ((0, 1, 16, mq.ERR_INVALID_ARG), (1, 0, 16, mq.ERR_INVALID_ARG), (-1, 1, 16, mq.ERR_INVALID_ARG), (1, 1, 0, mq.ERR_INVALID_ARG),
                        (1, 1, 24, mq.ERR_SHAPE), (1, 1, 65552, mq.ERR_SHAPE), (1 << 31, 1, 16, mq.ERR_SHAPE), (1, 1 << 31, 16, mq.ERR_SHAPE)):
        assert lib.matq_gemm_a8_plan(M, N, K, NULL, NULL, NULL) == st, (M, N, K)
    assert lib.matq_gemm_a8_plan(1, 1, 16, NULL, NULL, NULL) == mq.OK


def test_one_function_of_the_serving_module_looks_at_the_device_of_every_tensor():
    # that a tensor of another device is refused cannot be shown with one GPU or none, so the source is read: no argument becomes a pointer around tensor()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_b200", "csrc", "serving_module.cpp")
    text = open(path).read()
    assert text.count("is_cuda()") == 1 and text.count("current_device()") == 1
    assert re.findall(r"(\w+)?\(?THPVariable_Unpack\(\w+(?:\[\d+\])?\)(\.\w+)?", text) == [("", ""), ("", ".scalar_type")]
