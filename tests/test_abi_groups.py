"""Refusals of the entry points on 4-bit groups, and the plain forms that their GPU tests use (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr

lib = mq._lib
P = 0x10000              # never dereferenced: validation fails first
NULL = None


def test_quantize_groups_refusals():
    def call(W=P, N=4, K=256, ldw=256, group=64, packed=P, params=P):
        return lib.matq_quantize_groups(W, N, K, ldw, group, packed, params, NULL, NULL)
    for kw in (dict(W=NULL), dict(packed=NULL), dict(params=NULL), dict(N=-1), dict(K=-64)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for group in (0, -64, 16, 48, 256):
        assert call(group=group) == mq.ERR_UNSUPPORTED
    for kw in (dict(K=0), dict(K=224), dict(ldw=248), dict(ldw=260), dict(K=1 << 31, ldw=1 << 31), dict(N=1 << 31), dict(N=(1 << 31) - 1, K=1 << 30, ldw=1 << 30)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(W=P + 8), dict(packed=P + 4), dict(params=P + 4)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(N=0, W=NULL) == mq.OK


def test_gemv_groups_refusals():
    def call(packed=P, N=8, K=256, group=64, params=P, x=P, M=2, ldx=256, out=mq.OUT_F32, y=P, ldy=8, flags=0):
        return lib.matq_gemv_groups(packed, N, K, group, params, x, M, ldx, out, y, ldy, flags, NULL)
    for kw in (dict(packed=NULL), dict(params=NULL), dict(x=NULL), dict(y=NULL), dict(N=-1), dict(K=-64), dict(M=-1), dict(out=2), dict(flags=1), dict(flags=0x200)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for group in (0, 16, 96, 256):
        assert call(group=group) == mq.ERR_UNSUPPORTED
    for kw in (dict(K=0), dict(K=224), dict(K=65600, ldx=65600), dict(ldx=248), dict(ldx=260), dict(ldy=7), dict(N=1 << 31, ldy=1 << 31), dict(M=1 << 40)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(packed=P + 8), dict(params=P + 8), dict(x=P + 8)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(M=0, x=NULL) == mq.OK and call(N=0, ldy=0, packed=NULL) == mq.OK


def _cache(**kw):
    c = mq.PagedKv4(P, 10, 16, 2, 64, 3, P, 8, 8, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_kv4_append_refusals():
    def call(T=5, q=P, qh=4, ldq=256, k=P, ldk=128, v=P, ldv=128, cs=P, max_pos=100, rot=64, inter=0, qo=P + 0x1000, ldqo=256, **kw):
        c = _cache(**kw)
        return lib.matq_kv4_append(C.byref(c), T, q, qh, ldq, k, ldk, v, ldv, cs, max_pos, rot, inter, qo, ldqo, NULL, NULL)
    assert lib.matq_kv4_append(None, 1, P, 4, 256, P, 128, P, 128, P, 9, 64, 0, P, 256, NULL, NULL) == mq.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(q=NULL), dict(qo=NULL), dict(k=NULL), dict(v=NULL), dict(cs=NULL), dict(rot=-16), dict(qh=-1), dict(max_pos=-1), dict(page_size=0),
               dict(kv_heads=0), dict(head_dim=0), dict(batch=-1), dict(n_pages=-1), dict(table_width=-1), dict(table_stride=7), dict(page_table=None), dict(cu_q=None),
               dict(kv_len=None), dict(tiles=None), dict(qo=P, ldqo=264)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=80), dict(page_size=8), dict(page_size=24)):
        assert call(**kw) == mq.ERR_UNSUPPORTED, kw
    for kw in (dict(rot=8), dict(rot=80), dict(ldk=120), dict(ldk=132), dict(ldv=127), dict(ldq=248), dict(ldqo=260), dict(T=1 << 31)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(q=P + 8), dict(qo=P + 0x1008), dict(k=P + 2), dict(v=P + 8), dict(cs=P + 4), dict(tiles=P + 8)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(T=0) == mq.OK and call(batch=0) == mq.OK


def test_attn_paged4_refusals():
    def call(T=5, q=P, qh=4, ldq=256, scale=0.1, cap=0.0, window=0, max_q=5, max_kv=100, out=P, ldo=256, ws=P, ws_bytes=1 << 40, **kw):
        c = _cache(**kw)
        return lib.matq_attn_paged4(C.byref(c), T, q, qh, ldq, scale, cap, window, max_q, max_kv, out, ldo, ws, ws_bytes, NULL, NULL)
    nan = float("nan")
    for kw in (dict(T=-1), dict(q=NULL), dict(out=NULL), dict(qh=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(cap=-1.0), dict(cap=nan), dict(window=-1),
               dict(max_q=-1), dict(max_kv=-1), dict(kv_heads=0), dict(n_pages=0), dict(table_width=-1), dict(table_stride=7), dict(page_table=None), dict(cu_q=None), dict(kv_len=None),
               dict(tiles=None)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=96, ldq=384, ldo=384), dict(page_size=8), dict(page_size=48), dict(qh=5, ldq=320, ldo=320), dict(qh=130, ldq=130 * 64, ldo=130 * 64)):
        assert call(**kw) == mq.ERR_UNSUPPORTED, kw
    for kw in (dict(ldq=248), dict(ldq=260), dict(ldo=248), dict(ldo=258), dict(T=1 << 31), dict(n_pages=1 << 31), dict(kv_heads=1 << 23, qh=1 << 23, ldq=1 << 29, ldo=1 << 29)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(q=P + 8), dict(out=P + 8), dict(ws=P + 8), dict(tiles=P + 8)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    assert call(max_kv=100000, ws=NULL, ws_bytes=0) == mq.ERR_WORKSPACE
    assert call(T=4000, max_q=4000, max_kv=8000, ws=NULL, ws_bytes=0) == mq.ERR_WORKSPACE
    big = (1 << 31) - 1
    assert call(kv_heads=1 << 22, qh=1 << 22, ldq=1 << 28, ldo=1 << 28, batch=big, T=big, ws=NULL, ws_bytes=0) == mq.ERR_SHAPE         # a grid of 2^53
    assert call(T=0) == mq.OK and call(batch=0) == mq.OK


def test_attn_paged4_workspace():
    f = mq.attn_paged4_workspace_bytes
    assert f(0, 1, 8, 2, 128, 1, 1000) == 0 and f(4, 0, 8, 2, 128, 1, 1000) == 0 and f(4, 1, 8, 3, 128, 1, 1000) == 0 and f(4, 1, 8, 2, 96, 1, 1000) == 0
    assert f(1, 1, 32, 8, 128, 1, 64) == 0
    assert 0 < f(1, 1, 32, 8, 128, 1, 32768) < 1 << 24
    one = f(4096, 1, 32, 8, 128, 4096, 8192)
    assert one >= 8192 * 8 * 128 * 4                           # the keys and values of the chunk
    many = f(4096, 64, 32, 8, 128, 4096, 32768)
    assert many < 1 << 30                                      # not those of all the sequences at once
    # bounds that say nothing: the cache is read as it is, and the workspace holds partial outputs only
    assert f(4096, 1, 32, 8, 128, 4096, (1 << 31) - 1) <= 256 << 20 and f(4096, 1, 32, 8, 128, 4096, 5 << 20) <= 256 << 20
    huge = (1 << 63) - 1
    assert f(4, 1, 8, 2, 128, huge, 32768) == f(4, 1, 8, 2, 128, 4, 32768)
    assert f(4, 1, 8, 2, 128, 4, huge) == f(4, 1, 8, 2, 128, 4, (1 << 31) - 1) > 0
    assert f(4, 1, 8, 2, 128, 4, 32768, huge) == f(4, 1, 8, 2, 128, 4, 32768)
    assert f(4000, 1, 8, 2, 128, 4000, 1 << 20, 4096) < f(4000, 1, 8, 2, 128, 4000, 1 << 20) // 2      # a window bounds what is unpacked


def test_tile_bytes():
    assert [mq.kv4_tile_bytes(d) for d in (64, 128, 256)] == [1152, 2304, 4608]
    assert mq.kv4_tile_bytes(80) == mq.kv4_tile_bytes(0) == mq.kv4_tile_bytes(-64) == -1


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    u = torch.zeros(4, 64, dtype=torch.uint8)
    p = torch.zeros(4, 2, 2, dtype=torch.bfloat16)
    t = torch.zeros(1, 2, dtype=torch.int32)
    for f in (lambda: mq.quantize_groups(x, 64), lambda: mq.gemv_groups(u, p, x), lambda: mq.kv4_append(u, t, t[0], t[0], x, x),
              lambda: mq.attn_paged4(torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 1, 18 * 64, dtype=torch.uint8), t, t[0], t[0], 1, 1),
              lambda: mq._serving.gemv_groups(1, 2), lambda: mq._serving.attn_paged4(1)):
        with pytest.raises(TypeError):
            f()


def test_plain_forms_agree_with_one_another():
    """A cache's bytes stand for the values of its groups, tile by tile, and a value is off by half a step of its group at most (and the rounding of the scale)."""
    rng = np.random.default_rng(0)
    k, v = (gr.bf16_bits(rng.standard_normal((2, 3, 32, 128), dtype=np.float32)) for _ in range(2))
    tiles = gr.cache_bytes(k, v)
    assert tiles.shape == (2, 3, 2, 18 * 128)
    for h in range(2):
        half = gr.tile_half(*gr.quantise(k[1, 2, 16 * h:16 * h + 16], 64))
        assert np.array_equal(tiles[1, 2, h, :9 * 128], half)
    kd, vd = gr.cache_values(tiles)[:2]
    for bits, got in ((k, kd), (v, vd)):
        x = gr.bf16_values(bits).astype(np.float64)
        g = x.reshape(2, 3, 32, 2, 64)
        step = (g.max(-1) - g.min(-1)) / 15
        assert (np.abs(got.numpy() - x).reshape(g.shape) <= (0.5 + 16 * 2.0 ** -8) * step[..., None]).all()
