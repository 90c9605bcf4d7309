"""Refusals of the linear layer on 4-bit groups for many tokens, and its workspace (no GPU needed)."""
from paper_2502_06786_b200 import binding as mq

lib = mq._lib
P = 0x10000              # never dereferenced: validation fails first
NULL = None


def test_gemm_groups_refusals():
    def call(packed=P, N=8, K=256, group=64, params=P, x=P, M=40, ldx=256, out=mq.OUT_F32, y=P, ldy=8, ws=P, ws_bytes=1 << 30):
        return lib.matq_gemm_groups(packed, N, K, group, params, x, M, ldx, out, y, ldy, ws, ws_bytes, NULL, NULL)
    for kw in (dict(packed=NULL), dict(params=NULL), dict(x=NULL), dict(y=NULL), dict(N=-1), dict(K=-64), dict(M=-1), dict(out=2)):
        assert call(**kw) == mq.ERR_INVALID_ARG, kw
    for group in (0, 16, 96, 256):
        assert call(group=group) == mq.ERR_UNSUPPORTED
    for kw in (dict(K=0), dict(K=224), dict(K=65600, ldx=65600), dict(ldx=248), dict(ldx=260), dict(ldy=7), dict(N=1 << 31, ldy=1 << 31), dict(M=1 << 31),
               dict(M=1 << 24, N=1 << 30, ldy=1 << 30)):
        assert call(**kw) == mq.ERR_SHAPE, kw
    for kw in (dict(packed=P + 8), dict(params=P + 8), dict(x=P + 8), dict(ws=P + 8)):
        assert call(**kw) == mq.ERR_ALIGNMENT, kw
    need = mq.gemm_groups_workspace_bytes(40, 8, 256, 64)
    for kw in (dict(ws=NULL), dict(ws_bytes=need - 1), dict(ws_bytes=0)):
        assert call(**kw) == mq.ERR_WORKSPACE, kw
    assert call(M=0, x=NULL, ws=NULL) == mq.OK and call(N=0, ldy=0, packed=NULL, ws=NULL) == mq.OK


def test_gemm_groups_workspace_and_choice():
    f, pays = mq.gemm_groups_workspace_bytes, mq.gemm_groups_pays
    assert f(0, 8, 256, 64) == f(8, 0, 256, 64) == f(8, 8, 250, 64) == f(8, 8, 256, 16) == f(8, 8, 65600, 32) == 0
    M, N, K = 4096, 14336, 4096
    assert 2 * M * K < f(M, N, K, 128) < 2.2 * M * K + 4 * N * K // 128 + (1 << 20)
    assert f(1 << 20, 1 << 20, 65536, 32) > 1 << 37
    assert pays(33, 64, 64, 64) and pays(17, 14336, 4096, 128) and not pays(17, 2304, 2304, 64) and not pays(16, 65536, 65536, 64) and not pays(100, 64, 100, 64)
