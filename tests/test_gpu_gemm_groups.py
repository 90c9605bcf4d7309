"""Linear layer on weights in 4-bit groups for many tokens, against plain forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import synth
from tests import groups_ref as gr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu


def _case(M, N, K, group, seed, std=1.0):
    rng = np.random.default_rng(seed)
    w = gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02)
    codes, params = gr.quantise(w, group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32) * std).to(torch.bfloat16)
    return codes, params, x


def _check(y, want, tol):
    y = y.double().cpu()
    if not bool(((y - want).abs() <= tol).all()):
        raise AssertionError(float(((y - want).abs() / tol).max()))


def _run(codes, params, x, out_dtype=torch.float32, **kw):
    status = status_word()
    y = mq.gemm_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda(), out_dtype=out_dtype, dev_status=status, **kw)
    assert int(host(status)[0]) == mq.OK
    return y


# one block and less of K, odd numbers of blocks, rows and tokens that end inside a tile, K shared by 2, 4 and 8 CTAs, several tiles a CTA
SHAPES = [(1, 1, 128), (16, 128, 128), (17, 130, 256), (3, 1000, 384), (100, 129, 896), (128, 256, 1024), (129, 300, 2304), (40, 2500, 4096 - 128), (257, 128, 1152),
          (64, 100, 14336), (33, 20, 65536), (500, 700, 640)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_groups(M, N, K, group, out_dtype):
    codes, params, x = _case(M, N, K, group, M + N + K)
    y = _run(codes, params, x, out_dtype)
    bf16 = out_dtype == torch.bfloat16
    want, tol = gr.gemm(codes, params, x, bf16)
    _check(y, want, tol + (2.0 ** -8 * want.abs() if bf16 else 0))
    if not bf16:                                                 # 64 steps, each of which cuts off half a unit of 2^-23 on average
        assert float((y.double().cpu() - want).norm() / want.norm()) < 64 * 2.0 ** -24


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K,group", [(300, 9000, 256, 128), (700, 5001, 288, 32), (1000, 6000, 192, 64), (20, 40000, 128, 32)])
def test_gemm_groups_more_tiles_than_sms(M, N, K, group, out_dtype):
    # with bf16 outputs by pairs of CTAs, whose last tile may be half empty
    g = torch.Generator().manual_seed(M)
    W = (torch.randn(N, K, generator=g) * 0.02).to(torch.bfloat16).cuda()
    x = torch.randn(M, K, generator=g).to(torch.bfloat16)
    packed, params = mq.quantize_groups(W, group)
    codes, bits = gr.quantise(host(W.view(torch.int16)).view(np.uint16), group)
    status = status_word()
    y = mq.gemm_groups(packed, params, x.cuda(), out_dtype=out_dtype, dev_status=status)
    assert int(host(status)[0]) == mq.OK
    bf16 = out_dtype == torch.bfloat16
    want, tol = gr.gemm(codes, bits, x, bf16)
    _check(y, want, tol + (2.0 ** -8 * want.abs() if bf16 else 0))


@pytest.mark.parametrize("group,K", [(32, 32), (32, 96), (32, 160), (32, 4064), (64, 64), (64, 192), (64, 2368)])
def test_gemm_groups_rows_that_end_inside_a_block(group, K):
    for M in (6, 40):
        codes, params, x = _case(M, 170, K, group, K)
        _check(_run(codes, params, x), *gr.gemm(codes, params, x))


def test_gemm_groups_strides_and_nothing_to_do():
    codes, params, x = _case(60, 50, 256, 64, 1)
    wide = torch.randn(60, 256 + 40).to(torch.bfloat16)
    wide[:, 16:272] = x
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((60, 81), 9.0, device="cuda", dtype=dtype)
        mq.gemm_groups(dev(gr.pack(codes)), bf16_dev(params), wide.cuda()[:, 16:272], y=out[:, 5:55])
        want, tol = gr.gemm(codes, params, x)
        _check(out[:, 5:55], want, tol + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0))
        assert bool((out[:, :5] == 9).all()) and bool((out[:, 55:] == 9).all())
    assert mq.gemm_groups(dev(gr.pack(codes)), bf16_dev(params), x[:0].cuda()).shape == (0, 50)
    assert mq.gemm_groups(dev(gr.pack(codes[:0])), bf16_dev(params[:0]), x.cuda()).shape == (60, 0)


@pytest.mark.parametrize("exponent", [-126, -100, -40, 40, 100])
def test_gemm_groups_activations_of_any_size(exponent):
    codes, params, x = _case(40, 90, 1024, 64, 2)
    scaled = (x.double() * 2.0 ** exponent).to(torch.bfloat16)
    scaled[1] = x[1]                                             # each token has a factor of its own
    want, tol = gr.gemm(codes, params, scaled)
    _check(_run(codes, params, scaled), want, tol + 2.0 ** -149 * 1024)


def test_gemm_groups_outlier_zero_and_not_finite_tokens():
    codes, params, x = _case(50, 90, 1024, 128, 3)
    x[0] = 0
    x[1, 7] = 3e4
    x[2, 1000] = float("inf")
    x[3, 3] = float("nan")
    x[4, 5] = 3e38
    y = _run(codes, params, x).cpu()
    assert bool((y[0] == 0).all()) and not bool(torch.isfinite(y[2:4]).any())
    keep = [0, 1] + list(range(4, 50))
    _check(y[keep], *gr.gemm(codes, params, x[keep]))


def test_gemm_groups_groups_of_any_size_and_groups_that_are_not_finite():
    rng = np.random.default_rng(4)
    codes, params, x = _case(40, 150, 512, 64, 4)
    params[:, :, 0] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, (150, 8))).astype(np.float32))
    params[:, :, 1] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, (150, 8)) * rng.choice([-1, 1], (150, 8))).astype(np.float32))
    params[5, 3] = 0x7fc0
    params[7] = 0
    y = _run(codes, params, x).cpu()
    assert bool(torch.isnan(y[:, 5]).all()) and bool((y[:, 7] == 0).all())
    keep = [i for i in range(150) if i != 5]
    _check(y[:, keep], *gr.gemm(codes[keep], params[keep], x))


@pytest.mark.parametrize("M,N,K,dtype", [(40, 500, 2304, torch.float32), (300, 9000, 256, torch.bfloat16), (64, 128, 8192, torch.float32)])
def test_gemm_groups_same_bits_again_with_any_workspace_contents_on_a_stream_and_in_a_graph(M, N, K, dtype):
    W, x = bf16_dev(synth.normal_bf16((N, K), 0.02, 8)), bf16_dev(synth.normal_bf16((M, K), 1.0, 9))
    packed, params = mq.quantize_groups(W, 64)
    want = mq.gemm_groups(packed, params, x, out_dtype=dtype)
    need = mq.gemm_groups_workspace_bytes(M, N, K, 64)
    ws, y = torch.full((need,), 255, dtype=torch.uint8, device="cuda"), torch.zeros_like(want)
    mq.gemm_groups(packed, params, x, y=y, workspace=ws)
    assert torch.equal(y, want)
    with pytest.raises(mq.MatqError) as e:
        mq.gemm_groups(packed, params, x, y=y, workspace=ws[:need - 256])
    assert e.value.status == mq.ERR_WORKSPACE
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y.zero_()
        for _ in range(3):                                       # one call behind another in the same workspace
            mq.gemm_groups(packed, params, x, y=y, workspace=ws)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.gemm_groups(packed, params, x, y=y, workspace=ws)
    x2 = bf16_dev(synth.normal_bf16((M, K), 1.0, 10))
    want2 = mq.gemm_groups(packed, params, x2, out_dtype=dtype)
    x.copy_(x2)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want2)


def test_gemv_groups_of_many_tokens_is_the_same_call():
    codes, params, x = _case(48, 200, 1024, 64, 6)
    args = dev(gr.pack(codes)), bf16_dev(params), x.cuda()
    assert mq.gemm_groups_pays(48, 200, 1024, 64) and not mq.gemm_groups_pays(16, 1 << 20, 1024, 64)
    assert torch.equal(mq.gemv_groups(*args), mq.gemm_groups(*args))
    with pytest.raises(mq.MatqError) as e:
        mq.gemv_groups(*args, flags=1 << 9)
    assert e.value.status == mq.ERR_INVALID_ARG


def test_gemm_groups_stall_times_out_and_recovers():
    cases = [(40, 500, 2304, torch.float32), (300, 9000, 256, torch.bfloat16)]
    W, x = bf16_dev(synth.normal_bf16((9000, 2304), 0.02, 11)), bf16_dev(synth.normal_bf16((300, 2304), 1.0, 12))
    args = [(*mq.quantize_groups(W[:N, :K], 64), x[:M, :K], dtype) for M, N, K, dtype in cases]
    wants = [mq.gemm_groups(p, g, t, out_dtype=d) for p, g, t, d in args]
    assert mq.serving_test_stall(1) == 0
    try:
        for p, g, t, d in args:
            status = status_word()
            mq.gemm_groups(p, g, t, out_dtype=d, dev_status=status)
            assert int(host(status)[0]) == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    for (p, g, t, d), want in zip(args, wants):
        assert torch.equal(mq.gemm_groups(p, g, t, out_dtype=d), want)
