"""Weights in 4-bit groups: the quantiser and the product of a few tokens, against plain forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import synth
from tests import groups_ref as gr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu


def _bits(t):
    return host(t.view(torch.int16)).view(np.uint16)


# ------------------------------------------------------------------ quantize_groups

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,n", [(1, 1), (1, 3), (5, 7), (33, 18), (300, 9), (9, 112), (1001, 5)])
def test_quantize_groups_bit_exact(N, n, group):
    K = n * group
    w = synth.normal_bf16((N, K), 0.02, 100 + N + n)
    w[0, :group] = 0x3f00                                        # a constant group
    if n > 1:
        w[0, group:2 * group] = np.arange(group) % 2 * 0x8000    # zeros of both signs
    if n > 2:
        w[0, 2 * group:3 * group] = np.arange(group) % 3         # the smallest subnormals: a range that needs no codes
        w[-1, 2 * group:3 * group] = (0x3f80 + np.arange(group) * 15 // (group - 1)).astype(np.uint16)        # scale * q on many halves
        w[-1, :2] = [0x7f00, 0x0000]                             # a wide range
    status = status_word()
    packed, params = mq.quantize_groups(bf16_dev(w), group, dev_status=status)
    codes, p = gr.quantise(w, group)
    assert np.array_equal(_bits(params), p)
    assert np.array_equal(host(packed), gr.pack(codes))
    assert int(host(status)[0]) == mq.OK


def test_quantize_groups_ties():
    rng = np.random.default_rng(3)
    w = gr.bf16_bits(rng.integers(-60, 61, (400, 512)).astype(np.float32) / 8)          # ranges near 15: (x - low) / scale lands on and next to halves
    packed, params = mq.quantize_groups(bf16_dev(w), 32)
    codes, p = gr.quantise(w, 32)
    assert np.array_equal(_bits(params), p) and np.array_equal(host(packed), gr.pack(codes))


def test_quantize_groups_every_scale():
    # ranges that give every bf16 scale of many binades, and ranges next to where its rounding changes; values all over them
    rng = np.random.default_rng(8)
    scale = gr.bf16_values((np.arange(128)[None, :] + np.array([1, 10, 100, 126, 127, 128, 140, 200, 245, 250])[:, None] * 128).astype(np.uint16)).reshape(-1).astype(np.float64)
    top = np.concatenate([gr.bf16_bits((scale * f).astype(np.float32)) for f in (15.0, 15.03, 14.97, 15.06)])
    x = gr.bf16_values(top)[:, None].astype(np.float64) * rng.random((len(top), 32))
    w = gr.bf16_bits(x.astype(np.float32))
    w[:, 0], w[:, 1] = 0, top
    w[1::2] ^= 0x8000                                            # and below zero
    packed, params = mq.quantize_groups(bf16_dev(w), 32)
    codes, p = gr.quantise(w, 32)
    assert len(np.unique(p[:, 0, 0])) > 1000
    assert np.array_equal(_bits(params), p) and np.array_equal(host(packed), gr.pack(codes))


def test_quantize_groups_rows_apart_and_groups_that_are_not_finite():
    w = synth.normal_bf16((37, 320 + 24), 1.0, 5)
    status = status_word()
    W = bf16_dev(w)[:, 8:8 + 320]
    packed, params = mq.quantize_groups(W, 64, dev_status=status)
    codes, p = gr.quantise(w[:, 8:8 + 320], 64)
    assert np.array_equal(_bits(params), p) and np.array_equal(host(packed), gr.pack(codes)) and int(host(status)[0]) == mq.OK
    for bad in ([0x7f80], [0xff80], [0x7fc0], [0xffc0], [0x7f80, 0xff80], [0x7f7f, 0xff7f]):          # the last: finite, but the range is not
        x = w[:, 8:8 + 320].copy()
        x[11, 70:70 + len(bad)] = bad
        status = status_word()
        packed, params = mq.quantize_groups(bf16_dev(x), 64, dev_status=status)
        codes, p = gr.quantise(x, 64)
        assert int(host(status)[0]) == mq.ERR_NONFINITE
        assert (p[11, 1] == 0x7fc0).all() and (codes[11, 64:128] == 0).all()
        assert np.array_equal(_bits(params), p) and np.array_equal(host(packed), gr.pack(codes))


# ------------------------------------------------------------------ gemv_groups

def _case(M, N, K, group, seed, std=1.0):
    rng = np.random.default_rng(seed)
    w = gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02)
    codes, params = gr.quantise(w, group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32) * std).to(torch.bfloat16)
    return codes, params, x


def _check(y, want, tol):
    y = y.double().cpu()
    if y.dtype != want.dtype or not bool(((y - want).abs() <= tol).all()):
        raise AssertionError(float(((y - want).abs() / tol).max()))


SHAPES = [(1, 1, 128), (1, 17, 128), (2, 16, 256), (3, 100, 384), (5, 1001, 4096 - 128), (1, 2304, 9216), (7, 130, 2304), (8, 64, 1024), (9, 300, 640),
          (16, 515, 1536), (17, 48, 512), (33, 333, 896), (70, 40, 2048), (16, 300, 14336), (4, 5000, 256), (64, 20, 65536)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemv_groups(M, N, K, group, out_dtype):
    codes, params, x = _case(M, N, K, group, M + N + K)
    y = mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda(), out_dtype=out_dtype)
    want, tol = gr.gemv(codes, params, x)
    _check(y, want, tol + (2.0 ** -8 * want.abs() if out_dtype == torch.bfloat16 else 0))
    if out_dtype == torch.float32:
        assert float((y.double().cpu() - want).norm() / want.norm()) < 2e-6


@pytest.mark.parametrize("group,K", [(32, 32), (32, 96), (32, 160), (32, 4064), (64, 64), (64, 192), (64, 2368)])
def test_gemv_groups_rows_that_end_inside_a_block(group, K):
    for M in (1, 6, 20):
        codes, params, x = _case(M, 70, K, group, K)
        _check(mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda()), *gr.gemv(codes, params, x))


def test_gemv_groups_strides_and_nothing_to_do():
    codes, params, x = _case(6, 50, 256, 64, 1)
    wide = torch.randn(6, 256 + 40).to(torch.bfloat16)
    wide[:, 16:272] = x
    out = torch.full((6, 80), 9.0, device="cuda")
    mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), wide.cuda()[:, 16:272], y=out[:, 5:55])
    _check(out[:, 5:55], *gr.gemv(codes, params, x))
    assert bool((out[:, :5] == 9).all()) and bool((out[:, 55:] == 9).all())
    assert mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), x[:0].cuda()).shape == (0, 50)
    assert mq.gemv_groups(dev(gr.pack(codes[:0])), bf16_dev(params[:0]), x.cuda()).shape == (6, 0)


@pytest.mark.parametrize("exponent", [-126, -100, -40, 40, 100])
def test_gemv_groups_activations_of_any_size(exponent):
    codes, params, x = _case(3, 90, 1024, 64, 2)
    scaled = (x.double() * 2.0 ** exponent).to(torch.bfloat16)
    scaled[1] = x[1]                                             # each token has a factor of its own
    y = mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), scaled.cuda())
    want, tol = gr.gemv(codes, params, scaled)
    _check(y, want, tol + 2.0 ** -149 * 1024)                   # what falls below the smallest number


def test_gemv_groups_outlier_zero_and_not_finite_tokens():
    codes, params, x = _case(5, 90, 1024, 128, 3)
    x[0] = 0
    x[1, 7] = 3e4
    x[2, 1000] = float("inf")
    x[3, 3] = float("nan")
    y = mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda()).cpu()
    assert bool((y[0] == 0).all()) and not bool(torch.isfinite(y[2:4]).any())
    keep = [0, 1, 4]
    want, tol = gr.gemv(codes, params, x[keep])
    _check(y[keep], want, tol)


def test_gemv_groups_groups_of_any_size_and_groups_that_are_not_finite():
    rng = np.random.default_rng(4)
    codes, params, x = _case(2, 64, 512, 64, 4)
    params[:, :, 0] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, (64, 8))).astype(np.float32))
    params[:, :, 1] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, (64, 8))).astype(np.float32))
    params[5, 3] = 0x7fc0
    y = mq.gemv_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda()).cpu()
    assert bool(torch.isnan(y[:, 5]).all())
    keep = [i for i in range(64) if i != 5]
    want, tol = gr.gemv(codes[keep], params[keep], x)
    _check(y[:, keep], want, tol)


def test_gemv_groups_same_bits_again_and_behind_its_weights():
    # the call waits for its weights unless it is told that they are there
    for M in (1, 16):
        W = bf16_dev(synth.normal_bf16((700, 2304), 0.02, 6))
        x = bf16_dev(synth.normal_bf16((M, 2304), 1.0, 7))
        packed, params = mq.quantize_groups(W, 64)
        want = mq.gemv_groups(packed, params, x)
        for flags in (0, mq.GEMV_PDL):
            assert torch.equal(mq.gemv_groups(packed, params, x, flags=flags), want)
        p2, g2 = torch.zeros_like(packed), torch.zeros_like(params)
        mq.quantize_groups(W, 64, packed=p2, params=g2)
        assert torch.equal(mq.gemv_groups(p2, g2, x), want)


def test_groups_on_another_stream_and_in_a_graph():
    W, x = bf16_dev(synth.normal_bf16((300, 1024), 0.02, 8)), bf16_dev(synth.normal_bf16((4, 1024), 1.0, 9))
    want = mq.gemv_groups(*mq.quantize_groups(W, 128), x)
    packed, params, y = torch.zeros(300, 512, dtype=torch.uint8, device="cuda"), torch.zeros(300, 8, 2, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        mq.quantize_groups(W, 128, packed=packed, params=params)
        mq.gemv_groups(packed, params, x, y=y)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.quantize_groups(W, 128, packed=packed, params=params)
        mq.gemv_groups(packed, params, x, y=y, flags=0)
    x2 = bf16_dev(synth.normal_bf16((4, 1024), 1.0, 10))
    want2 = mq.gemv_groups(packed, params, x2)
    x.copy_(x2)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want2)
