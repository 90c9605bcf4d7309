"""Linear layer on weights in 4-bit groups where pairs of SMs share a tile, against plain forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu

# tiles of 160 to 256 tokens; rows and tokens that end inside a tile, a CTA whose 128 rows lie past the last; one tile a pair and several
SHAPES = [(300, 6439, 288, 32), (300, 6439, 320, 64), (130, 9547, 640, 128), (200, 9547, 544, 32), (200, 9547, 576, 64), (200, 9547, 640, 128), (513, 3849, 544, 32),
          (513, 3849, 576, 64), (513, 3849, 640, 128), (450, 4885, 544, 32), (450, 4885, 576, 64), (450, 4885, 640, 128), (1300, 9001, 640, 128), (130, 30000, 576, 64), (450, 20000, 1152, 32)]


def _case(M, N, K, group, seed):
    rng = np.random.default_rng(seed)
    codes, params = gr.quantise(gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02), group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32)).to(torch.bfloat16)
    assert mq.gemm_groups_plan(M, N, K, group, torch.bfloat16)[0]
    return codes, params, x


def _run(codes, params, x, **kw):
    status = status_word()
    y = mq.gemm_groups(dev(gr.pack(codes)), bf16_dev(params), x.cuda(), out_dtype=torch.bfloat16, dev_status=status, **kw)
    assert int(host(status)[0]) == mq.OK
    return y


def _check(y, codes, params, x):
    want, tol = gr.gemm(codes, params, x, True)
    assert bool(((y.double().cpu() - want).abs() <= tol + 2.0 ** -8 * want.abs()).all())


@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_pairs(M, N, K, group):
    codes, params, x = _case(M, N, K, group, M + N + K)
    _check(_run(codes, params, x), codes, params, x)


def test_outputs_apart_and_not_finite_tokens_and_groups():
    M, N, K, group = 450, 4885, 640, 128
    codes, params, x = _case(M, N, K, group, 1)
    x[0] = 0
    x[1, 7] = 3e4
    x[255, 600] = float("inf")
    x[449, 3] = float("nan")
    params[5, 3] = 0x7fc0
    params[4884, 0] = 0x7fc0
    params[7] = 0
    out = torch.full((M, N + 13), 9.0, device="cuda", dtype=torch.bfloat16)
    _run(codes, params, x, y=out[:, 5:5 + N])
    assert bool((out[:, :5] == 9).all()) and bool((out[:, 5 + N:] == 9).all())
    y = out[:, 5:5 + N].cpu()
    rows, tokens = [n for n in range(N) if n not in (5, 4884)], [m for m in range(M) if m not in (255, 449)]
    assert bool(torch.isnan(y[:, [5, 4884]]).all()) and not bool(torch.isfinite(y[[255, 449]]).any())
    assert bool((y[0, rows] == 0).all()) and bool((y[tokens, 7] == 0).all())
    _check(y[tokens][:, rows], codes[rows], params[rows], x[tokens])


def test_same_bits_again_in_a_graph_and_after_a_stall():
    M, N, K, group = 1300, 9001, 640, 128
    codes, params, x = _case(M, N, K, group, 2)
    args = dev(gr.pack(codes)), bf16_dev(params), x.cuda()
    want = mq.gemm_groups(*args, out_dtype=torch.bfloat16)
    ws = torch.full((mq.gemm_groups_workspace_bytes(M, N, K, group),), 255, dtype=torch.uint8, device="cuda")
    y = torch.zeros_like(want)
    for _ in range(10):
        assert torch.equal(mq.gemm_groups(*args, y=y, workspace=ws), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.gemm_groups(*args, y=y, workspace=ws)
        mq.gemm_groups(*args, y=y, workspace=ws)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    assert mq.serving_test_stall(1) == 0
    try:
        status = status_word()
        mq.gemm_groups(*args, y=y, workspace=ws, dev_status=status)
        assert int(host(status)[0]) == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    assert torch.equal(mq.gemm_groups(*args, y=y, workspace=ws), want)


@pytest.mark.parametrize("M,N,K,group", [(450, 4885, 544, 32), (200, 9547, 576, 64), (130, 9547, 640, 128)])
def test_groups_and_activations_of_any_size(M, N, K, group):
    rng = np.random.default_rng(5)
    codes, params, x = _case(M, N, K, group, 3)
    n = (N, K // group)
    params[:, :, 0] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, n)).astype(np.float32))
    params[:, :, 1] = gr.bf16_bits((2.0 ** rng.integers(-60, 60, n) * rng.choice([-1, 1], n)).astype(np.float32))
    params[7] = 0
    y = _run(codes, params, x)
    assert bool((y[:, 7] == 0).all())
    _check(y, codes, params, x)
    codes, params, x = _case(M, N, K, group, 4)
    x = (x.double() * 2.0 ** torch.from_numpy(rng.integers(-100, 100, (M, 1))).double()).to(torch.bfloat16)      # each token by its own
    _check(_run(codes, params, x), codes, params, x)
