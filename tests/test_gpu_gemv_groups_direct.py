"""The call for few tokens on 4-bit groups at sizes that the Python call hands to the one for many: each block of tokens, every width of columns, the longest rows."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev

pytestmark = pytest.mark.gpu

SHAPES = [(17, 512, 14336), (18, 40, 256), (24, 1000, 2304), (32, 333, 4096), (33, 333, 896), (40, 2304, 2304), (64, 130, 1152), (64, 20, 65536), (70, 40, 2048), (257, 64, 640),
          (2000, 100, 256), (1, 700, 65536), (9, 300, 65536)]


def _gemv(packed, params, x, dtype):
    y = torch.full((x.shape[0], packed.shape[0]), float("nan"), dtype=dtype, device="cuda")
    assert mq._serving.gemv_groups(packed, params, x, y, 0) == mq.OK
    return y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_every_number_of_tokens(M, N, K, group):
    rng = np.random.default_rng(M + N + K)
    codes, params = gr.quantise(gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02), group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32)).to(torch.bfloat16)
    x[-1] *= 2.0 ** 60                                           # past what tokens are first scaled by
    args = dev(gr.pack(codes)), bf16_dev(params), x.cuda()
    want, tol = gr.gemv(codes, params, x)
    y = _gemv(*args, torch.float32)
    assert bool(((y.double().cpu() - want).abs() <= tol).all())
    half = _gemv(*args, torch.bfloat16)
    assert bool(((half.double().cpu() - want).abs() <= tol + 2.0 ** -8 * want.abs()).all())
    assert torch.equal(_gemv(*args, torch.float32), y)


def test_blocks_of_one_two_and_four_times_eight_tokens_are_reached():
    tokens = {mq.gemv_groups_plan(M, N, K, group)[0] for M, N, K in SHAPES for group in (32, 64, 128)}
    assert min(tokens) <= 8 and any(8 < t <= 16 for t in tokens) and max(tokens) > 16
