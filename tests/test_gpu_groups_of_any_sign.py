"""Groups that another program wrote, whose scales are below zero where their first value is the largest: both linear layers take them alike."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(3, 300, 1024), (40, 300, 1024), (450, 4885, 640)])
def test_scales_below_zero(M, N, K, group):
    rng = np.random.default_rng(M + group)
    codes, params = gr.quantise(gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02), group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32)).to(torch.bfloat16)
    scale, low = (gr.bf16_values(params[..., i]) for i in (0, 1))
    other = params.copy()                                        # the same groups counted from their upper end, every second one
    other[:, ::2, 0] ^= 0x8000
    other[:, ::2, 1] = gr.bf16_bits((15 * scale + low)[:, ::2])
    codes = codes.reshape(N, -1, group)
    codes[:, ::2] = 15 - codes[:, ::2]
    codes = codes.reshape(N, K)
    other[0, :, 0] |= 0x8000                                     # a row whose low ends say nothing of its sizes
    other[0, :, 1] = 0
    c, s, at = torch.from_numpy(codes).double().unflatten(1, (-1, group)), *(torch.from_numpy(gr.bf16_values(other[..., i])).double().unsqueeze(-1) for i in (0, 1))
    want = x.double() @ (c * s + at).flatten(1).t()
    terms = x.double().abs() @ (c * s.abs() + at.abs() + 8 * s.abs()).flatten(1).t()
    args = dev(gr.pack(codes)), bf16_dev(other), x.cuda()
    for call in (mq.gemv_groups, mq.gemm_groups):
        for dtype in (torch.float32, torch.bfloat16):
            # groups_ref's bounds: sums rounded or cut off in 32 bits, with bf16 outputs over the whole row, and the outputs' own rounding
            steps = 72 + K // group + (K // 16 if dtype == torch.bfloat16 else 0)
            y = call(*args, out_dtype=dtype).double().cpu()
            assert bool(((y - want).abs() <= 2.0 ** -22 * steps * terms + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0)).all()), (call.__name__, dtype)
