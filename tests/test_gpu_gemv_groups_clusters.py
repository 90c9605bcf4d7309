"""gemv_groups where the CTAs of a cluster share K and walk several row steps, against plain forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev

pytestmark = pytest.mark.gpu

# parts of K of one length and of two; 2, 4 and 8 CTAs
SHAPES = [(25, 4832, 3712, 32), (25, 4832, 3840, 32), (17, 6400, 3712, 32), (25, 2768, 7296, 32), (25, 1392, 14464, 32), (25, 4832, 5120, 64), (25, 2768, 10496, 64),
          (25, 2768, 13568, 64), (25, 4832, 5504, 128), (25, 2768, 10880, 128), (25, 2768, 13952, 128)]


def _gemv(packed, params, x, dtype=torch.float32):
    y = torch.full((x.shape[0], packed.shape[0]), float("nan"), dtype=dtype, device="cuda")
    assert mq._serving.gemv_groups(packed, params, x, y, 0) == mq.OK              # never the call for many tokens
    return y


@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_several_steps_of_a_cluster(M, N, K, group):
    rng = np.random.default_rng(N + K)
    codes, params = gr.quantise(gr.bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * 0.02), group)
    x = torch.from_numpy(rng.standard_normal((M, K), dtype=np.float32)).to(torch.bfloat16)
    packed, groups = dev(gr.pack(codes)), bf16_dev(params)
    _, parts, steps = mq.gemv_groups_plan(M, N, K, group)
    assert parts > 1 and steps >= 3
    y = _gemv(packed, groups, x.cuda())
    want, tol = gr.gemv(codes, params, x)
    assert bool(((y.double().cpu() - want).abs() <= tol).all())
    for _ in range(20):
        assert torch.equal(_gemv(packed, groups, x.cuda()), y)


@pytest.mark.parametrize("M,N,K,group", [(16, 65536, 11008, 32), (16, 28672, 8192, 128), (8, 128256, 4096, 64), (16, 256000, 3584, 64)])
def test_matrices_of_an_output_heads_size(M, N, K, group):
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    packed = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device="cuda")
    params = (torch.randn(N, K // group, 2, generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    _, parts, steps = mq.gemv_groups_plan(M, N, K, group)
    assert parts > 1 and steps >= 3
    y = _gemv(packed, params, x)
    # 64 bits, a few thousand rows at a time; the bound is groups_ref.gemv's
    for lo in range(0, N, 4096):
        c = torch.stack([packed[lo:lo + 4096] & 15, packed[lo:lo + 4096] >> 4], -1).flatten(1).double().unflatten(1, (-1, group))
        s, low = (params[lo:lo + 4096, :, i].double().unsqueeze(-1) for i in (0, 1))
        want = x.double() @ (c * s + low).flatten(1).t()
        size = (c * s.abs() + low.abs()).flatten(1)
        tol = 2.0 ** -23 * (48 + K // group) * (x.double().abs() @ size.t())
        assert bool(((y[:, lo:lo + 4096].double() - want).abs() <= tol).all()), lo
    for _ in range(10):
        assert torch.equal(_gemv(packed, params, x), y)
