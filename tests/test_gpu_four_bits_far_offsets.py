"""Calls on 4-bit groups whose offsets pass 32 bits: what stands behind 4 GB of a matrix or a cache gives what it gives in one of its own."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests import kv4_rows_ref as rows_ref
from tests.util import dev, host, status_word

pytestmark = pytest.mark.gpu


def test_matrices():
    N, K, group, last = (1 << 21) + 777, 4096, 128, 3000
    g = torch.Generator(device="cuda").manual_seed(1)
    packed = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device="cuda")
    params = (torch.randn(N, K // group, 2, generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    assert packed.numel() > 1 << 32
    for M, call in ((2, mq.gemv_groups), (40, mq.gemm_groups)):
        x = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
        y = call(packed, params, x)[:, -last:].double()
        c = torch.stack([packed[-last:] & 15, packed[-last:] >> 4], -1).flatten(1).double().unflatten(1, (-1, group))
        s, low = (params[-last:, :, i].double().unsqueeze(-1) for i in (0, 1))
        want = x.double() @ (c * s + low).flatten(1).t()
        size = (c * s.abs() + low.abs() + 8 * s.abs()).flatten(1)
        # groups_ref.gemv's and gemm's bounds: fp32 sums rounded or cut off over 1024 columns, sums of groups in 22 bits
        assert bool(((y - want).abs() <= 2.0 ** -22 * (72 + K // group) * (x.double().abs() @ size.t())).all())
        del y, c, want, size


def test_quantised_matrices():
    N, K, group, last = (1 << 21) + 5, 4096, 64, 100           # 16 GB of weights, whose rows are 8 elements apart from one another
    W = torch.zeros(N, K + 8, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(last, K, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    W[-last:, :K] = tail.cuda()
    packed, params = mq.quantize_groups(W[:, :K], group)
    codes, bits = gr.quantise(tail.view(torch.int16).numpy().view(np.uint16), group)
    assert np.array_equal(host(packed[-last:]), gr.pack(codes)) and np.array_equal(host(params[-last:].view(torch.int16)).view(np.uint16), bits)
    assert not bool(packed[:-last].any())


@pytest.mark.parametrize("news,lens", [([1, 3], [700, 40]), ([600], [600])])
def test_caches(news, lens):
    Hq, Hkv, D, ps, T = 16, 2, 64, 256, sum(news)
    kb, vb, table = gr.make_cache(lens, Hkv, D, ps, 3)
    tiles = gr.cache_bytes(kb, vb)
    n = len(tiles)
    pages = (1 << 32) // tiles[0].size + n + 3
    cache = torch.zeros(pages, *tiles.shape[1:], dtype=torch.uint8, device="cuda")
    cache[-n:] = dev(tiles)
    far = torch.where(table >= 0, table + (pages - n), table)
    cu = [0] + [int(c) for c in np.cumsum(news)]
    args = dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32))
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    status = status_word()
    out = mq.attn_paged4(q.cuda(), cache, far.cuda(), *args, max(news), max(lens), dev_status=status)
    assert int(host(status)[0]) == mq.OK and torch.equal(out, mq.attn_paged4(q.cuda(), dev(tiles), table.cuda(), *args, max(news), max(lens)))
    rows_ref.check(out, *rows_ref.attn(q, tiles, table, cu, lens, D ** -0.5))
    kv = torch.randn(2, T, Hkv, D, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    near = dev(tiles)
    mq.kv4_append(cache, far.cuda(), *args, kv[0], kv[1], dev_status=status)
    mq.kv4_append(near, table.cuda(), *args, kv[0], kv[1])
    assert int(host(status)[0]) == mq.OK and torch.equal(cache[-n:], near) and not bool(cache[:-n].any()) and not torch.equal(near, dev(tiles))
