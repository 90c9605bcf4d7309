"""Attention windows that no position reaches, up to the largest number, also for tokens before their sequence's start."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [1 << 31, (1 << 63) - 4, (1 << 63) - 1])
@pytest.mark.parametrize("news,lens,D", [([1, 3], [40, 300], 128), ([9, 1], [2, 70], 64), ([60, 5], [20, 0], 256), ([600, 2], [500, 9], 64), ([600], [590], 128)])
def test_the_same_bits_as_without_a_window(news, lens, D, window):
    kb, vb, table = gr.make_cache(lens, 2, D, 16, 5)
    q = torch.randn(sum(news), 16, D, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    args = (table.cuda(), dev(np.array([0] + list(np.cumsum(news)), np.int32)), dev(np.array(lens, np.int32)), max(news), max(lens))
    k, v, tiles = bf16_dev(kb), bf16_dev(vb), dev(gr.cache_bytes(kb, vb))
    for call in (lambda w, s: mq.attn_paged(q, k, v, *args, window=w, dev_status=s), lambda w, s: mq.attn_paged4(q, tiles, *args, window=w, dev_status=s)):
        status = status_word()
        out = call(window, status)
        assert int(host(status)[0]) == mq.OK
        assert torch.equal(out, call(0, None))
        assert bool((out[:max(news[0] - lens[0], 0)] == 0).all())
