"""A product whose device-side wait gives up is reported by the decoder's step."""
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import serve
from tests.util import host, status_word

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,cache_bits", [(0, 16), (64, 4)])
def test_a_prompt_that_times_out_says_so(group, cache_bits):
    cfg = serve.Config(layers=1, group=group, cache_bits=cache_bits)
    model = serve.Decoder(cfg)
    x = torch.randn(40, cfg.hidden, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    want = model.forward(x, *_fresh(cfg))
    assert mq.serving_test_stall(1) == 0
    try:
        # each product by itself: attention over so few keys waits for nothing
        for name in ("q", "k", "v", "gate", "up"):
            status = status_word()
            serve.apply([model.layers[0][name]], x, status)
            assert int(host(status)[0]) == mq.ERR_TIMEOUT, name
        status = status_word()
        model.forward(x, *_fresh(cfg), status)
        assert int(host(status)[0]) == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    status = status_word()
    assert torch.equal(model.forward(x, *_fresh(cfg), status), want) and int(host(status)[0]) == mq.OK


def _fresh(cfg):
    cache = serve.PagedCache(cfg, 8)
    return cache, serve.Batch(cache, [("a", 40)])
