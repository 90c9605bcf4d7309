"""The decoder example with weights in 4-bit groups and a 4-bit cache: its steps against the same steps in 64 bits, and one prompt cut in different ways."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import serve
from tests import groups_ref as gr
from tests import serving_ref as sr
from tests.util import host, status_word

pytestmark = pytest.mark.gpu


def _bf16(t):
    return t.to(torch.bfloat16).double()


def _cached(t):
    """What a 4-bit cache makes of keys or values [T, heads, D]."""
    bits = host(t.to(torch.bfloat16).contiguous().view(torch.int16)).view(np.uint16)
    c, p = gr.quantise(bits, 64)
    p = np.repeat(gr.bf16_values(p).astype(np.float64), 64, axis=-2).reshape(*bits.shape, 2)
    return torch.from_numpy(c * p[..., 0] + p[..., 1]).to(t.device)


def _weight(l):
    packed, params = host(l.packed), gr.bf16_values(host(l.params.view(torch.int16)).view(np.uint16)).astype(np.float64)
    codes = np.stack([packed & 15, packed >> 4], -1).reshape(l.N, -1, l.K // params.shape[1])
    return torch.from_numpy((codes * params[..., :1] + params[..., 1:]).reshape(l.N, l.K)).to(l.packed.device)


def _plain(model, x):
    """The whole sequence at once in 64 bits with the values that weights and cache stand for, rounded to bf16 where the decoder stores bf16."""
    cfg = model.cfg
    T, D, G = x.shape[0], cfg.head_dim, cfg.q_heads // cfg.kv_heads
    cs = model.cos_sin[:T].double()
    cos, sin = cs[:, :D // 2], cs[:, D // 2:]
    keep = torch.ones(T, T, dtype=torch.bool, device=x.device).tril()
    if cfg.window:
        keep &= ~torch.ones_like(keep).tril(-cfg.window)
    x = x.double()

    def norm(t):
        return _bf16(t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6))

    def lin(l, t):
        return _bf16(t @ _weight(l).t())
    for l in model.layers:
        h = norm(x)
        q, k, v = (lin(l[n], h).view(T, -1, D) for n in "qkv")
        q, k = _bf16(sr.rotate(q, cos, sin, False)), _cached(sr.rotate(k, cos, sin, False))
        k, v = k.repeat_interleave(G, 1), _cached(v).repeat_interleave(G, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) * D ** -0.5
        if cfg.softcap:
            s = cfg.softcap * torch.tanh(s / cfg.softcap)
        a = _bf16(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(~keep, float("-inf")), -1), v)).reshape(T, -1)
        x = _bf16(x + lin(l["o"], a))
        h = norm(x)
        x = _bf16(x + lin(l["down"], _bf16(_bf16(torch.nn.functional.silu(lin(l["gate"], h))) * lin(l["up"], h))))
    return x


@pytest.mark.parametrize("kw", [dict(group=64), dict(group=32, window=20, softcap=30.0), dict(group=128, head_dim=128, q_heads=6, kv_heads=2, hidden=768)])
def test_prompts_chunks_and_single_tokens_agree(kw):
    cfg = serve.Config(cache_bits=4, **kw)
    model = serve.Decoder(cfg, seed=3)
    T = 75
    x = torch.randn(T, cfg.hidden, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(torch.bfloat16)
    want = _plain(model, x)
    scale = want.square().mean().sqrt()
    status = status_word()
    for cuts in ([75], [40, 35], [1] * 3 + [12, 5, 50, 2, 1, 1, 1]):
        cache = serve.PagedCache(cfg, 12)
        outs, at = [], 0
        for n in cuts:
            outs.append(model.forward(x[at:at + n], cache, serve.Batch(cache, [("s", n)]), status))
            at += n
        got = torch.cat(outs).double()
        # A key or value that is rounded to bf16 the other way can meet the other code where it lies next to the border of two: a few in a hundred elements, by a
        # step of a fifteenth of their group's range (0.3 of its rms), 0.06 of the rms together.  The first outputs of a sequence average few values; what they add to
        # the residual stream is half of its rms at most.  The bf16 roundings are under 0.01.
        assert float((got - want).square().mean().sqrt() / scale) < 0.04
    assert int(status.item()) == mq.OK


def test_groups_and_a_16_bit_cache_and_the_other_way_round():
    x = torch.randn(30, 512, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
    for kw in (dict(group=64), dict(cache_bits=4)):
        model = serve.Decoder(serve.Config(**kw), seed=4)
        outs = []
        for cuts in ([30], [17, 13]):
            cache, at, status = serve.PagedCache(model.cfg, 8), 0, status_word()
            got = []
            for n in cuts:
                got.append(model.forward(x[at:at + n], cache, serve.Batch(cache, [("s", n)]), status))
                at += n
            assert int(status.item()) == mq.OK
            outs.append(torch.cat(got).double())
        assert float((outs[0] - outs[1]).square().mean().sqrt() / outs[0].square().mean().sqrt()) < 0.04


def test_sequences_of_one_batch_do_not_touch_one_another():
    cfg = serve.Config(group=64, cache_bits=4)
    model = serve.Decoder(cfg, seed=4)
    x = torch.randn(60, cfg.hidden, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
    status = status_word()
    cache = serve.PagedCache(cfg, 8)
    both = model.forward(x, cache, serve.Batch(cache, [("a", 37), ("b", 23)]), status)
    y = x.clone()
    y[37:] = torch.randn(23, cfg.hidden, device="cuda").to(torch.bfloat16)
    cache = serve.PagedCache(cfg, 8)
    other = model.forward(y, cache, serve.Batch(cache, [("a", 37), ("b", 23)]), status)
    assert torch.equal(both[:37], other[:37]) and not torch.equal(both[37:], other[37:])
    assert int(status.item()) == mq.OK


def test_cache_of_four_bits_takes_nine_thirty_seconds():
    cfg = serve.Config(cache_bits=4)
    four, sixteen = serve.PagedCache(cfg, 4), serve.PagedCache(serve.Config(), 4)
    assert 32 * four.tiles[0].numel() == 9 * (sixteen.k[0].numel() + sixteen.v[0].numel()) * 2
    with pytest.raises(ValueError):
        serve.Decoder(serve.Config(cache_bits=8))


def test_example_runs(capsys):
    serve.main(four_bits=True)
    assert capsys.readouterr().out.startswith("ok")
