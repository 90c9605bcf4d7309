"""The decoder example: its steps against the same steps in 64 bits, and one prompt cut in different ways."""
import threading
import time

import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import serve
from tests import serving_ref as sr
from tests.util import status_word

pytestmark = pytest.mark.gpu


def _bf16(t):
    return t.to(torch.bfloat16).double()


def _plain(model, x):
    """The whole sequence at once in 64 bits with the sliced, dequantised weights, rounded to bf16 where the decoder stores bf16; activations
    are not quantised."""
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
        return _bf16(t @ (l.alpha.double()[:, None] * (l.sliced.double() - l.zero.double()[:, None])).t())
    for l in model.layers:
        h = norm(x)
        q, k, v = (lin(l[n], h).view(T, -1, D) for n in "qkv")
        q, k = _bf16(sr.rotate(q, cos, sin, False)), _bf16(sr.rotate(k, cos, sin, False))
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) * D ** -0.5
        if cfg.softcap:
            s = cfg.softcap * torch.tanh(s / cfg.softcap)
        a = _bf16(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(~keep, float("-inf")), -1), v)).reshape(T, -1)
        x = _bf16(x + lin(l["o"], a))
        h = norm(x)
        x = _bf16(x + lin(l["down"], _bf16(_bf16(torch.nn.functional.silu(lin(l["gate"], h))) * lin(l["up"], h))))
    return x


@pytest.mark.parametrize("kw", [dict(), dict(window=20, softcap=30.0, r=8), dict(head_dim=128, q_heads=6, kv_heads=2, hidden=768, r=2)])
def test_prompts_chunks_and_single_tokens_agree(kw):
    cfg = serve.Config(**kw)
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
        # Each of the 14 products of the two layers meets activations with an error of at most half a step of 1/127 of their largest (about a third of a
        # percent of their rms for a few hundred Gaussian values): together under 2 percent of the residual stream's rms, as are the bf16 roundings.
        assert float((got - want).square().mean().sqrt() / scale) < 0.03
    assert int(status.item()) == mq.OK


def test_sequences_of_one_batch_do_not_touch_one_another():
    cfg = serve.Config()
    model = serve.Decoder(cfg, seed=4)
    x = torch.randn(60, cfg.hidden, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
    alone = []
    for lo, hi in ((0, 37), (37, 60)):
        cache = serve.PagedCache(cfg, 8)
        alone.append(model.forward(x[lo:hi], cache, serve.Batch(cache, [("s", hi - lo)])))
    cache = serve.PagedCache(cfg, 8)
    both = model.forward(x, cache, serve.Batch(cache, [("a", 37), ("b", 23)]))
    assert torch.equal(both, torch.cat(alone))
    cache.release("a")
    assert len(cache.free) == 8 - 2


def test_cache_refuses_what_does_not_fit():
    cache = serve.PagedCache(serve.Config(), 2)
    cache.extend("a", 32)
    with pytest.raises(RuntimeError):
        cache.extend("a", 1)


def test_example_runs(capsys):
    serve.main()
    assert capsys.readouterr().out.startswith("ok")


def test_other_python_threads_run_while_a_call_waits_for_the_launch_queue():
    # A launch blocks while the stream's queue is full.  The queue is filled behind a kernel that takes about 0.3 s; another thread keeps time meanwhile.
    x = torch.randn(1, 64, device="cuda").to(torch.bfloat16)
    out = mq.quantize_tokens(x)
    torch.cuda.synchronize()
    stop, ticks = threading.Event(), []

    def keep_time():
        while not stop.is_set():
            ticks.append(time.perf_counter())
            time.sleep(0.001)
    t = threading.Thread(target=keep_time)
    t.start()
    time.sleep(0.02)
    torch.cuda._sleep(500_000_000)                              # clock cycles
    begin = time.perf_counter()
    for _ in range(3000):
        mq.quantize_tokens(x, *out)
    blocked = time.perf_counter() - begin
    stop.set()
    t.join()
    torch.cuda.synchronize()
    gaps = [b - a for a, b in zip(ticks, ticks[1:]) if b >= begin]
    assert blocked > 0.1, "the queue did not fill: nothing was tested"
    assert max(gaps) < 0.5 * blocked, (blocked, max(gaps))
