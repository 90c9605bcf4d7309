"""attn_paged4 in calls that unpack: every property of the call again where keys, values and weights are fp16."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests import kv4_rows_ref as rows_ref
from tests.util import dev, host, status_word

pytestmark = pytest.mark.gpu

NAN = 0x7fc0


def _call(news, lens, Hq, Hkv, D, ps=32, seed=0, softcap=0.0, window=0, scale=None, edit=None, fill=NAN, qstd=1.5):
    """(outputs, expected, bound, status, plan); the plan unpacks."""
    T = sum(news)
    kb, vb, table = gr.make_cache(lens, Hkv, D, ps, seed, fill=fill)
    wide = (torch.randn(T + 1, Hq * D + 16, generator=torch.Generator().manual_seed(seed + 1)) * qstd).to(torch.bfloat16)
    q = wide[:, 8:8 + Hq * D].unflatten(1, (Hq, D))
    if edit is not None:
        edit(q, kb, vb, table)
    tiles, status, cu = gr.cache_bytes(kb, vb), status_word(), [0] + [int(c) for c in np.cumsum(news)]
    plan = mq.attn_paged4_plan(T + 1, len(news), Hq, Hkv, D, max(news), max(lens), window)
    assert plan[2] > 0 and (plan[0] > 0) == (len(news) > 1)
    scale = D ** -0.5 if scale is None else scale
    out = torch.full((T + 1, Hq * D + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    od = out[:, :Hq * D].unflatten(1, (Hq, D))
    mq.attn_paged4(wide.cuda()[:, 8:8 + Hq * D].unflatten(1, (Hq, D)), dev(tiles), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)), max(news), max(lens),
                   scale=scale, softcap=softcap, window=window, out=od, dev_status=status)
    assert bool((od[T:] == 9).all()) and bool((out[:, Hq * D:] == 9).all())          # what belongs to nobody is left alone
    want, tol = rows_ref.attn(q[:T], tiles, table, cu, lens, scale, softcap, window)
    return od[:T].cpu().double(), want, tol, int(host(status)[0]), plan


def _check(got, want, tol, status, plan=None):
    assert status == mq.OK
    rows_ref.check(got, want, tol)


# one query tile a CTA and two, the key range in one part and in several; alone and beside single tokens, drafts and nothing
CASES = [([600], [600], 16, 2, 64, 16), ([450], [950], 16, 2, 64, 64), ([1409], [1409], 4, 1, 64, 32), ([1000, 1, 3, 0, 40], [1000, 500, 77, 9, 333], 16, 2, 64, 32),
         ([450], [450], 16, 2, 128, 16), ([150], [2150], 16, 2, 128, 128), ([1030], [1031], 32, 4, 128, 64), ([500, 1, 2, 0, 60], [801, 300, 2, 5, 60], 16, 2, 128, 256),
         ([256], [257], 16, 2, 256, 32), ([70], [2070], 16, 2, 256, 16), ([330, 1, 1, 0, 30], [331, 200, 1, 0, 95], 16, 2, 256, 64)]


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (50.0, 0), (1000.0, 0), (0.0, 1 << 33)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_unpacked(case, softcap, window):
    _check(*_call(*CASES[case], seed=100 + case, softcap=softcap, window=window))


@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("window", [1, 37, 300])
@pytest.mark.parametrize("news,lens,Hq,Hkv,D", [([1300], [1400], 16, 2, 64), ([2500, 1, 5], [2700, 900, 600], 16, 2, 64), ([850], [2000], 16, 2, 128), ([850, 1, 40], [851, 400, 40], 16, 2, 128),
                                                ([400], [1000], 16, 2, 256), ([400, 2], [401, 900], 16, 2, 256)])
def test_windows(news, lens, Hq, Hkv, D, window, softcap):
    _check(*_call(news, lens, Hq, Hkv, D, 16, seed=7, softcap=softcap, window=window))


@pytest.mark.parametrize("news,lens,D", [([700, 1], [500, 9], 64), ([500, 3], [30, 2], 128), ([400], [390], 256), ([1500], [0], 64)])
def test_rows_without_keys_are_zero(news, lens, D):
    plan = mq.attn_paged4_plan(sum(news) + 1, len(news), 16, 2, D, max(news), max(news), 0)
    assert plan[2] > 0
    T = sum(news)
    kb, vb, table = gr.make_cache(lens, 2, D, 16, 9, fill=NAN)
    table = torch.nn.functional.pad(table, (0, 100), value=-1)
    q = torch.randn(T, 16, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    tiles, status, cu = gr.cache_bytes(kb, vb), status_word(), [0] + [int(c) for c in np.cumsum(news)]
    out = mq.attn_paged4(q.cuda(), dev(tiles), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)), max(news), max(news), dev_status=status).cpu()
    _check(out, *rows_ref.attn(q, tiles, table, cu, lens, D ** -0.5), int(host(status)[0]))
    assert bool((out[:news[0] - lens[0]] == 0).all())


@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("n,ctx,D", [(600, 21, 64), (450, 500, 64), (450, 21, 128), (160, 2000, 128), (256, 21, 256), (70, 2000, 256)])
def test_groups_of_nan_reach_only_the_rows_that_see_them(n, ctx, D, window):
    while not mq.attn_paged4_plan(n + 1, 1, 16, 2, D, n, n + ctx, window)[2]:
        n *= 2
    L, ps, at = n + ctx, 16, n // 2
    key = L - n + at

    def edit(q, kb, vb, table):
        page, slot = int(table[0, key // ps]), key % ps
        vb[page, 0, slot, D - 3] = 0x7f80
        kb[page, 1, slot, 5] = NAN
    got, want, tol, status, _ = _call([n], [L], 16, 2, D, ps, seed=10, edit=edit, window=window)
    assert status == mq.OK
    sees = torch.tensor([i >= at and (not window or i < at + window) for i in range(n)])
    near = (got - want).abs() <= tol
    assert bool(near[~sees].all()) and bool(torch.isnan(got[sees][:, :8, D - 64:]).all())
    assert bool(near[sees][:, :8, :D - 64].all()) and bool(torch.isnan(got[sees][:, 8:]).all())


@pytest.mark.parametrize("n,L,D", [(600, 600, 64), (450, 950, 64), (450, 450, 128), (160, 2160, 128), (256, 256, 256)])
def test_scores_far_apart(n, L, D):
    # one key dominates: the reference of a row's exponents moves by hundreds from step to step
    _check(*_call([n], [L], 16, 2, D, 16, seed=11, scale=1.0, qstd=8.0))

    def rising(q, kb, vb, table):                                # and once more with every step, by a few
        q[:] = 0
        q[..., 0] = 4.0
        order = np.argsort(table[0].numpy()[:-(-L // 16)])
        for i, page in enumerate(table[0].tolist()[:len(order)]):
            kb[page, :, :, :64] = 0
            kb[page, :, :, 0] = gr.bf16_bits(np.full(16, i / 2, np.float32))
    _check(*_call([n], [L], 16, 2, D, 16, seed=12, scale=1.0, edit=rising))


@pytest.mark.parametrize("exponent", [-110, -60, -20, 20, 60, 100])
@pytest.mark.parametrize("n,L,D", [(600, 600, 64), (450, 950, 64), (450, 450, 128), (256, 256, 256)])
def test_queries_keys_and_values_of_any_size(n, L, D, exponent):
    f = np.float32(2.0 ** exponent)

    def queries(q, kb, vb, table):
        q *= 2.0 ** exponent

    def keys(q, kb, vb, table):
        kb[:] = gr.bf16_bits(gr.bf16_values(kb) * f)

    def values(q, kb, vb, table):
        vb[:] = gr.bf16_bits(gr.bf16_values(vb) * f)

    def all_apart(q, kb, vb, table):                             # each head by its own
        kb[:, 0] = gr.bf16_bits(gr.bf16_values(kb[:, 0]) * f)
        vb[:, 1] = gr.bf16_bits(gr.bf16_values(vb[:, 1]) * f)
        q[:, :8] *= 2.0 ** -exponent
    for edit, by in ((queries, exponent), (keys, exponent), (values, 0), (all_apart, 0)):
        _check(*_call([n], [L], 16, 2, D, 16, seed=13, edit=edit, scale=D ** -0.5 * 2.0 ** -by))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_and_values_of_one_level(D):
    def edit(q, kb, vb, table):
        kb[:] = kb[..., :1]
        vb[:] = vb[..., :1]
    _check(*_call([600], [700], 16, 2, D, 16, seed=15, edit=edit))


# (apart: exponents of two between the first key's score and the others')
@pytest.mark.parametrize("first", [-2, 0, 14, 40])
@pytest.mark.parametrize("apart", [12, 16, 18, 20, 21])
@pytest.mark.parametrize("n,L,D", [(450, 950, 64), (1500, 1500, 64), (330, 4330, 128), (1200, 2000, 128), (700, 900, 256)])
def test_many_small_weights_beside_a_large_one(n, L, D, apart, first):
    # a first key that draws most of the weight and whose value is zero, as prompts have it: the output is what the others leave
    def edit(q, kb, vb, table):
        q[:] = 0
        q[..., 0] = 1.0
        kb[..., :64] = 0
        kb[..., 0] = gr.bf16_bits(np.float32((first - apart) * np.log(2.0)))
        page = int(table[0, 0])
        kb[page, :, 0, 0] = gr.bf16_bits(np.float32(first * np.log(2.0)))
        vb[page, :, 0] = 0
    got, want, tol, status, _ = _call([n], [L], 16, 2, D, 32, seed=16, scale=1.0, edit=edit)
    _check(got, want, tol, status)


def test_same_bits_again_on_a_stream_in_a_graph_and_with_any_workspace_contents():
    for news, lens, D in (([450], [950], 64), ([450, 1, 4], [451, 300, 80], 128), ([70], [2070], 256)):
        T, Hq, Hkv = sum(news), 16, 2
        kb, vb, table = gr.make_cache(lens, Hkv, D, 16, 30)
        cache, q = dev(gr.cache_bytes(kb, vb)), torch.randn(T, Hq, D, device="cuda").to(torch.bfloat16)
        args = (table.cuda(), dev(np.array([0] + list(np.cumsum(news)), np.int32)), dev(np.array(lens, np.int32)), max(news), max(lens))
        assert mq.attn_paged4_plan(T, len(news), Hq, Hkv, D, max(news), max(lens))[2]
        ws = torch.empty(mq.attn_paged4_workspace_bytes(T, len(news), Hq, Hkv, D, max(news), max(lens)) + 32, dtype=torch.uint8, device="cuda")
        want = mq.attn_paged4(q, cache, *args)
        out = torch.zeros_like(want)
        for byte in (0, 255, 127, 124):                          # NaN and Inf of both types among them
            ws.fill_(byte)
            assert torch.equal(mq.attn_paged4(q, cache, *args, out=out, workspace=ws[16:]), want)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(5):
                mq.attn_paged4(q, cache, *args, out=out.zero_(), workspace=ws)
        s.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mq.attn_paged4(q, cache, *args, out=out, workspace=ws)
        out.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_bad_pages_and_bounds():
    def bad(page):
        def edit(q, kb, vb, table):
            table[0, 3] = page
        return edit
    for D in (64, 128, 256):
        for page in (-1, 1 << 30):
            kb, vb, table = gr.make_cache([700, 90], 2, D, 16, 12)
            good = table.clone()
            table[0, 3] = page
            q = torch.randn(702, 16, D).to(torch.bfloat16).cuda()
            cu, lens = dev(np.array([0, 700, 702], np.int32)), dev(np.array([700, 90], np.int32))
            cache, status = dev(gr.cache_bytes(kb, vb)), status_word()
            out = mq.attn_paged4(q, cache, table.cuda(), cu, lens, 700, 700, dev_status=status)
            assert int(host(status)[0]) == mq.ERR_PAGE
            assert torch.equal(out[700:], mq.attn_paged4(q, cache, good.cuda(), cu, lens, 700, 700)[700:])           # the other sequence has what it has
