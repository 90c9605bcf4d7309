"""The paged cache in 4-bit groups: the append that fills it and the attention over it, against plain forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu

NAN = 0x7fc0


def _angles(max_pos, rot):
    half = max(rot // 2, 1)
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * f
    return torch.cat([ang.cos(), ang.sin()], 1)[:, :rot].float().contiguous()


def _rotated(x, cs, pos, rot, interleaved):
    """bf16 patterns [T, H, D] turned by their positions, every product and sum in binary32, as patterns."""
    v = gr.bf16_values(x).copy()
    half = rot // 2
    c, s = cs[pos, None, :half], cs[pos, None, half:rot]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    va, vb = v[..., a].copy(), v[..., b].copy()
    v[..., a] = (va * c).astype(np.float32) - (vb * s).astype(np.float32)
    v[..., b] = (vb * c).astype(np.float32) + (va * s).astype(np.float32)
    out = x.copy()
    out[..., :rot] = gr.bf16_bits(v)[..., :rot]
    return out


# ------------------------------------------------------------------ kv4_append

APPENDS = [([1], [0], 1, 1, 64, 16, 64), ([1, 1, 1], [5, 0, 300], 32, 8, 128, 16, 128), ([7, 0, 33, 1], [0, 9, 60, 15], 16, 8, 256, 64, 256),
           ([130], [77], 12, 4, 64, 32, 32), ([3, 2], [1, 2], 5, 1, 128, 48, 48), ([2] * 70, list(range(70)), 4, 2, 128, 16, 0), ([40, 1], [10, 3], 80, 1, 256, 128, 96),
           ([1500, 600], [3, 0], 3, 1, 64, 16, 64), ([2100], [0], 2, 1, 128, 64, 128), ([2000, 49], [7, 1], 3, 2, 256, 32, 256)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("news,ctxs,Hq,Hkv,D,ps,rot", APPENDS)
def test_kv4_append(news, ctxs, Hq, Hkv, D, ps, rot, interleaved):
    T, extra = sum(news), 2                                     # rows that belong to no sequence
    lens = [n + c for n, c in zip(news, ctxs)]
    kb, vb, table = gr.make_cache(lens, Hkv, D, ps, 3)
    tiles = gr.cache_bytes(kb, vb)
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    rng = np.random.default_rng(T)
    qkv = gr.bf16_bits(rng.standard_normal((T + extra, (Hq + 2 * Hkv) * D + 8), dtype=np.float32))
    part = lambda t, lo, n: t[:, lo * D:(lo + n) * D].unflatten(1, (n, D))            # noqa: E731
    wide = bf16_dev(qkv)
    q, k, v = part(wide, 0, Hq), part(wide, Hq, Hkv), part(wide, Hq + Hkv, Hkv)
    cs = _angles(max(lens) + 1, rot) if rot else None
    args = (table.cuda(), dev(cu), dev(np.array(lens, np.int32)))
    cache, status = dev(tiles), status_word()
    q_out = torch.full((T + extra, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda")
    mq.kv4_append(cache, *args, k, v, cos_sin=None if cs is None else cs.cuda(), q=q, q_out=q_out, interleaved=interleaved, dev_status=status)
    assert int(host(status)[0]) == mq.OK
    pos = np.concatenate([np.arange(c, c + n) for n, c in zip(news, ctxs)])
    seq = np.repeat(np.arange(len(news)), news)
    page, slot = table.numpy()[seq, pos // ps], pos % ps
    rows = qkv[:T, :(Hq + 2 * Hkv) * D].reshape(T, -1, D)
    turned = _rotated(rows[:, :Hq + Hkv], cs.numpy(), pos, rot, interleaved) if rot else rows[:, :Hq + Hkv]
    assert np.array_equal(host(q_out.view(torch.int16)).view(np.uint16)[:T], turned[:, :Hq]) and bool((q_out[T:] == 3).all())
    kb[page, :, slot], vb[page, :, slot] = turned[:, Hq:], rows[:, Hq + Hkv:]
    assert np.array_equal(host(cache), gr.cache_bytes(kb, vb))
    # in place, and without queries
    again, qi = dev(tiles), part(wide.clone(), 0, Hq)
    mq.kv4_append(again, *args, k, v, cos_sin=None if cs is None else cs.cuda(), q=qi, q_out=qi, interleaved=interleaved)
    assert torch.equal(qi[:T], q_out[:T]) and torch.equal(again, cache)
    again = dev(tiles)
    mq.kv4_append(again, *args, k, v, cos_sin=None if cs is None else cs.cuda(), interleaved=interleaved)
    assert torch.equal(again, cache)


def test_kv4_append_bytes_of_a_tile():
    # the layout, one element at a time
    D = 128
    rng = np.random.default_rng(1)
    k = gr.bf16_bits(rng.standard_normal((16, 1, D), dtype=np.float32))
    v = gr.bf16_bits(rng.standard_normal((16, 1, D), dtype=np.float32))
    cache = torch.zeros(1, 1, 1, mq.kv4_tile_bytes(D), dtype=torch.uint8, device="cuda")
    mq.kv4_append(cache, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), dev(np.array([0, 16], np.int32)), dev(np.array([16], np.int32)), bf16_dev(k), bf16_dev(v))
    want = np.concatenate([gr.tile_half(*gr.quantise(t[:, 0], 64)) for t in (k, v)])
    assert np.array_equal(host(cache).reshape(-1), want)


def test_kv4_append_groups_that_are_not_finite():
    D = 128
    for bad in (0x7f80, 0xff80, NAN):
        k = gr.bf16_bits(np.random.default_rng(2).standard_normal((3, 2, D), dtype=np.float32))
        v = k.copy()
        v[1, 1, 70] = bad
        cache, status = torch.zeros(1, 2, 1, 18 * D, dtype=torch.uint8, device="cuda"), status_word()
        mq.kv4_append(cache, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), dev(np.array([0, 3], np.int32)), dev(np.array([3], np.int32)), bf16_dev(k), bf16_dev(v),
                      dev_status=status)
        assert int(host(status)[0]) == mq.ERR_NONFINITE
        kb, vb = np.zeros((1, 2, 16, D), np.uint16), np.zeros((1, 2, 16, D), np.uint16)
        kb[0, :, :3], vb[0, :, :3] = k.transpose(1, 0, 2), v.transpose(1, 0, 2)
        assert np.array_equal(host(cache), gr.cache_bytes(kb, vb))


def test_kv4_append_data_errors():
    Hkv, D, ps = 2, 64, 16
    kb, vb, table = gr.make_cache([20, 20], Hkv, D, ps, 4)
    tiles = gr.cache_bytes(kb, vb)
    k = torch.ones(2, Hkv, D, dtype=torch.bfloat16, device="cuda")
    cu = dev(np.array([0, 1, 2], np.int32))
    cs = _angles(20, 64).cuda()

    def run(table, lens, cs=cs):
        cache, status = dev(tiles), status_word()
        q = torch.full((2, 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
        mq.kv4_append(cache, table.cuda(), cu, dev(np.array(lens, np.int32)), k, k, cos_sin=cs, q=q, q_out=q, dev_status=status)
        changed = (host(cache) != tiles).reshape(len(tiles), -1).any(1).sum()
        return int(host(status)[0]), int(changed), bool((q[0] == 7).all())
    assert run(table, [20, 20])[:2] == (mq.OK, 2)
    bad = table.clone(); bad[0, 1] = -1
    assert run(bad, [20, 20]) == (mq.ERR_PAGE, 1, True)
    bad[0, 1] = len(tiles)
    assert run(bad, [20, 20]) == (mq.ERR_PAGE, 1, True)
    assert run(table, [0, 20]) == (mq.ERR_PAGE, 1, True)                          # a position below zero
    assert run(table, [table.shape[1] * ps + 1, 20], cs=_angles(400, 64).cuda()) == (mq.ERR_PAGE, 1, True)      # past the page table
    assert run(table, [20, 20], cs=_angles(19, 64).cuda()) == (mq.ERR_PAGE, 0, True)     # past the rotation table


# ------------------------------------------------------------------ attn_paged4

def _attend(news, lens, Hq, Hkv, D, ps, seed, softcap=0.0, window=0, fill=None, edit=None, hints=None, scale=None, qstd=1.5, qmul=1.0):
    T = sum(news)
    kb, vb, table = gr.make_cache(lens, Hkv, D, ps, seed, fill=fill)
    cu = [0] + list(np.cumsum(news))
    g = torch.Generator().manual_seed(seed + 1)
    wide = (torch.randn(T + 1, Hq * D + 16, generator=g) * qstd * qmul).to(torch.bfloat16)
    q = wide[:, 8:8 + Hq * D].unflatten(1, (Hq, D))
    if edit is not None:
        edit(kb, vb, table, q)
    tiles, status = gr.cache_bytes(kb, vb), status_word()
    out = torch.full((T + 1, Hq * D + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    mx = hints or (max(news + [1]), max(lens + [1]))
    qd = wide.cuda()[:, 8:8 + Hq * D].unflatten(1, (Hq, D))
    od = out[:, :Hq * D].unflatten(1, (Hq, D))
    scale = D ** -0.5 / qmul if scale is None else scale
    mq.attn_paged4(qd, dev(tiles), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)), mx[0], mx[1], scale=scale,
                   softcap=softcap, window=window, out=od, dev_status=status)
    got = od.cpu().double()
    assert bool((got[T:] == 9).all()) and bool((out[:, Hq * D:] == 9).all())         # what belongs to nobody is left alone
    want, tol = gr.attn(q[:T], tiles, table, cu, lens, scale, softcap, window, min(mx[0], T))
    return got[:T], want, tol, int(host(status)[0])


def _check(got, want, tol, status):
    assert status == mq.OK
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


CASES = [
    # new tokens, keys in all, q heads, kv heads, D, page
    ([1], [1], 1, 1, 64, 16), ([1], [2], 4, 2, 128, 16), ([1, 1, 1], [63, 64, 65], 8, 8, 128, 16), ([1], [1000], 32, 8, 128, 16),
    ([1, 1], [129, 700], 16, 8, 256, 32), ([1] * 5, [5, 17, 128, 300, 1], 12, 4, 64, 64), ([1, 1], [257, 90], 64, 1, 128, 128), ([1], [513], 6, 2, 256, 256),
    ([3, 5, 1], [3, 200, 77], 8, 2, 128, 16), ([6], [900], 16, 8, 256, 16), ([17], [17], 3, 1, 64, 16), ([2, 0, 4], [50, 31, 4], 10, 2, 128, 32),
    ([33], [100], 4, 4, 128, 16), ([16, 1, 9], [300, 40, 9], 4, 2, 64, 256), ([5, 12], [205, 412], 5, 1, 256, 128),
    # unpacked: alone, and beside single tokens and drafts
    ([40, 1, 70], [40, 500, 333], 8, 2, 128, 64), ([130], [130], 2, 1, 256, 64), ([129], [700], 5, 1, 128, 128),
    ([260], [261], 4, 2, 64, 256), ([150, 20], [150, 410], 16, 8, 256, 16), ([100, 1, 1, 4, 0, 5], [355, 1, 600, 77, 30, 5], 24, 8, 128, 16), ([300, 128], [300, 512], 2, 2, 128, 32),
    ([70, 2, 1], [70, 300, 257], 14, 2, 64, 32), ([513], [513], 3, 1, 128, 16), ([1, 90], [1000, 900], 4, 1, 128, 16),
]


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (50.0, 0), (0.0, 37), (20.0, 130)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attn_paged4(case, softcap, window):
    # stale slots hold groups of NaN: whatever is not a key of the sequence must not matter
    _check(*_attend(*CASES[case], seed=100 + case, softcap=softcap, window=window, fill=NAN))


@pytest.mark.parametrize("case", [2, 3, 8, 11, 13, 14, 15, 20, 23])
def test_attn_paged4_generous_bounds_change_little(case):
    news, lens = CASES[case][:2]
    for hints in ((max(news), 1 << 20), (max(news), 5000), (1 << 40, 1 << 40) if max(news) < 10 else (max(news), 70000)):
        _check(*_attend(*CASES[case], seed=200 + case, hints=hints, window=300))
        if hints[1] < 1 << 20:
            _check(*_attend(*CASES[case], seed=200 + case, hints=hints))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_paged4_chunks_with_bounds_that_say_nothing(D):
    # more keys than could be unpacked: rows by the hundred read the cache as it is
    _check(*_attend([200, 1, 30], [500, 40, 333], 8, 2, D, 32, seed=300, hints=(200, (1 << 31) - 1)))


def test_attn_paged4_fewer_tokens_than_rows_and_bounds():
    # rows behind the last sequence, as in a padded batch whose call was made for more tokens
    for lens in ([300], [300, 50]):
        kb, vb, table = gr.make_cache(lens, 2, 128, 16, 17)
        tiles, status = gr.cache_bytes(kb, vb), status_word()
        q = torch.randn(100, 8, 128).to(torch.bfloat16)
        cu = [0, 2, 3][:len(lens) + 1]
        out = torch.full((100, 8, 128), 9.0, dtype=torch.bfloat16, device="cuda")
        mq.attn_paged4(q.cuda(), dev(tiles), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)), 100, 4000, out=out, dev_status=status)
        want, tol = gr.attn(q[:cu[-1]], tiles, table, cu, lens, 128 ** -0.5, longest=100)
        _check(out[:cu[-1]].double().cpu(), want, tol, int(host(status)[0]))
        assert bool((out[cu[-1]:] == 9).all())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_attn_paged4_long_cache_is_split(D, ps):
    _check(*_attend([1, 2], [6001, 3000], 8, 4, D, ps, seed=6))
    _check(*_attend([1], [5000], 8, 4, D, ps, seed=7, window=1000))
    _check(*_attend([30], [2000], 8, 2, D, ps, seed=8))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_paged4_chunks_and_single_tokens_over_a_window(D):
    _check(*_attend([60, 1, 3], [2000, 1700, 900], 8, 2, D, 16, seed=21, window=500))
    _check(*_attend([60, 1, 3], [2000, 1700, 900], 8, 2, D, 64, seed=22, window=260, softcap=30.0))


def test_attn_paged4_rows_without_keys_are_zero():
    # more new tokens than keys: the first ones stand before the sequence's start
    for D in (64, 128, 256):
        for n, L in ((5, 3), (40, 30), (200, 70), (4, 0)):
            got, want, tol, status = _attend([n, 1], [L, 9], 4, 2, D, 16, seed=9)
            _check(got, want, tol, status)
            assert bool((got[:n - L] == 0).all())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [4, 30, 60, 200])
def test_attn_paged4_nonfinite_groups_reach_only_the_rows_that_see_them(D, n):
    # token n // 2 of the chunk has a value group of NaN for key head 0; its key is NaN for head 1 only
    L, ps, at = n + 21, 16, n // 2
    key = L - n + at

    def edit(kb, vb, table, q):
        page, slot = int(table[0, key // ps]), key % ps
        vb[page, 0, slot, D - 3] = 0x7f80
        kb[page, 1, slot, 5] = NAN
    for window in (0, 5):
        got, want, tol, status = _attend([n], [L], 4, 2, D, ps, seed=10, edit=edit, window=window)
        assert status == mq.OK
        sees = [i for i in range(n) if i >= at and (not window or i < at + window)]
        blind = [i for i in range(n) if i not in sees]
        assert bool(((got - want).abs() <= tol)[blind].all())
        assert bool(torch.isnan(got[sees][:, :2, D - 64:]).all())
        assert bool(((got - want).abs() <= tol)[sees][:, :2, :D - 64].all())
        assert bool(torch.isnan(got[sees][:, 2:]).all())


def test_attn_paged4_large_scores():
    # one key dominates: the running maximum moves by hundreds from tile to tile
    for D in (64, 128, 256):
        for n in (1, 15, 50, 150):
            _check(*_attend([n], [700], 4, 2, D, 16, seed=11, scale=1.0, qstd=8.0))


@pytest.mark.parametrize("exponent", [-110, -60, 60, 100, 120])
def test_attn_paged4_queries_of_any_size(exponent):
    for D in (64, 128, 256):
        for n in (1, 6):
            _check(*_attend([n], [300], 4, 2, D, 16, seed=12, qmul=2.0 ** exponent))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_paged4_groups_of_any_size(D):
    # values far from one, and keys whose queries make up for it
    for exponent in (-80, -30, 30, 80):
        def edit(kb, vb, table, q):
            vb[:] = gr.bf16_bits(gr.bf16_values(vb) * np.float32(2.0 ** exponent))
        _check(*_attend([3], [500], 4, 2, D, 16, seed=13, edit=edit))
    for exponent in (-80, 80):
        def edit(kb, vb, table, q):
            kb[:] = gr.bf16_bits(gr.bf16_values(kb) * np.float32(2.0 ** exponent))
        _check(*_attend([3], [500], 4, 2, D, 16, seed=14, edit=edit, scale=D ** -0.5 * 2.0 ** -exponent))


def test_attn_paged4_values_and_keys_of_one_level():
    # constant groups: a scale of zero
    def edit(kb, vb, table, q):
        kb[:] = kb[..., :1]
        vb[:] = vb[..., :1]
    for n in (2, 80):
        _check(*_attend([n], [200], 4, 2, 128, 16, seed=15, edit=edit))


def _status(news, lens, Hq, Hkv, D, ps, edit=None, lens_dev=None, cu_dev=None, hints=None):
    T = sum(news)
    kb, vb, table = gr.make_cache(lens, Hkv, D, ps, 12)
    q = torch.randn(T, Hq, D).to(torch.bfloat16)
    if edit:
        edit(table)
    status = status_word()
    cu = cu_dev or [0] + list(np.cumsum(news))
    hints = hints or (max(news), max(lens))
    out = mq.attn_paged4(q.cuda(), dev(gr.cache_bytes(kb, vb)), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens_dev or lens, np.int32)), *hints, dev_status=status)
    return out, int(host(status)[0])


def test_attn_paged4_data_errors():
    for D, n in ((128, 1), (128, 20), (128, 100), (256, 3), (256, 90)):
        def no_page(table):
            table[0, 1] = -1

        def far_page(table):
            table[0, 1] = 1 << 30
        assert _status([n], [n + 40], 4, 2, D, 16, no_page)[1] == mq.ERR_PAGE
        assert _status([n], [n + 40], 4, 2, D, 16, far_page)[1] == mq.ERR_PAGE
        assert _status([n], [n + 40], 4, 2, D, 16, lens_dev=[1 << 30])[1] == mq.ERR_PAGE
        assert _status([n], [n + 40], 4, 2, D, 16, cu_dev=[0, n + 5])[1] == mq.ERR_PAGE
        assert _status([n], [n + 40], 4, 2, D, 16)[1] == mq.OK
    # more keys than the call was told of
    assert _status([1500], [3000], 16, 2, 128, 16, hints=(1500, 1600))[1] == mq.ERR_PAGE


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 3, 60, 300])
@pytest.mark.parametrize("length", [-1, -(1 << 31)])
def test_attn_paged4_lengths_below_zero_see_nothing(D, n, length):
    out, status = _status([n, 1], [200, 9], 4, 2, D, 16, lens_dev=[length, 9])
    assert status == mq.OK and bool((out[:n] == 0).all()) and bool((out[n:] != 0).any())


def test_attn_paged4_stall_times_out_and_recovers():
    # only the kernels that take unpacked keys and values wait for anything
    assert mq.serving_test_stall(1) == 0
    try:
        for n, D in ((1, 64), (4, 128), (3, 256)):
            _check(*_attend([n], [n + 300], 4, 2, D, 16, seed=16))
        for D in (64, 128, 256):
            assert _status([1500], [3000], 16, 2, D, 16)[1] == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    for n, D in ((1, 64), (1, 128), (4, 128), (3, 256), (100, 128)):
        _check(*_attend([n], [n + 300], 4, 2, D, 16, seed=16))


def test_kv4_calls_on_another_stream_and_in_a_graph():
    Hq, Hkv, D, ps, L = 8, 2, 128, 16, 200
    for n in (1, 40):
        kb, vb, table = gr.make_cache([L], Hkv, D, ps, 30)
        tiles = gr.cache_bytes(kb, vb)
        args = (table.cuda(), dev(np.array([0, n], np.int32)), dev(np.array([L], np.int32)))
        g = torch.Generator().manual_seed(31)
        qkv = torch.randn(n, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16).cuda()
        cs = _angles(L, D).cuda()

        def step(cache, qkv, q_out, out, ws):
            mq.kv4_append(cache, *args, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], cos_sin=cs, q=qkv[:, :Hq], q_out=q_out)
            mq.attn_paged4(q_out, cache, *args, n, L, out=out, workspace=ws)
        ws = torch.empty(max(16, mq.attn_paged4_workspace_bytes(n, 1, Hq, Hkv, D, n, L)), dtype=torch.uint8, device="cuda")
        q_out, out = (torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = dev(tiles)
        step(cache, qkv, q_out, out, ws)
        want, want_cache = out.clone(), cache.clone()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        cache = dev(tiles)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            step(cache, qkv, q_out, out.zero_(), ws)
        s.synchronize()
        assert torch.equal(out, want) and torch.equal(cache, want_cache)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(cache, qkv, q_out, out, ws)
        cache.copy_(dev(tiles))
        out.zero_()
        ws.fill_(255)                                           # nothing is kept in a workspace from call to call
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache, want_cache)


def test_attn_paged4_same_bits_again_and_with_any_workspace_contents():
    for news, lens in (([1], [5000]), ([3, 1], [900, 2000]), ([100, 1], [400, 3000])):
        T = sum(news)
        kb, vb, table = gr.make_cache(lens, 2, 128, 16, 40)
        cache, q = dev(gr.cache_bytes(kb, vb)), torch.randn(T, 8, 128, device="cuda").to(torch.bfloat16)
        args = (table.cuda(), dev(np.array([0] + list(np.cumsum(news)), np.int32)), dev(np.array(lens, np.int32)), max(news), max(lens))
        need = mq.attn_paged4_workspace_bytes(T, len(news), 8, 2, 128, max(news), max(lens))
        outs = []
        for byte in (0, 255, 127):
            ws = torch.full((need + 32,), byte, dtype=torch.uint8, device="cuda")
            outs.append(mq.attn_paged4(q, cache, *args, workspace=ws[16:]))
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        if need:
            with pytest.raises(mq.MatqError) as e:
                mq.attn_paged4(q, cache, *args, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
            assert e.value.status == mq.ERR_WORKSPACE


def test_attn_paged4_more_sequences_than_are_unpacked_together():
    # 40 chunks, told that each may have 65536 keys of 4 heads of 256 elements: 512 MB of unpacked keys and values serve a few of them at a time
    news = [40 + i % 7 for i in range(12)] + [1] * 3
    lens = [60 + 31 * i for i in range(15)]
    _check(*_attend(news, lens, 8, 4, 256, 16, seed=50, hints=(46, 40000)))


def test_append_and_attend_as_a_decoder_does():
    """A prompt, a chunk, drafts and single tokens of two sequences go into the cache and attend to it; errors against attention over the values that were appended
    come from four bits alone."""
    Hq, Hkv, D, ps = 8, 2, 64, 32
    table = torch.arange(2 * 16, dtype=torch.int32).view(2, 16).flip(1).contiguous()
    cache = torch.zeros(32, Hkv, ps // 16, mq.kv4_tile_bytes(D), dtype=torch.uint8, device="cuda")
    cs, status = _angles(400, D).cuda(), status_word()
    lens = [0, 0]
    g = torch.Generator(device="cuda").manual_seed(60)
    for news in ([100, 37], [1, 1], [1, 60], [3, 2], [1, 1], [0, 1]):
        T = sum(news)
        lens = [a + b for a, b in zip(lens, news)]
        qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device="cuda").to(torch.bfloat16)
        cu = [0, news[0], T]
        args = (table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)))
        q = mq.kv4_append(cache, *args, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], cos_sin=cs, q=qkv[:, :Hq], dev_status=status)
        out = mq.attn_paged4(q, cache, *args, max(news), max(lens), dev_status=status)
        want, tol = gr.attn(q, host(cache), table, cu, lens, D ** -0.5, longest=max(news))
        _check(out.double().cpu(), want, tol, int(host(status)[0]))
