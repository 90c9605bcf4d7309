"""Token quantisation, the 8-bit linear layer, the paged append and the attention over the paged cache against plain 64-bit forms."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import synth
from tests import serving_ref as sr
from tests.util import bf16_dev, dev, host, status_word

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ quantize_tokens

@pytest.mark.parametrize("M,K", [(1, 16), (1, 2304), (3, 2048), (5, 2064), (37, 4096), (2, 9216), (4, 16384), (2, 16400), (2, 65536), (300, 736)])
def test_quantize_tokens_bit_exact(M, K):
    x = synth.normal_bf16((M, K), 1.0, 7000 + M + K)
    x[0, 0] = 0x42fe                                            # 127.0: scale 1, and the row's codes include exact halves
    x[0, 1:9] = [0x3f00, 0xbf00, 0x3fc0, 0xbfc0, 0x4020, 0x4060, 0x0001, 0x8001]     # +-0.5, +-1.5, 2.5, 3.5, the smallest subnormals
    if M > 1:
        x[1, :] = 0                                             # nothing to scale
    if M > 2:
        x[2, :] = 0x0001                                        # the smallest subnormal everywhere: the scale is held at 2^-126
    status = status_word()
    xq, s, r = mq.quantize_tokens(bf16_dev(x), dev_status=status)
    xq_r, s_r, r_r = sr.quantize_tokens(x)
    assert np.array_equal(host(s), s_r)
    assert np.array_equal(host(xq), xq_r)
    assert np.array_equal(host(r), r_r)
    assert int(host(status)[0]) == mq.OK


def test_quantize_tokens_ties_everywhere():
    # every row has a maximum that makes the quotients of many others land on or next to a half
    M, K = 256, 512
    rng = np.random.default_rng(11)
    x = synth.normal_bf16((M, K), 3.0, 12)
    x[:, 0] = rng.integers(0x3f80, 0x4380, M).astype(np.uint16)
    xq, s, r = mq.quantize_tokens(bf16_dev(x))
    xq_r, s_r, r_r = sr.quantize_tokens(x)
    assert np.array_equal(host(xq), xq_r) and np.array_equal(host(s), s_r) and np.array_equal(host(r), r_r)


def test_quantize_tokens_strides_and_nonfinite_rows():
    M, K = 6, 1040
    x = synth.normal_bf16((M, K + 24), 1.0, 13)
    X = bf16_dev(x)[:, 8:8 + K]
    xq = torch.full((M, K + 16), 99, dtype=torch.int8, device="cuda")
    _, s, r = mq.quantize_tokens(X, xq=xq[:, :K])
    xq_r, s_r, r_r = sr.quantize_tokens(x[:, 8:8 + K])
    assert np.array_equal(host(xq)[:, :K], xq_r) and np.array_equal(host(s), s_r) and (host(xq)[:, K:] == 99).all()
    for bad in (0x7f80, 0xff80, 0x7fc0):                         # +Inf, -Inf, NaN
        y = x[:, 8:8 + K].copy()
        y[3, K - 1] = bad
        status = status_word()
        xq, s, r = mq.quantize_tokens(bf16_dev(y), dev_status=status)
        assert int(host(status)[0]) == mq.ERR_NONFINITE
        keep = [0, 1, 2, 4, 5]
        assert np.array_equal(host(xq)[keep], xq_r[keep]) and np.array_equal(host(s)[keep], s_r[keep])
        assert np.isnan(host(s)[3]) and (host(xq)[3] == 0).all() and int(host(r)[3]) == 0


# ------------------------------------------------------------------ gemm_a8

def _linear(M, N, K, seed, full_range=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if full_range:                                               # the largest sums there are
        xq = torch.full((M, K), -127, dtype=torch.int8, device="cuda")
        q = torch.full((N, K), 255, dtype=torch.uint8, device="cuda")
    else:
        xq = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
        q = torch.randint(0, 256, (N, K), generator=g, device="cuda").to(torch.uint8)
    scale = torch.rand(M, generator=g, device="cuda") * 0.05 + 1e-3
    alpha = torch.rand(N, generator=g, device="cuda") * 1e-3 + 1e-4
    zero = torch.randn(N, generator=g, device="cuda") * 20 + 128
    return xq, scale, xq.int().sum(1).int(), q, alpha, zero


SHAPES = [(1, 1, 16), (1, 9216, 2304), (2, 130, 144), (7, 127, 128), (16, 129, 4096), (17, 2304, 9216), (33, 1000, 272), (64, 640, 1024),
          (65, 257, 3584), (100, 100, 2000), (128, 128, 128), (129, 300, 528), (255, 513, 640), (256, 256, 256), (257, 1025, 1152), (300, 2311, 736),
          (509, 3584, 2304), (700, 4096, 4096), (1025, 1537, 2064), (2048, 640, 144), (3, 5, 65536)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_a8(M, N, K, out_dtype):
    xq, s, r, q, a, z = _linear(M, N, K, M * 31 + N * 7 + K)
    status = status_word()
    y = mq.gemm_a8(xq, s, r, q, a, z, out_dtype=out_dtype, dev_status=status)
    want, tol = sr.gemm_a8(xq, s, q, a, z, out_dtype)
    assert bool(((y.double() - want).abs() <= tol).all())
    assert int(host(status)[0]) == mq.OK
    again = mq.gemm_a8(xq, s, r, q, a, z, out_dtype=out_dtype, flags=mq.GEMV_PDL)
    assert torch.equal(y, again)


@pytest.mark.parametrize("M,N,K", [(5, 40, 65536), (300, 300, 65536)])
def test_gemm_a8_largest_sums(M, N, K):
    xq, s, r, q, a, z = _linear(M, N, K, 5, full_range=True)
    y = mq.gemm_a8(xq, s, r, q, a, z)
    want, tol = sr.gemm_a8(xq, s, q, a, z, torch.float32)
    assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M", [3, 70, 600])
def test_gemm_a8_strides_nan_rows_and_empty(M):
    N, K = 333, 400
    xq, s, r, q, a, z = _linear(M, N, K, 77)
    xw = torch.zeros(M, K + 48, dtype=torch.int8, device="cuda"); xw[:, 16:16 + K] = xq
    qw = torch.zeros(N, K + 32, dtype=torch.uint8, device="cuda"); qw[:, :K] = q
    yw = torch.full((M, N + 3), 5.0, device="cuda")
    s = s.clone(); s[1] = float("nan")
    y = mq.gemm_a8(xw[:, 16:16 + K], s, r, qw[:, :K], a, z, y=yw[:, 1:1 + N])
    want, tol = sr.gemm_a8(xq, s, q, a, z, torch.float32)
    keep = [i for i in range(M) if i != 1]
    assert bool(((y.double() - want).abs() <= tol)[keep].all()) and bool(torch.isnan(y[1]).all())
    assert bool((yw[:, 0] == 5).all()) and bool((yw[:, N + 1:] == 5).all())
    assert mq.gemm_a8(xq[:0], s[:0], r[:0], q, a, z).shape == (0, N)
    assert mq.gemm_a8(xq, s, r, q[:0], a[:0], z[:0]).shape == (M, 0)


def test_linear_from_weights_to_outputs():
    # quantize -> slice -> quantize_tokens -> gemm_a8 at a nested precision, against 64 bits with the quantised operands
    M, N, K = 45, 384, 1024
    W = bf16_dev(synth.normal_bf16((N, K), 0.02, 31))
    x = synth.normal_bf16((M, K), 1.0, 32)
    q, a, z = mq.quantize(W)
    xq_r, s_r, _ = sr.quantize_tokens(x)
    xq, s, r = mq.quantize_tokens(bf16_dev(x))
    for rr in (8, 4, 2, 3):
        sl = q if rr == 8 else mq.slice_pack(q, rr, want_packed=False, want_unpacked=True)["sliced"]
        y = mq.gemm_a8(xq, s, r, sl, a, z)
        want, tol = sr.gemm_a8(dev(xq_r), dev(s_r), sl, a, z, torch.float32)
        assert bool(((y.double() - want).abs() <= tol).all())


# ------------------------------------------------------------------ kv_append

def _angles(max_pos, rot):
    half = max(rot // 2, 1)
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * f
    return torch.cat([ang.cos(), ang.sin()], 1)[:, :rot].float().contiguous()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("news,ctxs,Hq,Hkv,D,ps,rot", [
    ([1], [0], 1, 1, 64, 16, 64), ([1, 1, 1], [5, 0, 300], 32, 8, 128, 16, 128), ([7, 0, 33, 1], [0, 9, 60, 15], 16, 8, 256, 64, 256),
    ([130], [77], 12, 4, 64, 32, 32), ([3, 2], [1, 2], 5, 1, 24, 7, 16), ([2] * 70, list(range(70)), 4, 2, 128, 16, 0), ([40, 1], [10, 3], 6, 3, 80, 1, 80)])
def test_kv_append(news, ctxs, Hq, Hkv, D, ps, rot, interleaved):
    T = sum(news)
    lens = [n + c for n, c in zip(news, ctxs)]
    kc, vc, table = sr.make_cache(lens, Hkv, D, ps, 3)
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    g = torch.Generator().manual_seed(T)
    extra = 2                                                   # rows that belong to no sequence
    qkv = torch.randn(T + extra, (Hq + 2 * Hkv) * D + 8, generator=g).to(torch.bfloat16).cuda()
    q = qkv[:, :Hq * D].unflatten(1, (Hq, D)); k = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    v = qkv[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(1, (Hkv, D))
    cs = _angles(max(lens) + 1, rot) if rot else None
    kd, vd = kc.cuda(), vc.cuda()
    q_out = torch.full((T + extra, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda")
    status = status_word()
    mq.kv_append(kd, vd, table.cuda(), dev(cu), dev(np.array(lens, np.int32)), k, v, cos_sin=None if cs is None else cs.cuda(), q=q, q_out=q_out,
                 interleaved=interleaved, dev_status=status)
    assert int(host(status)[0]) == mq.OK
    pos = torch.cat([torch.arange(c, c + n) for n, c in zip(news, ctxs)])
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(news)]).long()
    page, slot = table[seq, pos // ps].long(), pos % ps

    def rotated(x):
        x = x[:T].cpu().double()
        if not rot:
            return x, torch.zeros_like(x)
        c, s = cs[pos, :rot // 2].double(), cs[pos, rot // 2:].double()
        y = sr.rotate(x, c, s, interleaved)
        size = torch.zeros_like(x)
        size[..., :rot] = x[..., :rot].abs().amax(-1, keepdim=True)
        return y, 2.0 ** -8 * y.abs() + 2.0 ** -22 * size       # rounding to 8 bits, two products and a sum in 32
    want, tol = rotated(q)
    assert bool(((q_out[:T].cpu().double() - want).abs() <= tol).all())
    assert bool((q_out[:T, :, rot:] == q[:T, :, rot:]).all()) and bool((q_out[T:] == 3).all())
    want, tol = rotated(k)
    got = kd.cpu()[page, :, slot]
    assert bool(((got.double() - want).abs() <= tol).all())
    assert torch.equal(vd.cpu()[page, :, slot], v[:T].cpu())
    # nothing else in the cache has changed
    kc[page, :, slot] = got; vc[page, :, slot] = v[:T].cpu()
    assert torch.equal(kd.cpu(), kc) and torch.equal(vd.cpu(), vc)
    # in place, and without queries
    k2, v2 = kc.cuda(), vc.cuda()
    qi = qkv.clone()[:, :Hq * D].unflatten(1, (Hq, D))
    mq.kv_append(k2, v2, table.cuda(), dev(cu), dev(np.array(lens, np.int32)), k, v, cos_sin=None if cs is None else cs.cuda(), q=qi, q_out=qi,
                 interleaved=interleaved)
    assert torch.equal(qi[:T], q_out[:T]) and torch.equal(k2, kd)
    k3, v3 = kc.cuda(), vc.cuda()
    mq.kv_append(k3, v3, table.cuda(), dev(cu), dev(np.array(lens, np.int32)), k, v, cos_sin=None if cs is None else cs.cuda(), interleaved=interleaved)
    assert torch.equal(k3, kd) and torch.equal(v3, vd)


def test_kv_append_data_errors():
    Hkv, D, ps = 2, 64, 16
    kc, vc, table = sr.make_cache([20, 20], Hkv, D, ps, 4)
    k = torch.ones(2, Hkv, D, dtype=torch.bfloat16, device="cuda")
    cu = dev(np.array([0, 1, 2], np.int32))
    cs = _angles(20, 64).cuda()

    def run(table, lens, cs=cs):
        kd, vd, status = kc.cuda(), vc.cuda(), status_word()
        q = torch.full((2, 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
        mq.kv_append(kd, vd, table.cuda(), cu, dev(np.array(lens, np.int32)), k, k, cos_sin=cs, q=q, q_out=q, dev_status=status)
        changed = (vd.cpu() != vc).flatten(1).any(1).sum()
        return int(host(status)[0]), int(changed), bool((q[0] == 7).all())
    assert run(table, [20, 20])[:2] == (mq.OK, 2)
    bad = table.clone(); bad[0, 1] = -1
    assert run(bad, [20, 20]) == (mq.ERR_PAGE, 1, True)
    bad[0, 1] = kc.shape[0]
    assert run(bad, [20, 20]) == (mq.ERR_PAGE, 1, True)
    assert run(table, [0, 20]) == (mq.ERR_PAGE, 1, True)                          # a position below zero
    assert run(table, [table.shape[1] * ps + 1, 20], cs=_angles(400, 64).cuda()) == (mq.ERR_PAGE, 1, True)      # past the page table
    assert run(table, [20, 20], cs=_angles(19, 64).cuda()) == (mq.ERR_PAGE, 0, True)     # past the rotation table


# ------------------------------------------------------------------ attn_paged

def _attend(news, lens, Hq, Hkv, D, ps, seed, softcap=0.0, window=0, fill=None, edit=None, hints=None, scale=None, qstd=1.5):
    T = sum(news)
    kc, vc, table = sr.make_cache(lens, Hkv, D, ps, seed, fill=fill)
    cu = [0] + list(np.cumsum(news))
    g = torch.Generator().manual_seed(seed + 1)
    wide = (torch.randn(T + 1, Hq * D + 16, generator=g) * qstd).to(torch.bfloat16)
    q = wide[:, 8:8 + Hq * D].unflatten(1, (Hq, D))
    if edit is not None:
        edit(kc, vc, table, q)
    status = status_word()
    out = torch.full((T + 1, Hq * D + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    mx = hints or (max(news + [1]), max(lens + [1]))
    qd = wide.cuda()[:, 8:8 + Hq * D].unflatten(1, (Hq, D))
    od = out[:, :Hq * D].unflatten(1, (Hq, D))
    scale = D ** -0.5 if scale is None else scale
    mq.attn_paged(qd, kc.cuda(), vc.cuda(), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens, np.int32)), mx[0], mx[1], scale=scale,
                  softcap=softcap, window=window, out=od, dev_status=status)
    got = od.cpu().double()
    assert bool((got[T:] == 9).all()) and bool((out[:, Hq * D:] == 9).all())         # what belongs to nobody is left alone
    want, tol = sr.attn(q[:T], kc, vc, table, cu, lens, scale, softcap, window)
    return got[:T], want, tol, int(host(status)[0])


def _check(got, want, tol, status):
    assert status == mq.OK
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


CASES = [
    # new tokens, keys in all, q heads, kv heads, D, page
    ([1], [1], 1, 1, 64, 16), ([1], [2], 4, 2, 128, 16), ([1, 1, 1], [63, 64, 65], 8, 8, 128, 16), ([1], [1000], 32, 8, 128, 16),
    ([1, 1], [129, 700], 16, 8, 256, 32), ([1] * 5, [5, 17, 128, 300, 1], 12, 4, 64, 64), ([1, 1], [257, 90], 64, 1, 128, 128), ([1], [513], 6, 2, 256, 256),
    ([3, 5, 1], [3, 200, 77], 8, 2, 128, 16), ([6], [900], 16, 8, 256, 16), ([17], [17], 3, 1, 64, 16), ([2, 0, 4], [50, 31, 4], 10, 2, 128, 32),
    ([33], [100], 4, 4, 128, 16), ([40, 1, 70], [40, 500, 333], 8, 2, 128, 64), ([130], [130], 2, 1, 256, 64), ([129], [700], 5, 1, 128, 128),
    ([260], [261], 4, 2, 64, 256), ([150, 20], [150, 410], 16, 8, 256, 16), ([100], [355], 24, 8, 128, 16), ([300, 128], [300, 512], 2, 2, 128, 32),
    ([70], [70], 14, 2, 64, 32), ([513], [513], 3, 1, 128, 16),
]


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (50.0, 0), (0.0, 37), (20.0, 130)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attn_paged(case, softcap, window):
    # stale slots hold NaN: whatever is not a key of the sequence must not matter
    _check(*_attend(*CASES[case], seed=100 + case, softcap=softcap, window=window, fill=float("nan")))


MANY = [
    # enough query tiles to fill the GPU: the kernels of 128 rows, one tile per CTA and two
    ([140] * 20, [140 + 17 * i for i in range(20)], 8, 2, 128, 16), ([140] * 20, [400 - 13 * i for i in range(20)], 8, 2, 64, 64),
    ([40] * 20 + [3, 0, 1], [40 + 9 * i for i in range(20)] + [3, 0, 200], 8, 2, 64, 32), ([60] * 30, [60 + 5 * i for i in range(30)], 4, 2, 128, 128),
    ([33] * 30, [33 + 11 * i for i in range(30)], 4, 2, 256, 64),
]


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (50.0, 0), (0.0, 37), (20.0, 130)])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_attn_paged_many_query_tiles(case, softcap, window):
    _check(*_attend(*MANY[case], seed=300 + case, softcap=softcap, window=window, fill=float("nan")))


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (20.0, 130)])
@pytest.mark.parametrize("case", [i for i, c in enumerate(CASES) if max(c[0]) * c[2] // c[3] > 16])
def test_attn_paged_tiles_of_128_rows(case, softcap, window):
    # the hint of a long range: query tiles of 128 rows, and parts that hold no key
    _check(*_attend(*CASES[case], seed=400 + case, softcap=softcap, window=window, fill=float("nan"), hints=(max(CASES[case][0]), 1 << 20)))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_paged_nonfinite_values_in_tiles_of_128_rows(D):
    def edit(kc, vc, table, q):
        vc[table[0, 60 // 16], :, 60 % 16, D // 2] = float("inf")             # keys that rows from 60 - 20 = 40 on see
        vc[table[0, 90 // 16], 1, 90 % 16, 3] = float("nan")
    got, want, tol, status = _attend([80], [100], 8, 2, D, 16, seed=410, edit=edit, hints=(80, 1 << 20))
    assert status == mq.OK
    bad = ~torch.isfinite(want)
    assert bool(bad[40:].any()) and not bool(bad[:40].any())
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert bool((got[~bad] - want[~bad]).abs().le(tol[~bad]).all())


@pytest.mark.parametrize("hints", [(1, 1), (1, 100000), (5000, 1), (64, 64)])
def test_attn_paged_hints_change_no_result(hints):
    _check(*_attend([40, 1, 9], [300, 700, 9], 8, 2, 128, 16, seed=5, hints=hints))


@pytest.mark.parametrize("hints", [(1 << 62, 1 << 62), (1, (1 << 63) - 1)])
@pytest.mark.parametrize("window", [(1 << 63) - 1, 1 << 31])
def test_attn_paged_hints_and_windows_of_any_size(hints, window):
    _check(*_attend([40, 1, 9], [300, 700, 9], 8, 2, 128, 16, seed=9, hints=hints, window=window))
    _check(*_attend([1, 2], [300, 31], 8, 2, 64, 16, seed=10, hints=hints, window=window))


def test_serving_views_of_one_row_may_have_any_stride():
    x = torch.randn(3, 67, device="cuda", dtype=torch.float32).to(torch.bfloat16)[:1, :64]
    xq, scale, rowsum = mq.quantize_tokens(x)
    wq, ws, wr = mq.quantize_tokens(x.contiguous())
    assert torch.equal(xq, wq) and torch.equal(scale, ws) and torch.equal(rowsum, wr)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_paged_long_cache_is_split(D):
    _check(*_attend([1, 2], [6001, 3000], 8, 4, D, 16, seed=6))
    _check(*_attend([1], [5000], 8, 4, D, 16, seed=7, window=1000))
    _check(*_attend([30], [4000], 8, 2, D, 64, seed=8))


def test_attn_paged_rows_without_keys_are_zero():
    # more new tokens than keys: the first ones stand before the sequence's start
    for D in (64, 128, 256):
        for n, L in ((5, 3), (40, 30), (200, 70), (4, 0)):
            got, want, tol, status = _attend([n, 1], [L, 9], 4, 2, D, 16, seed=9)
            _check(got, want, tol, status)
            assert bool((got[:n - L] == 0).all())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [4, 60, 200])
def test_attn_paged_nonfinite_values_reach_only_the_rows_that_see_them(D, n):
    # token n // 2 of the chunk has a NaN in one value element and an Inf in another; its key is NaN for head 1 only
    L, ps, at = n + 21, 16, n // 2
    key = L - n + at

    def edit(kc, vc, table, q):
        page, slot = int(table[0, key // ps]), key % ps
        vc[page, 0, slot, 3] = float("nan")
        vc[page, 0, slot, D - 1] = float("inf")
        kc[page, 1, slot, 5] = float("nan")
    for window in (0, 5):
        got, want, tol, status = _attend([n], [L], 4, 2, D, ps, seed=10, edit=edit, window=window)
        assert status == mq.OK
        sees = [i for i in range(n) if i >= at and (not window or i < at + window)]
        for h in range(4):
            for i in range(n):
                if i not in sees:
                    assert bool(((got[i, h] - want[i, h]).abs() <= tol[i, h]).all()), (h, i)
        assert bool(torch.isnan(got[sees, :2, 3]).all()) and bool((got[sees, :2, D - 1] == float("inf")).all())
        others = [d for d in range(D) if d not in (3, D - 1)]
        assert bool(((got - want).abs() <= tol)[sees][:, :2][:, :, others].all())
        assert bool(torch.isnan(got[sees, 2:]).all())


def test_attn_paged_large_scores():
    # one key dominates: the running maximum moves by hundreds from tile to tile
    for D in (64, 128, 256):
        for n in (1, 50, 150):
            _check(*_attend([n], [900], 4, 2, D, 16, seed=11, scale=1.0, qstd=8.0))


def test_attn_paged_data_errors():
    for D, n in ((128, 1), (128, 100), (256, 3)):
        def no_page(kc, vc, table, q):
            table[0, 1] = -1
        *_, status = _attend_status([n], [n + 40], 4, 2, D, 16, no_page)
        assert status == mq.ERR_PAGE

        def far_page(kc, vc, table, q):
            table[0, 1] = 1 << 30
        *_, status = _attend_status([n], [n + 40], 4, 2, D, 16, far_page)
        assert status == mq.ERR_PAGE
        *_, status = _attend_status([n], [n + 40], 4, 2, D, 16, None, lens_dev=[1 << 30])
        assert status == mq.ERR_PAGE
        *_, status = _attend_status([n], [n + 40], 4, 2, D, 16, None, cu_dev=[0, n + 5])
        assert status == mq.ERR_PAGE


def _attend_status(news, lens, Hq, Hkv, D, ps, edit, lens_dev=None, cu_dev=None):
    T = sum(news)
    kc, vc, table = sr.make_cache(lens, Hkv, D, ps, 12)
    q = torch.randn(T, Hq, D).to(torch.bfloat16)
    if edit:
        edit(kc, vc, table, q)
    status = status_word()
    cu = cu_dev or [0] + list(np.cumsum(news))
    out = mq.attn_paged(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array(lens_dev or lens, np.int32)), max(news),
                        max(lens), dev_status=status)
    return out, int(host(status)[0])


# ------------------------------------------------------------------ error path of the waits, streams, graphs

def test_serving_test_stall_times_out_and_recovers():
    xq, s, r, q, a, z = _linear(100, 300, 512, 3)
    xl, sl, rl, ql, al, zl = _linear(600, 600, 512, 4)
    few = _linear(7, 300, 512, 3)                               # up to 8 tokens there is no device-side wait
    assert mq.serving_test_stall(1) == 0
    try:
        status = status_word()
        want, tol = sr.gemm_a8(few[0], few[1], few[3], few[4], few[5], torch.float32)
        assert bool(((mq.gemm_a8(*few, dev_status=status).double() - want).abs() <= tol).all()) and int(host(status)[0]) == mq.OK
        for args in ((xq, s, r, q, a, z), (xl, sl, rl, ql, al, zl)):
            status = status_word()
            y = torch.full((args[0].shape[0], args[3].shape[0]), 5.0, device="cuda")
            mq.gemm_a8(*args, y=y, dev_status=status)
            assert int(host(status)[0]) == mq.ERR_TIMEOUT and bool((y == 5).all())
        for D, n in ((64, 1), (128, 1), (256, 2), (128, 100), (256, 100)):
            _, status = _attend_status([n], [n + 300], 4, 2, D, 16, None)
            assert status == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    for args in ((xq, s, r, q, a, z), (xl, sl, rl, ql, al, zl)):
        want, tol = sr.gemm_a8(args[0], args[1], args[3], args[4], args[5], torch.float32)
        assert bool(((mq.gemm_a8(*args).double() - want).abs() <= tol).all())
    for D, n in ((64, 1), (128, 1), (256, 2), (128, 100), (256, 100)):
        _check(*_attend([n], [n + 300], 4, 2, D, 16, seed=13))


@pytest.mark.parametrize("D,news", [(64, [140] * 20), (128, [140] * 20), (128, [60] * 30), (256, [60] * 20)])
def test_attn_paged_many_query_tiles_large_scores_errors_and_stall(D, news):
    lens = [n + 30 + 19 * i for i, n in enumerate(news)]
    _check(*_attend(news, lens, 8, 2, D, 16, seed=14, scale=1.0, qstd=8.0))

    def no_page(kc, vc, table, q):
        table[3, 1] = -1
    assert _attend_status(news, lens, 8, 2, D, 16, no_page)[1] == mq.ERR_PAGE
    assert mq.serving_test_stall(1) == 0
    try:
        assert _attend_status(news, lens, 8, 2, D, 16, None)[1] == mq.ERR_TIMEOUT
    finally:
        assert mq.serving_test_stall(0) == 1
    _check(*_attend(news, lens, 8, 2, D, 16, seed=15))


def test_serving_calls_on_another_stream_and_in_a_graph():
    xq, s, r, q, a, z = _linear(300, 300, 512, 3)
    y0 = mq.gemm_a8(xq, s, r, q, a, z)
    kc, vc, table = sr.make_cache([300, 40], 2, 128, 16, 14)
    kc, vc, table = kc.cuda(), vc.cuda(), table.cuda()
    qq = torch.randn(41, 8, 128, device="cuda").to(torch.bfloat16)
    cu, lens = dev(np.array([0, 1, 41], np.int32)), dev(np.array([300, 40], np.int32))
    ws = torch.empty(mq.attn_paged_workspace_bytes(41, 2, 8, 2, 128, 40, 300) + 16, dtype=torch.uint8, device="cuda")
    o0 = mq.attn_paged(qq, kc, vc, table, cu, lens, 40, 300)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y1, o1 = torch.empty_like(y0), torch.empty_like(o0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        mq.gemm_a8(xq, s, r, q, a, z, y=y1)
        mq.attn_paged(qq, kc, vc, table, cu, lens, 40, 300, out=o1, workspace=ws)
        side.synchronize()
        assert torch.equal(y0, y1) and torch.equal(o0, o1)
        with torch.cuda.graph(graph, stream=side):
            mq.gemm_a8(xq, s, r, q, a, z, y=y1)
            mq.attn_paged(qq, kc, vc, table, cu, lens, 40, 300, out=o1, workspace=ws)
        y1.zero_(); o1.zero_()
        graph.replay()
        side.synchronize()
    assert torch.equal(y0, y1) and torch.equal(o0, o1)


# ------------------------------------------------------------------ workspaces, marginal sizes and values

@pytest.mark.parametrize("D,n,L,hint", [(64, 100, 1100, 1 << 20), (128, 100, 1100, 1 << 20), (256, 40, 900, 900), (128, 1, 5000, 5000), (64, 300, 2800, 2800)])
def test_attn_paged_workspace_of_any_16_byte_alignment(D, n, L, hint):
    # parts of the key range go through the workspace, which may start at any multiple of 16 bytes (the hint of a long range: query tiles of 128 rows)
    Hq, Hkv, ps = 8, 2, 16
    kc, vc, table = sr.make_cache([L], Hkv, D, ps, 21)
    q = (torch.randn(n, Hq, D, generator=torch.Generator().manual_seed(22)) * 1.5).to(torch.bfloat16)
    want, tol = sr.attn(q, kc, vc, table, [0, n], [L], D ** -0.5)
    need = mq.attn_paged_workspace_bytes(n, 1, Hq, Hkv, D, n, hint)
    assert need > 0
    ws = torch.empty(need + 48, dtype=torch.uint8, device="cuda")
    outs = []
    for at in (0, 16, 48):
        status = status_word()
        o = mq.attn_paged(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), dev(np.array([0, n], np.int32)), dev(np.array([L], np.int32)), n, hint,
                          workspace=ws[at:at + need], dev_status=status)
        assert int(host(status)[0]) == mq.OK
        assert bool(((o.cpu().double() - want).abs() <= tol).all())
        outs.append(o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_gemm_a8_more_tokens_than_any_grid_of_small_tiles_holds():
    M, N, K = 128 * 65535 + 130, 16, 16
    xq, s, r, q, a, z = _linear(M, N, K, 91)
    status = status_word()
    y = mq.gemm_a8(xq, s, r, q, a, z, dev_status=status)
    assert int(host(status)[0]) == mq.OK
    for lo in range(0, M, 1 << 21):
        hi = min(M, lo + (1 << 21))
        want, tol = sr.gemm_a8(xq[lo:hi], s[lo:hi], q, a, z, torch.float32)
        assert bool(((y[lo:hi].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M", [1, 5, 64, 400])
def test_weights_written_two_calls_before_a_call_that_fetches_them_early(M):
    # slice_pack writes W2, a call that fetches W1 early follows, then one that fetches W2 early: its predecessor writes no weights
    N, K, n_small = 4096, 4096, 64
    g = torch.Generator(device="cuda").manual_seed(33)
    codes = [torch.randint(0, 256, (N, K), generator=g, device="cuda").to(torch.uint8) for _ in range(4)]
    xq, s, r, q1, a1, z1 = _linear(M, n_small, K, 34)
    a2, z2 = torch.rand(N, generator=g, device="cuda") + 0.5, torch.full((N,), 128.0, device="cuda")
    x = torch.randn(K, generator=g, device="cuda").to(torch.bfloat16)
    small = mq.slice_pack(q1, 4, want_unpacked=True)
    sliced, packed = torch.empty_like(codes[0]), torch.empty((N, K // 2), dtype=torch.uint8, device="cuda")
    ys, vs = [], []
    for c in codes * 3:
        mq.slice_pack(c, 4, packed=packed, sliced_unpacked=sliced)
        mq.gemm_a8(xq, s, r, small["sliced"], a1, z1, flags=mq.GEMV_PDL)
        ys.append(mq.gemm_a8(xq, s, r, sliced, a2, z2, flags=mq.GEMV_PDL))
        mq.slice_pack(c, 4, packed=packed, sliced_unpacked=sliced)
        mq.gemv(small["packed"], K, 4, a1, z1, x[None], flags=mq.GEMV_PDL)
        vs.append(mq.gemv(packed, K, 4, a2, z2, x[None], flags=mq.GEMV_PDL))
    for i, c in enumerate(codes * 3):
        out = mq.slice_pack(c, 4, want_unpacked=True)
        torch.cuda.synchronize()
        assert torch.equal(ys[i], mq.gemm_a8(xq, s, r, out["sliced"], a2, z2))
        assert torch.equal(vs[i], mq.gemv(out["packed"], K, 4, a2, z2, x[None]))


def _sign_scores(D, n, L, exponent, step=None, seed=51):
    """Queries and keys of +-2^a: every product q . k is an integer times 2^exponent, exact in 32 bits, so that two scores are equal or far apart.
    Before position ``step`` the keys are 2^-exponent times as large."""
    a = exponent // 2

    def edit(kc, vc, table, q):
        g = torch.Generator().manual_seed(seed)
        q.copy_(torch.randint(0, 2, q.shape, generator=g).to(torch.bfloat16) * 2 - 1)
        q.mul_(2.0 ** a)
        kc.copy_(torch.randint(0, 2, kc.shape, generator=g).to(torch.bfloat16) * 2 - 1)
        kc.mul_(2.0 ** a)
        if step is not None:
            for j in range(step):
                kc[table[0, j // kc.shape[2]], :, j % kc.shape[2]] *= 2.0 ** -(2 * a)
    return edit


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,L,hint", [(1, 700, 700), (4, 700, 700), (60, 500, 1 << 20), (140, 900, 1 << 20), (140, 300, 300)])
@pytest.mark.parametrize("exponent", [4, 16, 24, 30, 34, 40, 60, 100])
def test_attn_paged_scores_of_any_finite_size(D, n, L, hint, exponent):
    # one key (or several of one score) takes all the weight, however far the scores lie from zero, and whichever kernel and split does it
    for step in (None, 200):
        _check(*_attend([n], [L], 4, 2, D, 16, seed=52, scale=1.0, hints=(n, hint), edit=_sign_scores(D, n, L, exponent, step)))


@pytest.mark.parametrize("D,news", [(64, [140] * 20), (128, [140] * 20), (256, [60] * 20)])
@pytest.mark.parametrize("exponent", [24, 34, 60])
def test_attn_paged_many_query_tiles_scores_of_any_finite_size(D, news, exponent):
    lens = [n + 30 + 19 * i for i, n in enumerate(news)]
    _check(*_attend(news, lens, 8, 2, D, 16, seed=53, scale=1.0, edit=_sign_scores(D, news, lens, exponent)))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,L,hint", [(4, 700, 700), (60, 500, 1 << 20), (140, 900, 1 << 20), (140, 300, 300)])
@pytest.mark.parametrize("exponent", [30, 60])
def test_attn_paged_rows_with_large_and_with_ordinary_scores(D, n, L, hint, exponent):
    # heads of one token, and neighbouring tokens, share a tile: every second row's scores are ordinary ones
    signs = _sign_scores(D, n, L, exponent, 200)

    def edit(kc, vc, table, q):
        signs(kc, vc, table, q)
        q.flatten(0, 1)[::2].mul_(2.0 ** -(exponent + 3))
        q[1::3].mul_(2.0 ** -(exponent // 2))
    _check(*_attend([n], [L], 4, 2, D, 16, seed=54, scale=1.0, hints=(n, hint), edit=edit))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,L,hint", [(1, 60, 60), (4, 700, 700), (60, 300, 1 << 20), (140, 300, 300)])
@pytest.mark.parametrize("cap", [0.5, 30.0, 300.0, 1e4, 1e5, 1e6, 1e8, 1e20, 3e38, float("inf")])
def test_attn_paged_cap_of_any_size(D, n, L, hint, cap):
    # a cap far above the scores leaves them as they are, to the precision of 32 bits: its tanh has to keep a relative accuracy
    got, want, tol, status = _attend([n], [L], 4, 2, D, 16, seed=61, softcap=cap, hints=(n, hint), qstd=6.0)
    if cap > 1e19:
        got0, want, tol, _ = _attend([n], [L], 4, 2, D, 16, seed=61, hints=(n, hint), qstd=6.0)      # in 64 bits s / cap vanishes, or is NaN times infinity
    _check(got, want, tol, status)


@pytest.mark.parametrize("D,news", [(64, [140] * 20), (128, [140] * 20), (256, [60] * 20)])
@pytest.mark.parametrize("cap", [100.0, 1e5, 1e7])
def test_attn_paged_many_query_tiles_cap_of_any_size(D, news, cap):
    lens = [n + 30 + 19 * i for i, n in enumerate(news)]
    _check(*_attend(news, lens, 8, 2, D, 16, seed=62, softcap=cap, qstd=6.0))
    _check(*_attend(news, lens, 8, 2, D, 16, seed=63, softcap=cap, qstd=600.0))           # scores past the cap, and up to a few hundred


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,hint", [(1, 200), (3, 200), (60, 200), (60, 1 << 20), (300, 200)])
@pytest.mark.parametrize("length", [-1, -5, -(1 << 31) + 400, -(1 << 31)])
def test_attn_paged_lengths_below_zero_see_nothing(D, n, hint, length):
    # as for padding: a sequence's length may be anything below its number of new tokens
    news, lens = [n, n], [200 + n, 40 + n]
    kc, vc, table = sr.make_cache(lens, 2, D, 16, 71)
    q = torch.randn(2 * n, 4, D, generator=torch.Generator().manual_seed(72)).to(torch.bfloat16)
    want, tol = sr.attn(q, kc, vc, table, [0, n, 2 * n], [0, lens[1]], D ** -0.5)
    status = status_word()
    out = mq.attn_paged(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), dev(np.array([0, n, 2 * n], np.int32)), dev(np.array([length, lens[1]], np.int32)), n, hint,
                        dev_status=status)
    assert int(host(status)[0]) == mq.OK and bool((out[:n] == 0).all())
    assert bool(((out.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("news,lens", [([300, 2], [300, 700]), ([400], [150]), ([257, 300], [900, 299])])
def test_attn_paged_one_cta_walks_tiles_with_and_without_keys(D, news, lens):
    # hints of one new token: a CTA takes all tiles of a sequence, and a part of the key range lies past the first ones (or they see no key at all)
    for hint in (100000, 2000):
        _check(*_attend(news, lens, 8, 2, D, 16, seed=81, hints=(1, hint), fill=float("nan")))
        _check(*_attend(news, lens, 8, 2, D, 16, seed=82, hints=(4, hint), window=70, fill=float("nan")))


def test_attn_paged_workspaces_that_do_not_fit_are_refused():
    kc, vc, table = sr.make_cache([5000], 2, 64, 16, 91)
    q = torch.randn(1, 4, 64).to(torch.bfloat16).cuda()
    args = (q, kc.cuda(), vc.cuda(), table.cuda(), dev(np.array([0, 1], np.int32)), dev(np.array([5000], np.int32)), 1, 5000)
    need = mq.attn_paged_workspace_bytes(1, 1, 4, 2, 64, 1, 5000)
    assert need > 0
    for bad, error in ((torch.empty(need, dtype=torch.uint8), TypeError), (np.empty(need, np.uint8), TypeError), (torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2], TypeError)):
        with pytest.raises(error, match="workspace"):
            mq.attn_paged(*args, workspace=bad)
    for size, start, status in ((need - 1, 0, mq.ERR_WORKSPACE), (need, 8, mq.ERR_ALIGNMENT)):
        with pytest.raises(mq.MatqError) as e:
            mq.attn_paged(*args, workspace=torch.empty(need + 16, dtype=torch.uint8, device="cuda")[start:start + size])
        assert e.value.status == status
    a = mq.attn_paged(*args, workspace=torch.empty(need // 4, dtype=torch.float32, device="cuda"))
    assert torch.equal(a, mq.attn_paged(*args))


@pytest.mark.parametrize("cap", [0.0, 50.0])
def test_attn_paged_rows_that_stand_for_no_query_cost_nothing(cap):
    # Groups of 5 and 7 leave rows of a query tile empty: they hold what the kernel before left in shared memory.  Behind a product of huge numbers a call takes
    # as long as behind one of ordinary numbers, and gives the same.
    def time_of(fill, q, kc, vc, table, cu, lens, n, L, ws):
        a = torch.full((4096, 4096), fill, device="cuda", dtype=torch.bfloat16)
        b = torch.empty_like(a)
        out, times = torch.empty_like(q), []
        for _ in range(9):
            torch.matmul(a, a, out=b)
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            mq.attn_paged(q, kc, vc, table, cu, lens, n, L, softcap=cap, out=out, workspace=ws)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end))
        return sorted(times)[4], out
    for D, Hkv, G, n, L in ((128, 8, 5, 1000, 3000), (64, 4, 7, 2000, 4000)):
        pages = -(-L // 16)
        kc = torch.randn(pages, Hkv, 16, D, device="cuda").to(torch.bfloat16)
        vc = torch.randn_like(kc)
        table = torch.randperm(pages, device="cuda").to(torch.int32)[None]
        cu, lens = dev(np.array([0, n], np.int32)), dev(np.array([L], np.int32))
        q = torch.randn(n, Hkv * G, D, device="cuda").to(torch.bfloat16)
        ws = torch.empty(mq.attn_paged_workspace_bytes(n, 1, Hkv * G, Hkv, D, n, L) + 16, dtype=torch.uint8, device="cuda")
        t1, o1 = time_of(1.0, q, kc, vc, table, cu, lens, n, L, ws)
        t2, o2 = time_of(1e30, q, kc, vc, table, cu, lens, n, L, ws)
        assert torch.equal(o1, o2)
        assert t2 < 1.4 * t1, (t1, t2)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap,window", [(0.0, 0), (30.0, 0), (30.0, 37)])
@pytest.mark.parametrize("n,L,hint", [(1, 59, 59), (3, 700, 700), (9, 29, 29), (9, 409, 1 << 20), (60, 500, 1 << 20), (140, 300, 300), (700, 1003, 1003)])
def test_attn_paged_does_not_depend_on_what_the_cache_holds_elsewhere(D, cap, window, n, L, hint):
    # not in the last bit: slots past a sequence's end and pages of nobody hold zeros, noise, huge numbers, infinities or NaN
    first = None
    for fill in (0.0, None, 1e30, -1e30, float("inf"), float("nan")):
        got, want, tol, status = _attend([n], [L], 4, 2, D, 16, seed=95, softcap=cap, window=window, hints=(n, hint), fill=fill)
        if first is None:
            first = got
            _check(got, want, tol, status)
        assert torch.equal(got, first), fill


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,L,hint", [(1, 700, 700), (4, 700, 700), (60, 500, 1 << 20), (140, 900, 1 << 20), (140, 300, 300)])
@pytest.mark.parametrize("exponent,cap", [(24, 2.0 ** 31), (30, 2.0 ** 38), (34, 2.0 ** 41), (34, 2.0 ** 60), (60, 2.0 ** 69), (60, 2.0 ** 99), (40, 50.0)])
def test_attn_paged_large_scores_under_a_large_cap(D, n, L, hint, exponent, cap):
    for step in (None, 200):
        _check(*_attend([n], [L], 4, 2, D, 16, seed=56, scale=1.0, softcap=cap, hints=(n, hint), edit=_sign_scores(D, n, L, exponent, step)))
