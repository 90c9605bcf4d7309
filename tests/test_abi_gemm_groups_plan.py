"""How the call for many tokens on 4-bit groups shares out its sizes (no GPU needed)."""
import random

import pytest
import torch

from paper_2502_06786_b200 import binding as mq

plan = mq.gemm_groups_plan


def test_tiles_are_as_wide_as_the_products_take_them():
    """tcgen05.mma: a CTA's 128 rows with tokens in steps of 16, a pair's 256 rows in steps of 32, 256 at most."""
    rng = random.Random(0)
    sizes = [(M, N, K) for M in range(1, 1200, 7) for N, K in ((14336, 4096), (9547, 640), (3849, 640))]
    sizes += [(rng.randint(1, 1 << rng.randint(1, 20)), rng.randint(1, 1 << rng.randint(1, 18)), 128 * rng.randint(1, 512)) for _ in range(4000)]
    widths = set()
    for M, N, K in sizes:
        for group in (32, 64, 128):
            for dtype in (torch.float32, torch.bfloat16):
                pairs, tokens, parts = plan(M, N, K, group, dtype)
                assert tokens > 0 and tokens % (32 if pairs else 16) == 0 and tokens <= (256 if pairs else 128), (M, N, K, group)
                assert parts in (1, 2, 4, 8) and (dtype == torch.bfloat16 and parts == 1 or not pairs)
                if pairs:
                    widths.add(tokens)
    assert widths >= {160, 192, 224, 256}


def test_refusals():
    for args, st in (((0, 8, 256, 64), mq.ERR_INVALID_ARG), ((8, 0, 256, 64), mq.ERR_INVALID_ARG), ((8, 8, -64, 64), mq.ERR_INVALID_ARG), ((8, 8, 256, 16), mq.ERR_UNSUPPORTED),
                     ((8, 8, 0, 64), mq.ERR_SHAPE), ((8, 8, 250, 64), mq.ERR_SHAPE), ((8, 8, 65600, 32), mq.ERR_SHAPE), ((1 << 31, 8, 256, 64), mq.ERR_SHAPE),
                     ((1 << 24, 1 << 30, 256, 64), mq.ERR_SHAPE)):
        with pytest.raises(mq.MatqError) as e:
            plan(*args)
        assert e.value.status == st, args
    assert mq._lib.matq_gemm_groups_plan(8, 8, 256, 64, 2, None, None, None) == mq.ERR_INVALID_ARG
    assert mq._lib.matq_gemm_groups_plan(8, 8, 256, 64, mq.OUT_BF16, None, None, None) == mq.OK
