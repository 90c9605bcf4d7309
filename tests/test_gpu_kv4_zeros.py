"""attn_paged4: rows and keys of zeros, whose factors are the smallest there are, in calls that unpack."""
import numpy as np
import pytest
import torch

from paper_2502_06786_b200 import binding as mq
from tests import groups_ref as gr
from tests import kv4_rows_ref as rows_ref
from tests.util import dev, host, status_word

pytestmark = pytest.mark.gpu


def _run(n, L, Hq, Hkv, D, edit, softcap=0.0, window=0):
    kb, vb, table = gr.make_cache([L], Hkv, D, 32, 3)
    q = torch.randn(n, Hq, D, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    edit(q, kb, vb)
    tiles, status, cu = gr.cache_bytes(kb, vb), status_word(), [0, n]
    plan = mq.attn_paged4_plan(n, 1, Hq, Hkv, D, n, L, window)
    assert plan[2] == 1
    out = mq.attn_paged4(q.cuda(), dev(tiles), table.cuda(), dev(np.array(cu, np.int32)), dev(np.array([L], np.int32)), n, L, softcap=softcap, window=window, dev_status=status)
    assert int(host(status)[0]) == mq.OK
    rows_ref.check(out, *rows_ref.attn(q, tiles, table, cu, [L], D ** -0.5, softcap, window))
    return plan


# one part of the key range, and several, of which some rows see no key
@pytest.mark.parametrize("softcap", [0.0, 30.0])
@pytest.mark.parametrize("n,L,Hq,Hkv,D", [(1024, 1024, 8, 1, 64), (600, 600, 16, 2, 64), (450, 950, 16, 2, 64), (450, 450, 16, 2, 128), (704, 1204, 8, 1, 128), (256, 256, 16, 2, 256),
                                          (640, 640, 8, 2, 256)])
def test_zeros(n, L, Hq, Hkv, D, softcap):
    def prompt_of_zeros(q, kb, vb):
        q[:], kb[:], vb[:] = 0, 0, 0

    def queries(q, kb, vb):
        q[::3] = 0                                               # whole tokens
        q[1::3, 1] = 0                                           # a head of others

    def keys(q, kb, vb):
        q[::3] = 0
        kb[:, 0] = 0                                             # all keys of a head
        vb[:, -1] = 0

    def small(q, kb, vb):
        q[::2] = 0
        q[1::2] *= 2.0 ** -100
        kb[:] = gr.bf16_bits(gr.bf16_values(kb) * np.float32(2.0 ** -60))
    for edit in (prompt_of_zeros, queries, keys, small):
        _run(n, L, Hq, Hkv, D, edit, softcap)
