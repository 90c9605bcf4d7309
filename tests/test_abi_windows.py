"""Attention windows that no position reaches, up to the largest number: the same launches as without one (no GPU needed)."""
import pytest

from paper_2502_06786_b200 import binding as mq


@pytest.mark.parametrize("window", [1 << 31, 1 << 62, (1 << 63) - 1])
def test_windows_past_every_position_choose_what_no_window_does(window):
    for T, batch, Hq, Hkv, D, max_q, max_kv in ((30, 1, 8, 2, 128, 30, 40), (100, 3, 8, 2, 64, 60, 5000), (600, 1, 16, 2, 64, 600, 600), (4096, 1, 32, 8, 128, 4096, 8192),
                                                (70, 2, 16, 2, 256, 60, 9000), (5, 1, 8, 2, 128, 5, (1 << 63) - 1)):
        args = T, batch, Hq, Hkv, D, max_q, max_kv
        assert mq.attn_paged4_plan(*args, window) == mq.attn_paged4_plan(*args), args
        assert mq.attn_paged4_workspace_bytes(*args, window) == mq.attn_paged4_workspace_bytes(*args), args
        assert mq.attn_paged_workspace_bytes(*args, window) == mq.attn_paged_workspace_bytes(*args), args
