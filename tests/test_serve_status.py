"""The decoder example hands its status word to every call that can report something (host only)."""
import types

import pytest
import torch

from paper_2502_06786_b200 import serve


@pytest.mark.parametrize("T", [1, serve.FEW, serve.FEW + 1, 40])
@pytest.mark.parametrize("grouped", [False, True])
def test_every_product_gets_the_status_word(monkeypatch, T, grouped):
    K, N = 128, 64
    status, seen = torch.zeros(1, dtype=torch.int32), []

    def noted(result):
        def call(*args, dev_status=None, **kw):
            seen.append(dev_status)
            return result
        return call
    y = torch.zeros(T, N, dtype=torch.bfloat16)
    monkeypatch.setattr(serve.mq, "gemv_groups", noted(y))
    monkeypatch.setattr(serve.mq, "gemv_grouped", noted(None))
    monkeypatch.setattr(serve.mq, "quantize_tokens", noted((None, None, None)))
    monkeypatch.setattr(serve.mq, "gemm_a8", noted(y))
    if grouped:
        linear = serve.GroupedLinear.__new__(serve.GroupedLinear)
        linear.packed, linear.params = None, None
    else:
        linear = types.SimpleNamespace(N=N, K=K, r=4, packed=None, sliced=None, alpha=None, zero=None)
    out = serve.apply([linear, linear], torch.zeros(T, K, dtype=torch.bfloat16), status)
    assert [tuple(o.shape) for o in out] == [(T, N)] * 2
    assert seen and all(s is status for s in seen)
