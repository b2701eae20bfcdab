"""Compressor.store8: a call that is refused has not touched the cache."""
import types

import pytest
import torch

from paper_2607_16213_amd import selkv as S


def test_refused_biases_come_before_the_write(monkeypatch):
    wrote = []
    monkeypatch.setattr(S, "cache8_write", lambda *a, **k: wrote.append(a))
    p = S.params(batch=1, n_heads_kv=2, group=2, head_dim=64)
    comp = S.Compressor.__new__(S.Compressor)
    comp.p, comp.K_out, comp.V_out, comp.m = p, None, None, 32
    cache = types.SimpleNamespace(capacity=64)
    for bias in (torch.zeros((1, 2, 63)), torch.zeros((1, 2, 64))):      # a wrong size; host memory
        with pytest.raises(ValueError, match="bias"):
            comp.store8(cache, bias)
    assert not wrote
    comp.store8(cache)
    assert len(wrote) == 1
