"""What the binding of the operators around the paged cache refuses by itself, before a device is needed."""
import types

import pytest


def test_weights_to_be_written_need_weights_to_be_read():
    import torch

    from paper_2511_21513_amd import binding

    def called(*_):
        raise AssertionError("the library was called")

    cache = types.SimpleNamespace(device=-1, B=1, Hkv=2, d=64, capacity=32, page_size=16, _ref=None)
    ia = binding.IntAttn.__new__(binding.IntAttn)
    ia.device, ia._lib, ia._ctx = -1, types.SimpleNamespace(intattn_cache_forward=called, intattn_destroy=lambda _: None), None
    ia._stream = lambda *_: None
    q, s, w = torch.zeros((1, 4, 1, 64), dtype=torch.int8), torch.ones((1, 4, 1)), torch.zeros((1, 2, 32))
    with pytest.raises(ValueError, match="weight_out needs weight"):
        ia.cache_forward(cache, q, s, weight_out=w)
    for more in ({}, dict(weight=w), dict(weight=w, weight_out=w.clone())):
        with pytest.raises(AssertionError, match="library was called"):
            ia.cache_forward(cache, q, s, **more)
