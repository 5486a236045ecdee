"""Which heads the example's serving layer (paper_1603_02297_amd/decoder.py) takes: refusals before anything is in the cache."""
import pytest
import torch

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import decoder


@pytest.mark.parametrize("dim", [16, 288])
def test_heads_that_share_no_keys_evenly_are_refused_before_anything_is_mapped(monkeypatch, dim):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write", "ttc_pages_append", "ttc_pages_read", "ttc_attend_pages"):
        monkeypatch.setattr(ttc, name, lambda *args, name=name: called.append(name))
    cache = decoder.PagedCache(3, 2, dim, 8, 9, 24, torch.float32, torch.float32, device="cpu")
    w = decoder.weights(32, 3, 2, dim, 4, 16, torch.float32, device="cpu")
    with pytest.raises(ValueError, match="heads"):
        decoder.layer(torch.randn(3, 32), torch.ones(3, dtype=torch.int32), cache, w, 3, 2)
    assert not called and cache.cached.tolist() == [0, 0, 0] and cache.free.numel() == 9


def test_what_the_library_refuses_is_refused_before_anything_is_mapped(monkeypatch):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write"):
        monkeypatch.setattr(ttc, name, lambda *args, name=name: called.append(name))

    def no(*args):
        raise ttc.TtcError(ttc.TTC_ERR_ALLOC, "ttc_attend_create")
    monkeypatch.setattr(ttc, "ttc_attend_create", no)
    cache = decoder.PagedCache(3, 2, 16, 8, 9, 24, torch.float32, torch.float32, device="cpu")
    with pytest.raises(ttc.TtcError):
        decoder.layer(torch.randn(3, 32), torch.ones(3, dtype=torch.int32), cache, decoder.weights(32, 4, 2, 16, 4, 16, torch.float32, device="cpu"), 4, 2)
    assert not called and cache.cached.tolist() == [0, 0, 0] and cache.free.numel() == 9

