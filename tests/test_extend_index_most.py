"""extend_index() of sequences of different lengths: how many rows a sequence has added
cannot be told from t0 and t, so it has to be said (on the CPU: refused before a tensor is
looked at)."""
import pytest
import torch

import paper_2503_10571_amd as radar


class _Reached(Exception):
    pass


def test_most_is_needed(monkeypatch):
    def reached(*a):
        raise _Reached

    monkeypatch.setattr(radar.cache_ops, "_cache", reached)
    cfg = radar.Config(2, 4, 2, 64, 64, 4, 4, 128)
    lens0, lens = torch.tensor([100, 57]), torch.tensor([101, 65])
    # (t - t0 = 1 row would leave out seven of the second sequence's)
    with pytest.raises(ValueError, match="most"):
        radar.extend_index(cfg, None, None, 100, 101, None, lens0=lens0, lens=lens)
    with pytest.raises(_Reached):
        radar.extend_index(cfg, None, None, 100, 101, None, lens0=lens0, lens=lens, most=8)
    with pytest.raises(_Reached):
        radar.extend_index(cfg, None, None, 0, 101, None, lens0=lens0, lens=lens)
    with pytest.raises(_Reached):
        radar.extend_index(cfg, None, None, 100, 101, None)
