"""Attention over keys that hold NaN: the softmax of a row with a NaN logit is NaN
everywhere, outputs and weights, wherever the NaNs lie and however the call is cut
(a part of the cache that holds nothing else has no maximum)."""
import pytest
import torch

import paper_2503_10571_amd as radar

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t", [3000, 70000])
def test_weights_beside_keys_of_nan(t, dtype):
    B, Hkv, G, d = 2, 1, 2, 64
    cfg = radar.Config(B, Hkv * G, Hkv, d, 64, 16, 16, t + 3, dtype)
    q = torch.randn(B, Hkv * G, d, device="cuda").to(dtype)
    K, V = (torch.randn(B, Hkv, t + 3, d, device="cuda").to(dtype) for _ in range(2))
    for first, n in [(0, n) for n in range(64, 577, 64)] + [(64, 64), (384, 384), (t - 1, 1), (0, t)]:
        bad = K.clone()
        bad[0, :, first:first + n] = float("nan")
        mass = torch.ones(B, Hkv, t + 3, device="cuda")
        out = radar.attend_accumulate(cfg, q, bad, V, mass, t)
        assert bool(out[0].isnan().all()), (first, n)
        assert bool(mass[0, :, :t].isnan().all()), (first, n, int(mass[0].isnan().sum()))
        assert bool(out[1].isfinite().all()) and bool(mass[1].isfinite().all())
        assert bool((mass[:, :, t:] == 1).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,P,t", [(1, 300, 40), (1, 20000, 100), (20, 20000, 100), (70, 3000, 50)])
def test_outputs_beside_keys_of_nan(B, P, t, dtype):
    Hkv, G, d = 1, 2, 64
    cfg = radar.Config(B, Hkv * G, Hkv, d, 64, 16, 16, t, dtype)
    q = torch.randn(B, Hkv * G, d, device="cuda").to(dtype)
    Kp, Vp = (torch.randn(Hkv, P, d, device="cuda").to(dtype) for _ in range(2))
    K, V = (torch.randn(B, Hkv, t, d, device="cuda").to(dtype) for _ in range(2))
    for first, n in [(0, n) for n in (1, 64, 128, 192, 256)] + [(P - 1, 1), (0, P)]:
        bad = Kp.clone()
        bad[:, first:first + n] = float("nan")
        assert bool(radar.attend_prefix(cfg, q, bad, Vp, P, K, V, t).isnan().all()), (first, n)
    bad = K.clone()
    bad[0, :, :] = float("nan")
    out = radar.attend_prefix(cfg, q, Kp, Vp, P, bad, V, t)
    assert bool(out[0].isnan().all()) and bool(out[1:].isfinite().all())
