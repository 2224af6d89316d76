"""RadarLayer between a draft and what is taken of it: sequences that become others take
their drafted rows along, and a refused path leaves every byte as it was."""
import pytest
import torch

import paper_2503_10571_amd as radar

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("schedule", ["fixed", "sqrt"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fork_between_draft_and_keep(dtype, schedule):
    B, Hq, Hkv, d, T, N, cap = 4, 4, 2, 64, 45, 6, 80
    print(f"[case] fork between draft and keep {dtype} {schedule}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(5)

    def rand(*s):
        return torch.randn(*s, generator=g, device="cuda").to(dtype)

    omega = torch.randn(64, d, generator=g, device="cuda").bfloat16().float()
    layer = radar.RadarLayer(radar.Config(B, Hq, Hkv, d, 64, 4, 4, cap, dtype), omega, top_k=8, schedule=schedule)
    layer.prefill(rand(B, T, Hkv, d), rand(B, T, Hkv, d))
    layer.accumulate(rand(B, Hq, d))
    k, v = rand(B, N, Hkv, d), rand(B, N, Hkv, d)
    layer.draft(rand(B, N, Hq, d), k, v)
    K, V, mass = layer.K.clone(), layer.V.clone(), layer.mass.clone()
    assert torch.equal(K[:, :, T:T + N], k.transpose(1, 2))
    for bad in ([[0, 0], [0, 1], [0, 1], [0, 1]], [[0, 1], [2, 1], [0, 1], [0, 1]], [[0, 1], [0, 1], [0, 1], [0, N]]):
        summ = layer.summaries.clone()
        with pytest.raises(ValueError):
            layer.keep(torch.tensor(bad, dtype=torch.int32, device="cuda"))
        assert (layer.t, layer.pos) == (T, T) and torch.equal(layer.summaries, summ)
        assert torch.equal(layer.K, K) and torch.equal(layer.V, V)
    src = [1, 0, 1, 2]                                 # a swap, a copy and one behind another
    layer.fork(torch.tensor(src, device="cuda"), first=7)
    path = [[0, 2, 5], [1, 2, 3], [0, 1, 2], [3, 4, 5]]
    layer.keep(torch.tensor(path, dtype=torch.int32, device="cuda"))
    assert (layer.t, layer.pos) == (T + 3, T + 3)
    for b in range(B):
        assert torch.equal(layer.K[b, :, 7:T], K[src[b], :, 7:T])
        assert torch.equal(layer.K[b, :, T:T + 3], K[src[b]][:, [T + i for i in path[b]]])
        assert torch.equal(layer.V[b, :, T:T + 3], V[src[b]][:, [T + i for i in path[b]]])
        assert torch.equal(layer.mass[b], mass[src[b]])
    # (the rows below 7 were said to be the same already, and are not: no segment of theirs)
    fresh = torch.zeros_like(layer.summaries)
    radar.build_index(layer.cfg, layer.K, omega, layer.t, fresh)
    c = layer.cfg.seg_len
    a, b = (x.flatten()[:B * Hkv * layer.cfg.summary_rows * 64].view(B, Hkv, -1, 64)[:, :, (7 + c - 1) // c:layer.t // c]
            for x in (layer.summaries, fresh))
    assert a.shape[2] > 0 and torch.equal(a, b)
