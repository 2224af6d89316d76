"""RadarLayer.prefill: a chunk that is not the layer's is refused before anything
is written (on the CPU: the cache is host memory and no kernel is reached)."""
import pytest
import torch

import paper_2503_10571_amd as radar


def _layer(rope=None):
    cfg = radar.Config(2, 4, 2, 64, 64, 16, 16, 32, torch.bfloat16)
    layer = radar.RadarLayer.__new__(radar.RadarLayer)
    layer.cfg, layer.schedule, layer.rope, layer.t, layer.pos = cfg, "fixed", rope, 0, 0
    layer.K, layer.V = (torch.full((2, 2, 32, 64), 9.0).bfloat16() for _ in range(2))
    layer._reindex = lambda: None
    return layer


def _x(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape).to(dtype)


GOOD = (2, 3, 2, 64)


@pytest.mark.parametrize("rope", [None, object()])
@pytest.mark.parametrize("shape,dtype", [
    ((2, 3, 1, 64), torch.bfloat16),             # one kv head of two
    ((1, 3, 2, 64), torch.bfloat16),             # one sequence of two
    ((2, 1, 2, 64), torch.bfloat16),             # one token beside three
    ((2, 3, 2, 1), torch.bfloat16),
    ((2, 3, 2, 64), torch.float32),
    ((2, 2, 64), torch.bfloat16),                # one token without its axis
    ((3, 2, 64), torch.bfloat16),
])
def test_chunks_of_another_shape_or_type(shape, dtype, rope):
    layer = _layer(rope)
    bad = _x(*shape, dtype=dtype)
    calls = [(_x(*GOOD), bad), (bad, bad)]
    if shape != (2, 1, 2, 64):                   # as k it is a chunk of one token
        calls.append((bad, _x(*GOOD)))
    for k, v in calls:
        if k is v and shape == (2, 1, 2, 64):
            continue
        with pytest.raises(ValueError, match="must be torch.bfloat16"):
            layer.prefill(k, v)
    assert layer.t == layer.pos == 0
    assert bool((layer.K == 9).all()) and bool((layer.V == 9).all())


def test_query_output_without_rope():
    layer = _layer()
    k, v, q = _x(*GOOD), _x(*GOOD), _x(2, 3, 4, 64)
    out = torch.zeros_like(q)
    assert layer.prefill(k, v, q=q, q_out=out) is out
    assert torch.equal(out, q) and layer.t == layer.pos == 3
    assert torch.equal(layer.K[:, :, :3], k.transpose(1, 2)) and bool((layer.K[:, :, 3:] == 9).all())
    assert layer.prefill(k, v, q=q) is q and layer.prefill(k, v) is None
    for bad in (dict(q_out=out), dict(q=q, q_out=out[:, :1]), dict(q=q, q_out=out.float())):
        with pytest.raises(ValueError, match="q_out"):
            layer.prefill(k, v, **bad)
    with pytest.raises(radar.RadarError, match="capacity"):
        layer.prefill(_x(2, 30, 2, 64), _x(2, 30, 2, 64), q=q, q_out=torch.zeros_like(q))
    assert layer.t == 9


def test_chunks_that_want_a_gradient():
    layer = _layer()
    with pytest.raises(RuntimeError, match="gradient"):
        layer.prefill(_x(*GOOD).requires_grad_(), _x(*GOOD))
    with torch.no_grad():
        layer.prefill(_x(*GOOD).requires_grad_(), _x(*GOOD))
    assert layer.t == 3 and not layer.K.requires_grad
