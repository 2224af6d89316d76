"""RadarLayer.step at a token that restructures is append(), then decode(), those of
a subclass too (on the CPU: both are replaced)."""
import torch

import paper_2503_10571_amd as radar


def test_restructuring_step_calls_append_and_decode():
    calls = []

    class Layer(radar.RadarLayer):
        def append(self, k_new, v_new):
            calls.append(("append", k_new, v_new))

        def decode(self, q, out=None, selected=None, scores=None):
            calls.append(("decode", q, out))
            return "output"

    layer = Layer.__new__(Layer)
    layer.cfg = radar.Config(1, 1, 1, 64, 64, 4, 0, 64, torch.float32)
    layer.schedule, layer.rope, layer.t, layer.pos = "sqrt", None, 24, 24   # 25 = 5^2 comes
    assert layer.step("q", "k", "v", out="o") == "output"
    assert calls == [("append", "k", "v"), ("decode", "q", "o")]
