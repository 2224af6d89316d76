"""The calls that autograd does not know refuse operands whose gradient would be
lost (checked before anything else, on the CPU)."""
import types

import pytest
import torch

import paper_2503_10571_amd as radar

CFG = radar.Config(1, 2, 2, 64, 64, 16, 16, 32, torch.float32)
ROPE = types.SimpleNamespace(inv_freq=torch.ones(32, dtype=torch.float64))


def _calls():
    x, y, c, m = torch.zeros(1, 1, 2, 64), torch.zeros(1, 2, 64), torch.zeros(1, 2, 32, 64), torch.zeros(1, 2, 32)
    for i in range(3):
        a = [x.clone().requires_grad_(i == j) for j in range(3)]
        yield "fill", lambda a=a: radar.rotary_fill(CFG, ROPE, c, c, a[0], a[1], 0, q=a[2])
    for i in range(5):
        a = [v.clone().requires_grad_(i == j) for j, v in enumerate((y, c[0], c[0], c, c))]
        yield "prefix", lambda a=a: radar.attend_prefix(CFG, a[0], a[1], a[2], 3, a[3], a[4], 3)
    for i in range(3):
        a = [v.clone().requires_grad_(i == j) for j, v in enumerate((y, c, c))]
        yield "accumulate", lambda a=a: radar.attend_accumulate(CFG, *a, m, 3)


def test_operands_that_want_a_gradient_are_refused():
    for name, call in _calls():
        with pytest.raises(RuntimeError, match=f"{name}.* has no gradient"):
            call()
        # not recorded: on to the next check
        with torch.no_grad(), pytest.raises(ValueError, match="device"):
            call()
