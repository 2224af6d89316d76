"""Calls of the rotary operators beside those of test_gpu_rotary.py: operands
without heads."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from test_gpu_rotary import DT, _close, _grid, _ref, _rope  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
def test_one_operand_without_heads(dtype):
    """The other one is rotated all the same."""
    rope = _rope(64)
    qkv = torch.randn(2, 5, 4, 64, device="cuda").to(DT[dtype])
    x, none = qkv[:, :, :3], qkv[:, :, :0]
    ref = _ref(x, rope, _grid(3, 2, 5))
    for into in (None, torch.full_like(x, 7.0)):
        a, b = radar.rotary_qk(rope, x, none, 3, q_out=into)
        _close(a, *ref)
        assert b.shape == (2, 5, 0, 64)
        a, b = radar.rotary_qk(rope, none, x, 3, k_out=into)
        _close(b, *ref)
        assert a.shape == (2, 5, 0, 64)
    a, b = radar.rotary_qk(rope, none, none, 3)
    assert a.shape == b.shape == (2, 5, 0, 64)
