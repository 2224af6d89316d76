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


@pytest.mark.parametrize("dtype", list(DT))
def test_new_outputs_are_zero_behind_the_lengths(dtype):
    """Also where the memory they get held something else."""
    B, T, Hq, Hkv, d = 3, 6, 4, 2, 64
    rope = _rope(64)
    q = torch.randn(B, T, Hq, d, device="cuda").to(DT[dtype])
    k, v = (torch.randn(B, T, Hkv, d, device="cuda").to(DT[dtype]) for _ in range(2))
    lens = torch.tensor([6, 0, 2], device="cuda")
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, 20, DT[dtype])
    K, V = (torch.zeros(B, Hkv, 20, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    ref, tol = _ref(q, rope, _grid(4, B, T))

    def calls():
        yield radar.rotary(rope, q, 4, lens=lens)
        yield radar.rotary_qk(rope, q, k, 4, lens=lens)[0]
        yield radar.rotary_fill(cfg, rope, K, V, k, v, 4, q=q, lens=lens)
        a, b = radar.rotary_qk(rope, k, q, 4, lens=lens)
        assert bool((a[1] == 0).all())
        yield b

    it = calls()
    for _ in range(4):
        used = [torch.full_like(q, float("nan")) for _ in range(4)]
        del used
        got = next(it)
        for b, n in enumerate((6, 0, 2)):
            _close(got[b, :n], ref[b, :n], tol[b, :n])
            assert bool((got[b, n:] == 0).all())
        del got
