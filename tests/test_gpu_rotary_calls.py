"""Calls of the rotary operators beside those of test_gpu_rotary.py: operands
without heads, new outputs behind the lengths, autograd."""
import copy
import dataclasses
import os
import pickle
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


# ---- autograd: the gradient of the rotation is the inverse rotation of the output's ----
POS = pytest.mark.parametrize("where", ["int", "sequence", "token"])


def _places(where, B, T):
    """(pos argument, its grid [B][T])."""
    if where == "int":
        return 777, _grid(777, B, T)
    if where == "sequence":
        p = torch.tensor([5 + 1000 * b for b in range(B)])
        return p.cuda(), p[:, None] + torch.arange(T)
    p = torch.randint(0, 100000, (B, T), generator=torch.Generator().manual_seed(2))
    return p.cuda(), p


@POS
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
def test_autograd_of_qk(dtype, inter, inverse, where):
    """q and k as slices of one leaf, whose gradient holds both and zeros for v."""
    B, T, Hq, Hkv, d = 2, 5, 4, 2, 64
    rope = _rope(48, inter, "yarn", 4.0)
    pos, grid = _places(where, B, T)
    qkv = torch.randn(B, T, Hq + 2 * Hkv, d, device="cuda").to(DT[dtype]).requires_grad_()
    q, k, _ = qkv.split([Hq, Hkv, Hkv], 2)
    a, b = radar.rotary_qk(rope, q, k, pos, inverse=inverse)
    _close(a.detach(), *_ref(q, rope, grid, inverse))
    da, db = torch.randn_like(a), torch.randn_like(b)
    torch.autograd.backward([a, b], [da, db])
    _close(qkv.grad[:, :, :Hq], *_ref(da, rope, grid, not inverse))
    _close(qkv.grad[:, :, Hq:Hq + Hkv], *_ref(db, rope, grid, not inverse))
    assert not bool(qkv.grad[:, :, Hq + Hkv:].any())
    # one token, and only one of the two wants a gradient
    for i in range(2):
        q1, k1 = (x[:, 0].detach().clone().requires_grad_(i == j) for j, x in enumerate((q, k)))
        if where == "token":
            pos1, grid1 = pos[:, :1].contiguous(), grid[:, :1]
        else:
            pos1, grid1 = pos, grid[:, :1]
        got = radar.rotary_qk(rope, q1, k1, pos1, inverse=inverse)
        dy = torch.randn_like(got[i])
        got[i].backward(dy)
        _close((q1, k1)[i].grad[:, None], *_ref(dy[:, None], rope, grid1, not inverse))
        assert (k1, q1)[i].grad is None


def test_autograd_against_differences():
    """The map is linear: a difference over a step of any length is its derivative."""
    rope = _rope(48, True, "yarn", 4.0)
    x = torch.randn(2, 5, 3, 64, device="cuda", requires_grad=True)
    y = torch.randn(2, 5, 3, 64, device="cuda")
    fwd = radar.rotary(rope, x, 777)
    (fwd * y).sum().backward()
    for i in (0, 30, 50):
        e = torch.zeros_like(x)
        e[1, 2, 0, i] = 1.0
        with torch.no_grad():
            diff = (radar.rotary(rope, x + e, 777).double() - fwd.double()).mul(y.double()).sum()
        # as in test_gradient: both rotations of the pair's values, and x + e
        lim = 8 * 2.0 ** -24 * float((x.detach()[1, 2, 0].abs().max() + 1) * y[1, 2, 0].abs().max()) * rope.mscale * 8
        assert abs(float(diff) - float(x.grad[1, 2, 0, i])) <= lim


@POS
def test_autograd_with_lengths(where):
    """No gradient reaches the tokens behind the lengths."""
    B, T = 3, 6
    rope = _rope(64)
    pos, grid = _places(where, B, T)
    lens = torch.tensor([6, 0, 2], device="cuda")
    x = torch.randn(B, T, 2, 64, device="cuda", requires_grad=True)
    out = radar.rotary(rope, x, pos, lens=lens)
    dy = torch.randn_like(out)
    out.backward(dy)
    ref, tol = _ref(dy, rope, grid, True)
    for b, n in enumerate((6, 0, 2)):
        _close(x.grad[b, :n], ref[b, :n], tol[b, :n])
        assert not bool(x.grad[b, n:].any()) and not bool(out[b, n:].any())


def test_autograd_of_broadcast_operands_and_odd_gradients():
    """A head shared by all: the sum of its gradients. A gradient of one element's
    memory, and one that begins off 16 bytes."""
    rope = _rope(64)
    x = torch.randn(2, 3, 1, 64, device="cuda", requires_grad=True)
    out = radar.rotary(rope, x.expand(2, 3, 4, 64), 9)
    dy = torch.randn_like(out)
    (g,) = torch.autograd.grad(out, x, dy, retain_graph=True)
    ref, tol = _ref(dy, rope, _grid(9, 2, 3), True)
    ref, tol = ref.sum(2, keepdim=True), (tol + 3 * 2.0 ** -24 * ref.abs()).sum(2, keepdim=True)
    _close(g, ref, tol + 3 * 2.0 ** -24 * tol)
    one = torch.ones((), device="cuda").expand(2, 3, 4, 64)
    odd = torch.ones(2 * 3 * 4 * 64 + 1, device="cuda")[1:].view(2, 3, 4, 64)
    (a,) = torch.autograd.grad(out, x, one, retain_graph=True)
    (b,) = torch.autograd.grad(out, x, odd)
    assert torch.equal(a, b)


def test_autograd_twice():
    """The gradient of <R' y, z> in y is R z."""
    rope = _rope(64, True)
    x = torch.randn(1, 4, 2, 64, device="cuda", requires_grad=True)
    y = torch.randn(1, 4, 2, 64, device="cuda", requires_grad=True)
    z = torch.randn(1, 4, 2, 64, device="cuda")
    (g,) = torch.autograd.grad(radar.rotary(rope, x, 3), x, y, create_graph=True)
    (gg,) = torch.autograd.grad(g, y, z)
    _close(gg, *_ref(z, rope, _grid(3, 1, 4)))


def test_autograd_finds_changes_in_place():
    rope = _rope(64)
    x = torch.randn(2, 1, 2, 64, device="cuda", requires_grad=True)
    for name in ("pos", "lens"):
        kw = dict(pos=torch.tensor([3, 5], device="cuda"), lens=torch.tensor([1, 1], device="cuda"))
        out = radar.rotary(rope, x, **kw)
        kw[name] += 1
        with pytest.raises(RuntimeError, match="inplace"):
            out.sum().backward()


def test_autograd_refusals():
    rope = _rope(64)
    x = torch.randn(2, 3, 2, 64, device="cuda", requires_grad=True)
    k = torch.randn(2, 3, 2, 64, device="cuda")
    for call in (lambda: radar.rotary(rope, x, 0, out=torch.empty_like(k)),
                 lambda: radar.rotary_qk(rope, k, x, 0, q_out=k),
                 lambda: radar.rotary_qk(rope, x, k, 0, k_out=k)):
        with pytest.raises(RuntimeError, match="gradient"):
            call()
    learned = radar.Rope(rope.inv_freq.clone().requires_grad_())
    with pytest.raises(RuntimeError, match="inv_freq"):
        radar.rotary(learned, k, 0)
    with torch.no_grad():                                # nothing is recorded here
        assert not radar.rotary(learned, x, 0, out=torch.empty_like(k)).requires_grad
    assert not radar.rotary(rope, k, 0).requires_grad


def test_autograd_captured():
    """Forward and backward in one graph: every replay the eager gradients."""
    rope = _rope(64)
    pos = torch.tensor([3, 9], device="cuda")
    x = torch.randn(2, 4, 3, 64, device="cuda", requires_grad=True)
    dy = torch.randn(2, 4, 3, 64, device="cuda")

    def both(x):
        out = radar.rotary(rope, x, pos)
        return out.detach(), torch.autograd.grad(out, x, dy)[0]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(x)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, dx = both(x)
    for rep in range(3):
        pos += 11
        with torch.no_grad():
            x.mul_(0.5)
        want, wdx = both(x.detach().clone().requires_grad_())
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        assert torch.equal(out, want) and torch.equal(dx, wdx), rep


# ---- the operator's handle ---------------------------------------------------------
def test_rope_copies():
    """Deep copies and pickles hold frequencies of their own; equal are those of the
    same tensor."""
    rope = _rope(48, True, "yarn", 4.0)
    x = torch.randn(2, 3, 2, 64, device="cuda")
    want = radar.rotary(rope, x, 99)
    for other in (copy.copy(rope), copy.deepcopy(rope), pickle.loads(pickle.dumps(rope))):
        assert (other.rot_dim, other.interleaved, other.mscale) == (48, True, rope.mscale)
        assert torch.equal(radar.rotary(other, x, 99), want)
        same = other.inv_freq is rope.inv_freq
        assert (other == rope) is same and len({rope, other}) == (1 if same else 2)
    assert copy.copy(rope) == rope == radar.Rope(rope.inv_freq, True, rope.mscale)
    assert rope != radar.Rope(rope.inv_freq, False, rope.mscale) and rope != 1
    deep = copy.deepcopy(rope)
    assert deep.inv_freq.data_ptr() != rope.inv_freq.data_ptr()
    rope.inv_freq.zero_()
    assert torch.equal(radar.rotary(deep, x, 99), want)
    # with a changed field, as a dataclass
    flat = dataclasses.replace(deep, interleaved=False)
    _close(radar.rotary(flat, x, 99), *_ref(x, flat, _grid(99, 2, 3)))


@pytest.mark.parametrize("fill", [False, True])
def test_captured_call_with_lengths_and_its_own_output(fill):
    """Shorter lengths in a later replay: zeros where the one before wrote."""
    B, T, H, d = 3, 6, 2, 64
    rope = _rope(64)
    cfg = radar.Config(B, H, H, d, 64, 16, 16, 20, torch.float32)
    x, k, v = (torch.randn(B, T, H, d, device="cuda") for _ in range(3))
    K, V = (torch.zeros(B, H, 20, d, device="cuda") for _ in range(2))
    lens = torch.tensor([6, 5, 4], device="cuda")

    def call():
        if fill:
            return radar.rotary_fill(cfg, rope, K, V, k, v, 4, q=x, lens=lens)
        return radar.rotary(rope, x, 4, lens=lens)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    for now in ([6, 6, 6], [6, 0, 2], [1, 3, 0]):
        lens.copy_(torch.tensor(now, device="cuda"))
        want = call()
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        assert torch.equal(out, want)
        for b, n in enumerate(now):
            assert not bool(out[b, n:].any())
