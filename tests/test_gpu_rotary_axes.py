"""Rotary positions on several axes, on the GPU against 64 bits.

An element of a rotated pair (a, b) is one of a c - b s, b c + a s with c and s
within 3 2^-24 of theirs (the turn's fraction in 32 bits: 2^-24 of a turn at
most half, 2 pi 2^-25 of a radian; sine, cosine and mscale rounded: 2 steps),
two products and a sum: 8 2^-24 (|a| + |b|) m, and half a step of the output's
type."""
import copy
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from test_gpu_canaries import Guarded  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DTYPES = pytest.mark.parametrize("dtype", list(DT))


def turned(x, freq, axis, pos, inter, m=1.0, inverse=False):
    """x [B][T][H][d] in 64 bits and the tolerance, positions pos [A][B][T]."""
    r, y = 2 * len(freq), x.double()
    i = torch.arange(r // 2)
    lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + r // 2)
    ang = torch.stack([pos[int(axis[j])].double() * float(freq[j]) for j in range(r // 2)], -1)
    c, s = m * torch.cos(ang)[:, :, None], m * torch.sin(ang)[:, :, None]
    if inverse:
        s = -s
    out, tol = y.clone(), torch.zeros_like(y)
    out[..., lo], out[..., hi] = y[..., lo] * c - y[..., hi] * s, y[..., hi] * c + y[..., lo] * s
    tol[..., lo] = tol[..., hi] = 8 * 2.0 ** -24 * m * (y[..., lo].abs() + y[..., hi].abs())
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
    return out, tol + half * (out.abs() + tol)


def near(got, ref, tol):
    assert not bool(got.isnan().any())
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


CASES = [  # B, T, Hq, Hk, d, sections, cycled, inter
    (1, 1, 4, 1, 128, (16, 24, 24), False, False),
    (2, 5, 8, 2, 128, (22, 21, 21), True, False),
    (3, 33, 2, 2, 64, (16, 16), False, True),
    (2, 67, 4, 4, 64, (8, 8, 8), True, True),         # 48 of 64 dims
    (1, 129, 5, 1, 128, (5, 2, 3), False, False),      # 20 dims: halves off 16 bytes
    (2, 9, 3, 1, 64, (1, 0, 4), True, True),           # an axis of no pairs
    (1, 300, 2, 1, 256, (128,), False, False),         # one axis
    (4, 7, 1, 1, 16, (2, 2, 2, 2), False, False),
]


@DTYPES
@pytest.mark.parametrize("B,T,Hq,Hk,d,sections,cycled,inter", CASES)
def test_rotary_qk(B, T, Hq, Hk, d, sections, cycled, inter, dtype):
    print(f"[case] axes B{B} T{T} Hq{Hq}/{Hk} d{d} {sections} cycled={cycled} inter={inter} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    axis = radar.rope_axes(sections, cycled)
    freq, _ = radar.rope_frequencies(2 * sum(sections))
    rope = radar.Rope(freq.cuda(), inter, 1.25, axis.cuda())
    x = torch.randn(B, T, Hq + Hk, d, generator=g, device="cuda").to(DT[dtype])
    q, k = x[:, :, :Hq], x[:, :, Hq:]
    pos = torch.randint(-3, 1 << 20, (len(sections), B, T), generator=g, device="cuda")
    for inverse in (False, True):
        qo, ko = radar.rotary_qk(rope, q, k, pos, inverse=inverse)
        near(qo, *turned(q, freq, axis, pos, inter, 1.25, inverse))
        near(ko, *turned(k, freq, axis, pos, inter, 1.25, inverse))
        assert torch.equal(qo, radar.rotary(rope, q, pos, inverse=inverse))
    # in place, and only some tokens
    lens = torch.tensor([max(0, T - 2 * b) for b in range(B)], device="cuda")
    y = q.contiguous()
    y = Guarded(y.shape, y.dtype, init=y)
    radar.rotary(rope, y.t, pos, out=y.t, lens=lens)
    ref = radar.rotary(rope, q, pos)
    torch.cuda.synchronize()
    assert y.intact()
    for b in range(B):
        n = int(lens[b])
        assert torch.equal(y.t[b, :n], ref[b, :n]) and torch.equal(y.t[b, n:], q[b, n:])


@DTYPES
@pytest.mark.parametrize("inter", [False, True])
def test_equal_axes_are_one_position(inter, dtype):
    """Every other kind of position is the same on all axes, bit for bit."""
    freq, _ = radar.rope_frequencies(128)
    plain = radar.Rope(freq.cuda(), inter)
    rope = radar.Rope(plain.inv_freq, inter, axis=radar.rope_axes((16, 24, 24)).cuda())
    x = torch.randn(2, 9, 3, 128, device="cuda").to(DT[dtype])
    each = torch.randint(0, 100000, (2, 9), device="cuda")
    for pos in (1234, each[:, 0].contiguous(), each):
        want = radar.rotary(plain, x, pos)
        assert torch.equal(radar.rotary(rope, x, pos), want)
    assert torch.equal(radar.rotary(rope, x, each.expand(3, 2, 9).contiguous()), want)
    one = torch.randint(0, 1000, (3, 2, 1), device="cuda")       # one token, no token axis
    assert torch.equal(radar.rotary(rope, x[:, 0], one), radar.rotary(rope, x[:, :1], one)[:, 0])


def test_axis_out_of_range_is_nan():
    freq, _ = radar.rope_frequencies(64)
    axis = torch.zeros(32, dtype=torch.int32, device="cuda")
    axis[3], axis[7] = 2, -1
    rope = radar.Rope(freq.cuda(), axis=axis)
    x = torch.randn(1, 4, 2, 64, device="cuda")
    out = radar.rotary(rope, x, torch.arange(8, device="cuda").view(2, 1, 4))
    bad = [3, 7, 35, 39]
    assert bool(out[..., bad].isnan().all())
    rest = [i for i in range(64) if i not in bad]
    assert not bool(out[..., rest].isnan().any())


@DTYPES
def test_fill(dtype):
    B, T, Hq, Hkv, d, cap = 3, 21, 4, 2, 64, 40
    g = torch.Generator(device="cuda").manual_seed(7)
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, cap, DT[dtype])
    freq, _ = radar.rope_frequencies(48)
    axis = radar.rope_axes((8, 8, 8), True)
    rope = radar.Rope(freq.cuda(), False, 1.0, axis.cuda())
    x = torch.randn(B, T, Hq + 2 * Hkv, d, generator=g, device="cuda").to(DT[dtype])
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    pos = torch.randint(0, 5000, (3, B, T), generator=g, device="cuda")
    lens = torch.tensor([21, 0, 7], device="cuda")
    rows = torch.tensor([0, 3, 19], device="cuda")
    K, V = (Guarded((B, Hkv, cap, d), DT[dtype], init=torch.zeros(B, Hkv, cap, d)) for _ in range(2))
    qo = radar.rotary_fill(cfg, rope, K.t, V.t, k, v, rows, pos=pos, q=q, lens=lens)
    torch.cuda.synchronize()
    assert K.intact() and V.intact()
    rq, tq = turned(q, freq, axis, pos, False)
    rk, tk = turned(k, freq, axis, pos, False)
    for b in range(B):
        n, r = int(lens[b]), int(rows[b])
        near(qo[b, :n], rq[b, :n], tq[b, :n])
        assert not bool(qo[b, n:].any())
        near(K.t[b, :, r:r + n].transpose(0, 1), rk[b, :n], tk[b, :n])
        assert torch.equal(V.t[b, :, r:r + n].transpose(0, 1), v[b, :n])
        K.t[b, :, r:r + n], V.t[b, :, r:r + n] = 0, 0
    assert not bool(K.t.any()) and not bool(V.t.any())


@DTYPES
def test_gradients(dtype):
    """Autograd against the transposed map, and (fp32) against differences."""
    B, T, H, d = 2, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    freq, _ = radar.rope_frequencies(48)
    axis = radar.rope_axes((10, 14))
    rope = radar.Rope(freq.cuda(), True, 1.5, axis.cuda())
    pos = torch.randint(0, 900, (2, B, T), generator=g, device="cuda")
    q, k = (torch.randn(B, T, H, d, generator=g, device="cuda").to(DT[dtype]).requires_grad_() for _ in range(2))
    wq, wk = (torch.randn(B, T, H, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    qo, ko = radar.rotary_qk(rope, q, k, pos)
    torch.autograd.backward((qo, ko), (wq, wk))
    near(q.grad, *turned(wq, freq, axis, pos, True, 1.5, True))
    near(k.grad, *turned(wk, freq, axis, pos, True, 1.5, True))
    if dtype == "f32":
        # the map is linear: its difference along u is its value at u, whatever the step
        u = torch.randn(B, T, H, d, generator=g, device="cuda")
        plus, minus = (q + u).detach(), (q - u).detach()
        diff = (radar.rotary(rope, plus, pos).double() - radar.rotary(rope, minus, pos).double()) / 2
        lhs, rhs = float((diff * wq.double()).sum()), float((q.grad.double() * u.double()).sum())
        # both outputs' tolerances and the gradient's, and q + u and q - u rounded
        lim = sum(float((turned(x, freq, axis, pos, True, 1.5)[1] * wq.abs()).sum()) / 2 for x in (plus, minus))
        lim += float((turned(wq, freq, axis, pos, True, 1.5, True)[1] * u.abs()).sum())
        lim += float((turned(wq, freq, axis, pos, True, 1.5, True)[0].abs() * (q.detach().abs() + u.abs())).sum()) * 2.0 ** -23
        assert abs(lhs - rhs) <= lim
    # a change of the positions before the backward pass is found
    out = radar.rotary(rope, q, pos)
    pos += 1
    with pytest.raises(RuntimeError):
        out.sum().backward()


def test_replayed_and_other_stream():
    freq, _ = radar.rope_frequencies(128)
    rope = radar.Rope(freq.cuda(), axis=radar.rope_axes((16, 24, 24)).cuda())
    x = torch.randn(2, 40, 4, 128, device="cuda").bfloat16()
    pos = torch.randint(0, 5000, (3, 2, 40), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        radar.rotary(rope, x, pos)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = radar.rotary(rope, x, pos)
    for i in range(4):
        x.copy_(torch.randn(2, 40, 4, 128, device="cuda"))
        pos.copy_(torch.randint(0, 5000, (3, 2, 40), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, radar.rotary(rope, x, pos))


def test_copies_and_equality():
    freq, _ = radar.rope_frequencies(64)
    axis = radar.rope_axes((16, 16)).cuda()
    rope = radar.Rope(freq.cuda(), axis=axis)
    other = copy.deepcopy(rope)
    assert torch.equal(other.axis, axis) and other.axis.data_ptr() != axis.data_ptr()
    assert rope == radar.Rope(rope.inv_freq, axis=axis) and rope != radar.Rope(rope.inv_freq)
    x = torch.randn(1, 3, 2, 64, device="cuda")
    pos = torch.arange(6, device="cuda").view(2, 1, 3)
    assert torch.equal(radar.rotary(rope, x, pos), radar.rotary(other, x, pos))


def test_binding_refuses():
    freq, _ = radar.rope_frequencies(64)
    axis = radar.rope_axes((16, 16)).cuda()
    f = freq.cuda()
    for bad in (axis[:31], axis.long(), axis.cpu(), torch.stack([axis, axis], 1)[:, 0]):
        with pytest.raises(ValueError):
            radar.Rope(f, axis=bad)
    x = torch.randn(2, 3, 2, 64, device="cuda")
    rope = radar.Rope(f, axis=axis)
    ok = torch.zeros(2, 2, 3, dtype=torch.int64, device="cuda")
    for bad in (ok.int(), ok[:, :1].contiguous(), ok[..., :2].contiguous(), ok[:0], ok.transpose(1, 2), ok.cpu()):
        with pytest.raises(ValueError):
            radar.rotary(rope, x, bad)
    with pytest.raises(ValueError):
        radar.rotary(radar.Rope(f), x, ok)
