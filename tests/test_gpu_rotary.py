"""Rotary positions on the GPU against the formulas in 64 bits: both pair
layouts, parts of the head (those whose halves do not end on 16 bytes too),
strided operands, far positions, the gradient, and the fill of the cache.

Tolerance. a' = m (a cos - b sin) is taken in 32 bits: the reduced angle is off
by 2 pi 2^-26 = 1.6 2^-24, sine and cosine by two units (2 2^-24), each product
with m and with an operand and the sum by half a unit: fewer than 8 2^-24 of
m (|a| + |b|). Then one rounding to the output type, half a step of the value
(eps / 2)."""
import math

import pytest
import torch

import paper_2503_10571_amd as radar

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(rot, inter=False, scaling="none", factor=1.0, device="cuda"):
    f, m = radar.rope_frequencies(rot, 10000.0, scaling, factor, trained_len=4096)
    return radar.Rope(f.to(device), inter, m)


def _pairs(rot, inter):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)


def _ref(x, rope, pos, inverse=False):
    """(value, tolerance) of the rotation of x [B][T][H][d] at positions
    pos [B][T], in 64 bits on the CPU."""
    x = x.detach().double().cpu()
    lo, hi = _pairs(rope.rot_dim, rope.interleaved)
    ang = pos.double().cpu()[..., None] * rope.inv_freq.cpu()
    c, s = (rope.mscale * f(ang)[:, :, None] for f in (torch.cos, torch.sin))
    s = -s if inverse else s
    y, size = x.clone(), torch.zeros_like(x)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo] = size[..., hi] = rope.mscale * (a.abs() + b.abs())
    return y, 8 * 2.0 ** -24 * size


def _close(got, ref, tol):
    half = 0.0 if got.dtype == torch.float32 else torch.finfo(got.dtype).eps / 2
    err = (got.double().cpu() - ref).abs()
    lim = tol + half * (ref.abs() + tol)
    assert bool((err <= lim).all()), float((err - lim).max())


def _grid(pos, B, T):
    return torch.full((B, 1), pos) + torch.arange(T)


ROT = [  # d, rot, inter
    (128, 128, False), (128, 128, True), (64, 64, False), (64, 32, True), (128, 96, False),
    (128, 20, False), (128, 6, True), (64, 2, False), (64, 24, False), (80, 80, True),
    (256, 256, False), (256, 256, True), (16, 16, False), (48, 18, True)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("d,rot,inter", ROT)
def test_rotary(d, rot, inter, dtype):
    print(f"[case] rotary d={d} rot={rot} inter={inter} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(d + rot)
    rope = _rope(rot, inter)
    for B, T, H in ((1, 1, 1), (2, 7, 5), (3, 2, 33)):
        x = torch.randn(B, T, H, d, generator=g, device="cuda").to(DT[dtype])
        for inverse in (False, True):
            got = radar.rotary(rope, x, 1000, inverse=inverse)
            _close(got, *_ref(x, rope, _grid(1000, B, T), inverse))
        same = x.clone()
        assert radar.rotary(rope, same, 1000, out=same, inverse=True) is same
        assert torch.equal(same, got)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_far_positions(scaling):
    rope = _rope(128, False, scaling, 8.0 if scaling != "none" else 1.0)
    x = torch.randn(2, 3, 4, 128, device="cuda")
    for pos in (0, 131071, (1 << 20) + 1, (1 << 31) - 5, -77):
        _close(radar.rotary(rope, x, pos), *_ref(x, rope, _grid(pos, 2, 3)))


def test_positions_of_each_sequence_and_token():
    rope = _rope(64, True)
    x = torch.randn(3, 5, 2, 64, device="cuda")
    first = torch.tensor([0, 9999, 123456], device="cuda")
    ref, tol = _ref(x, rope, first[:, None].cpu() + torch.arange(5))
    _close(radar.rotary(rope, x, first), ref, tol)
    each = torch.randint(0, 100000, (3, 5), device="cuda")
    _close(radar.rotary(rope, x, each), *_ref(x, rope, each.cpu()))


@pytest.mark.parametrize("dtype", list(DT))
def test_strided_qk(dtype):
    """q and k as slices of one projection's output, transposed too, and into
    slices of another tensor; the rest of it stays."""
    B, T, Hq, Hkv, d = 2, 9, 6, 3, 64
    rope = _rope(d)
    qkv = torch.randn(B, T, Hq + 2 * Hkv, d, device="cuda").to(DT[dtype])
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    rq, rk = _ref(q, rope, _grid(5, B, T)), _ref(k, rope, _grid(5, B, T))
    for a, b in (radar.rotary_qk(rope, q, k, 5),):
        _close(a, *rq)
        _close(b, *rk)
    turned = q.transpose(1, 2).contiguous().transpose(1, 2)      # head-major memory
    _close(radar.rotary(rope, turned, 5), *rq)
    into = torch.full_like(qkv, 7.0)
    radar.rotary_qk(rope, q, k, 5, q_out=into[:, :, :Hq], k_out=into[:, :, Hq:Hq + Hkv])
    _close(into[:, :, :Hq], *rq)
    _close(into[:, :, Hq:Hq + Hkv], *rk)
    assert bool((into[:, :, Hq + Hkv:] == 7.0).all())
    # one token without its axis; in place of the projection's output
    q1, k1 = radar.rotary_qk(rope, q[:, 4], k[:, 4], 9)
    assert q1.shape == (B, Hq, d)
    _close(q1[:, None], rq[0][:, 4:5], rq[1][:, 4:5])
    v = qkv[:, :, Hq + Hkv:].clone()
    radar.rotary_qk(rope, q, k, 5, q_out=q, k_out=k)
    _close(qkv[:, :, :Hq], *rq)
    assert torch.equal(qkv[:, :, Hq + Hkv:], v)


def test_lens_leave_the_rest():
    rope = _rope(64)
    x = torch.randn(4, 6, 2, 64, device="cuda")
    out = torch.full_like(x, 3.0)
    radar.rotary(rope, x, 0, out=out, lens=torch.tensor([6, 0, 2, 99], device="cuda"))
    ref, tol = _ref(x, rope, _grid(0, 4, 6))
    for b, n in enumerate((6, 0, 2, 6)):
        _close(out[b, :n], ref[b, :n], tol[b, :n])
        assert bool((out[b, n:] == 3.0).all())


@pytest.mark.parametrize("rot", [16, 6])
def test_more_tokens_than_a_launch_has_threads(rot):
    """2^26 tokens of a wave each are 2^32 threads."""
    T = (1 << 26) + 5
    rope = _rope(rot)
    x = torch.zeros(1, T, 1, 16, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 3, (1 << 25) - 1, 1 << 25, (1 << 25) + 4, T - 6, T - 5, T - 1])
    x[:, at.cuda()] = torch.randn(1, len(at), 1, 16, device="cuda").bfloat16()
    was = x[:, at.cuda()].clone()
    radar.rotary(rope, x, 0, out=x)
    _close(x[:, at.cuda()], *_ref(was, rope, at[None]))
    x[:, at.cuda()] = 0
    assert not bool(x.any())


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,T", [("bf16", 20000), ("bf16", 40000), ("f32", 10000), ("f32", 20000)])
def test_large_calls(dtype, T, inter):
    """Calls of 328 and 655 MB, which pass the caches by: the bits of small ones."""
    rope = _rope(96 if inter else 128, inter)
    x = torch.randn(1, T, 32, 128, device="cuda").to(DT[dtype])
    out = radar.rotary(rope, x, 7)
    for t in range(0, T, 5000):
        assert torch.equal(out[:, t:t + 5000], radar.rotary(rope, x[:, t:t + 5000], 7 + t))


@pytest.mark.parametrize("inter", [False, True])
def test_gradient(inter):
    """inverse is the transposed map: <R x, y> = <x, R' y>, and what differences
    of <R x, y> give (the map is linear, so a step of any length is exact)."""
    rope = _rope(48, inter, "yarn", 4.0)
    x, y = (torch.randn(2, 5, 3, 64, device="cuda") for _ in range(2))
    fwd, back = radar.rotary(rope, x, 777), radar.rotary(rope, y, 777, inverse=True)
    lhs, rhs = (fwd.double() * y.double()).sum(), (x.double() * back.double()).sum()
    size = float((x.double().abs() * y.double().abs()).sum()) * rope.mscale * 2
    assert abs(float(lhs - rhs)) <= 16 * 2.0 ** -24 * size
    _close(back, *_ref(y, rope, _grid(777, 2, 5), True))
    for i in (0, 30, 50):
        e = torch.zeros_like(x)
        e[1, 2, 0, i] = 1.0
        diff = (radar.rotary(rope, x + e, 777).double() - fwd.double()).mul(y.double()).sum()
        lim = 8 * 2.0 ** -24 * float((x[1, 2, 0].abs().max() + 1) * y[1, 2, 0].abs().max()) * rope.mscale * 8
        assert abs(float(diff) - float(back[1, 2, 0, i])) <= lim


def _cache(cfg, fill=9.0, pinned=False):
    shape = (cfg.batch, cfg.n_kv_heads, cfg.capacity, cfg.head_dim)
    if pinned:
        return [torch.full(shape, fill, dtype=cfg.dtype).pin_memory() for _ in range(2)]
    return [torch.full(shape, fill, dtype=cfg.dtype, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("where", ["device", "host"])
@pytest.mark.parametrize("dtype", list(DT))
def test_fill(dtype, where):
    B, T, Hq, Hkv, d, cap = 2, 37, 8, 2, 128, 50
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, cap, DT[dtype])
    rope = _rope(64, False, "linear", 2.0)
    qkv = torch.randn(B, T, Hq + 2 * Hkv, d, device="cuda").to(DT[dtype])
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    K, V = _cache(cfg, pinned=where == "host")
    out = radar.rotary_fill(cfg, rope, K, V, k, v, 11, q=q)
    torch.cuda.synchronize()
    _close(out, *_ref(q, rope, _grid(11, B, T)))
    ref, tol = _ref(k, rope, _grid(11, B, T))
    _close(K[:, :, 11:48].transpose(1, 2), ref, tol)
    assert torch.equal(V[:, :, 11:48].transpose(1, 2).cpu(), v.cpu())
    for x in (K, V):
        assert bool((x[:, :, :11] == 9.0).all()) and bool((x[:, :, 48:] == 9.0).all())


def test_fill_ragged():
    """Rows and lengths of each sequence; rows outside the capacity are skipped,
    also where a sequence begins before row 0."""
    B, T, Hkv, d, cap = 4, 6, 3, 64, 20
    cfg = radar.Config(B, Hkv, Hkv, d, 64, 16, 16, cap, torch.float32)
    rope = _rope(64, True)
    k, v = (torch.randn(B, T, Hkv, d, device="cuda") for _ in range(2))
    K, V = _cache(cfg)
    rows = torch.tensor([0, 17, 9, -2], device="cuda")
    lens = torch.tensor([6, 6, 0, 4], device="cuda")
    pos = torch.tensor([100, 200, 300, 400], device="cuda")
    assert radar.rotary_fill(cfg, rope, K, V, k, v, rows, pos=pos, lens=lens) is None
    ref, tol = _ref(k, rope, pos.cpu()[:, None] + torch.arange(T))
    want = {(0, i): i for i in range(6)} | {(1, 17 + i): i for i in range(3)} | {(3, i - 2): i for i in (2, 3)}
    for b in range(B):
        for r in range(cap):
            if (b, r) in want:
                t = want[b, r]
                _close(K[b, :, r], ref[b, t], tol[b, t])
                assert torch.equal(V[b, :, r], v[b, t])
            else:
                assert bool((K[b, :, r] == 9.0).all()) and bool((V[b, :, r] == 9.0).all())


def test_one_token_of_each_sequence():
    """The decode form: [B][Hkv][d] rows at rows of their own."""
    cfg = radar.Config(3, 4, 2, 128, 64, 16, 16, 40, torch.bfloat16)
    rope = _rope(128)
    q = torch.randn(3, 4, 128, device="cuda").bfloat16()
    k, v = (torch.randn(3, 2, 128, device="cuda").bfloat16() for _ in range(2))
    K, V = _cache(cfg)
    rows = torch.tensor([0, 39, 7], device="cuda")
    out = radar.rotary_fill(cfg, rope, K, V, k, v, rows, q=q)
    _close(out[:, None], *_ref(q[:, None], rope, rows.cpu()[:, None]))
    ref, tol = _ref(k[:, None], rope, rows.cpu()[:, None])
    at = torch.arange(3, device="cuda")
    _close(K[at, :, rows], ref[:, 0], tol[:, 0])
    assert torch.equal(V[at, :, rows], v)
    assert int((K != 9.0).any(-1).sum()) == 6


def test_empty_calls():
    cfg = radar.Config(2, 4, 2, 64, 64, 16, 16, 40, torch.float32)
    rope, x = _rope(64), torch.empty(2, 0, 4, 64, device="cuda")
    assert radar.rotary(rope, x, 0).shape == x.shape
    K, V = _cache(cfg)
    e = torch.empty(2, 0, 2, 64, device="cuda")
    assert radar.rotary_fill(cfg, rope, K, V, e, e, 40) is None


def test_stream_and_graph():
    """On a stream of the caller's, and captured: every replay reads the
    positions and rows that the device arrays hold then."""
    cfg = radar.Config(2, 4, 2, 64, 64, 16, 16, 64, torch.float32)
    rope = _rope(64)
    q, k, v = (torch.randn(2, h, 64, device="cuda") for h in (4, 2, 2))
    K, V = _cache(cfg)
    rows = torch.tensor([3, 5], device="cuda")
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        radar.rotary_fill(cfg, rope, K, V, k, v, rows, q=q, q_out=out)
    s.synchronize()
    _close(out[:, None], *_ref(q[:, None], rope, rows.cpu()[:, None]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        radar.rotary_fill(cfg, rope, K, V, k, v, rows, q=q, q_out=out)
    for rep in range(3):
        rows += 7
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        _close(out[:, None], *_ref(q[:, None], rope, rows.cpu()[:, None]))
        ref, tol = _ref(k[:, None], rope, rows.cpu()[:, None])
        _close(K[torch.arange(2, device="cuda"), :, rows], ref[:, 0], tol[:, 0])


def test_refusals():
    cfg = radar.Config(2, 4, 2, 64, 64, 16, 16, 64, torch.float32)
    rope = _rope(64)
    x = torch.randn(2, 3, 4, 64, device="cuda")
    with pytest.raises(ValueError, match="16 bytes"):
        radar.rotary(rope, torch.randn(2, 3, 4, 65, device="cuda")[..., :64], 0)
    with pytest.raises(ValueError, match="16 bytes"):
        radar.rotary(rope, torch.randn(2, 3, 64, 4, device="cuda").transpose(2, 3), 0)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        radar.rotary(rope, x.half(), 0)
    with pytest.raises(ValueError, match="shape"):
        radar.rotary(rope, x, 0, out=x[:, :2])
    with pytest.raises(ValueError, match="share a place"):
        radar.rotary(rope, x, 0, out=x[:, :1].expand(2, 3, 4, 64))
    with pytest.raises(ValueError, match="other strides"):
        radar.rotary(rope, x, 0, out=x.as_strided((2, 3, 4, 64), (768, 64, 192, 1)))
    with pytest.raises(ValueError, match="pos"):
        radar.rotary(rope, x, torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="pos"):
        radar.rotary(rope, x, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(radar.RadarError, match="invalid argument"):
        radar.rotary(_rope(128), x, 0)                   # more rotated dims than dims
    with pytest.raises(radar.RadarError, match="instantiated"):
        radar.rotary(_rope(8), torch.randn(1, 1, 1, 24, device="cuda"), 0)
    K, V = _cache(cfg)
    k = torch.randn(2, 3, 2, 64, device="cuda")
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.rotary_fill(cfg, rope, K, V, k, k, 62)
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.rotary_fill(cfg, rope, K, V, k, k, -1)
    with pytest.raises(ValueError, match="n_kv_heads"):
        radar.rotary_fill(cfg, rope, K, V, x, x, 0)
    with pytest.raises(ValueError, match="q_out"):
        radar.rotary_fill(cfg, rope, K, V, k, k, 0, q_out=x)
    torch.cuda.synchronize()
    assert bool((K == 9.0).all()) and bool((V == 9.0).all())
    assert math.isfinite(float(x.sum()))
