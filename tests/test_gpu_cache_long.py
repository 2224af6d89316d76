"""The cache operators at sizes that take every loop of their kernels more than
once: blocks of several tiles at every width, hundreds of partials, calls that pass
the caches, long caches with special masses. Tolerances: _cache_ref.py and
test_gpu_rotary.py."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
import _cache_ref as R  # noqa: E402
from test_gpu_evict import _run as evict_and_check  # noqa: E402
from test_gpu_evict import _want as evicted  # noqa: E402
from test_gpu_prefix import DTYPES, _cfg, _check_mass, _check_prefix, _inputs  # noqa: E402
from test_gpu_rotary import DT, _rope  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu


# ---- attention: tiles of a block ---------------------------------------------------
# A block of the prefix has about Hkv row_tiles P / 512 rows, or twice as many, in
# tiles of 32 to 128: at least three here, the last one partial.
@DTYPES
@pytest.mark.parametrize("ramp", ["flat", "rising", "falling"])
@pytest.mark.parametrize("B,Hq,Hkv,d,P", [
    (4, 8, 2, 128, 60011),         # 16 query rows a kv head
    (8, 8, 2, 128, 60011),         # 32
    (16, 8, 2, 128, 60011),        # 64
    (16, 8, 2, 64, 60011),
    (32, 8, 2, 128, 60011),        # 128
    (32, 8, 2, 64, 60011),
    (33, 4, 1, 128, 60011),        # 132: a second row tile of four
    (128, 4, 1, 128, 30011),       # 512: four row tiles
])
def test_blocks_of_several_tiles(B, Hq, Hkv, d, P, ramp, dtype):
    """Keys that grow (or shrink) along the prefix: the running maximum moves on in
    the middle of a block, or never after its first tile."""
    print(f"[case] blocks B{B} Hq{Hq}/{Hkv} d{d} P{P} {ramp} {dtype}", flush=True)
    lens = [0, 5, 77] + [40] * (B - 3)
    q, Kp, Vp, K, V = _inputs(B, Hq, Hkv, d, P, 77, lens, dtype, seed=B)
    if ramp != "flat":
        f = torch.linspace(0.05, 4.0, Kp.shape[1], device="cuda")
        Kp *= (f if ramp == "rising" else f.flip(0))[:, None].to(Kp.dtype)
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    L = torch.tensor(lens, device="cuda")
    out = radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, 77, lens=L)
    some = sorted({0, 1, 2, B // 2, B - 1})      # (in 64 bits all would take long)
    G = Hq // Hkv
    for b in some:
        for h in range(Hkv):
            k, v = torch.cat([Kp[h, :P], K[b, h, :lens[b]]]), torch.cat([Vp[h, :P], V[b, h, :lens[b]]])
            ref, tol, _, _ = R.attend(q[b, h * G:(h + 1) * G], k, v, DT[dtype], B * G)
            err = (out[b, h * G:(h + 1) * G].double() - ref).abs()
            assert bool((err <= tol).all()), (b, h, float((err / tol).max()))
    assert torch.equal(out, radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, 77, lens=L))


# ---- attention: hundreds of partials of a head --------------------------------------
@DTYPES
@pytest.mark.parametrize("G,P,t,lens", [
    (1, 131072, 131072, None), (4, 131072, 70001, None), (1, 0, 131072, None),
    (4, 131072, 131072, [131070]), (8, 131072, 131072, [3])])
def test_prefix_of_one_long_sequence(G, P, t, lens, dtype):
    print(f"[case] long prefix G{G} P{P} t{t} {lens} {dtype}", flush=True)
    q, Kp, Vp, K, V = _inputs(1, G, 1, 64, P, t, lens, dtype, seed=G)
    cfg = _cfg(1, G, 1, 64, K.shape[2], dtype)
    L = None if lens is None else torch.tensor(lens, device="cuda")
    out = radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, t, lens=L)
    _check_prefix(out, q, Kp, Vp, P, K, V, t, lens, dtype, 1, G, 1)


@DTYPES
@pytest.mark.parametrize("G,t,lens", [(1, 131072, None), (4, 131072, None), (1, 131072, [131071]),
                                      (4, 70001, [69999]), (8, 131072, [100])])
def test_weights_of_one_long_sequence(G, t, lens, dtype):
    print(f"[case] long weights G{G} t{t} {lens} {dtype}", flush=True)
    q, _, _, K, V = _inputs(1, G, 1, 64, 0, t, lens, dtype, seed=t + G)
    cfg = _cfg(1, G, 1, 64, K.shape[2], dtype)
    L = None if lens is None else torch.tensor(lens, device="cuda")
    mass0 = torch.rand(1, 1, cfg.capacity, device="cuda") * 1e-4
    mass = mass0.clone()
    out = radar.attend_accumulate(cfg, q, K, V, mass, t, lens=L)
    _check_mass(out, mass, mass0, q, K, V, t, lens, dtype, 1, G, 1)


# ---- rotary: a prompt on its way into the cache, past the caches ------------------
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,T", [("bf16", 9000), ("f32", 5000)])
def test_large_fills(dtype, T, inter, ragged):
    """More than 256 MB read and written, the rotated queries in place: the bits of
    calls that are not."""
    B, Hq, Hkv, d, row = 2, 32, 8, 128, 11
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, T + 50, DT[dtype])
    rope = _rope(96 if inter else 128, inter)
    size = torch.finfo(DT[dtype]).bits // 8
    assert 2 * B * T * (Hq + 2 * Hkv) * d * size > 256 << 20
    qkv = torch.randn(B, T, Hq + 2 * Hkv, d, device="cuda").to(DT[dtype])
    q, k, v = qkv.split([Hq, Hkv, Hkv], 2)
    was = qkv.clone()
    lens = torch.tensor([T, T // 3], device="cuda") if ragged else None
    n = lens.tolist() if ragged else [T, T]
    K, V, K2, V2 = (torch.full((B, Hkv, T + 50, d), 9.0, dtype=DT[dtype], device="cuda") for _ in range(4))
    radar.rotary_fill(cfg, rope, K, V, k, v, row, q=q, q_out=q, lens=lens)
    q2, k2, v2 = was.split([Hq, Hkv, Hkv], 2)
    for t in range(0, T, 1000):
        at = slice(t, t + 1000)
        kw = {} if lens is None else dict(lens=(lens - t).clamp(0, 1000))
        radar.rotary_fill(cfg, rope, K2, V2, k2[:, at], v2[:, at], row + t, q=q2[:, at], q_out=q2[:, at], **kw)
    assert torch.equal(qkv, was)
    assert torch.equal(K, K2) and torch.equal(V, V2)
    for b in range(B):
        assert bool((K[b, :, row + n[b]:] == 9.0).all()) and bool((V[b, :, :row] == 9.0).all())
        assert torch.equal(V[b, :, row:row + n[b]].transpose(0, 1), v[b, :n[b]])


# ---- eviction of long caches ---------------------------------------------------------
@pytest.mark.parametrize("kind", ["signed", "special"])
def test_special_masses_across_slices(kind):
    def masses(B, Hkv, cap, g):
        if kind == "signed":                      # -0 equals 0
            return torch.randint(-2, 3, (B, Hkv, cap), generator=g).float() * 0.0 + \
                torch.randint(0, 2, (B, Hkv, cap), generator=g).float().neg()
        v = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-42, 3e38, 1.0])
        return v[torch.randint(0, 8, (B, Hkv, cap), generator=g)]

    for heavy in (1, 37, 5000, 17000):
        evict_and_check(2, 1, 64, 18001, 4, heavy, 50, [18001, 17999], "bf16", masses=masses)


def test_invalid_lengths_across_slices():
    evict_and_check(6, 1, 64, 18001, 4, 5000, 50, [18001, 18002, -1, 9000, 0, 5054], "bf16")
    evict_and_check(6, 1, 64, 18001, 4, 5000, 50, [17000, 1 << 40, -(1 << 40), 8192, 5055, 1], "f32", alias=True)


def test_graph_replays_across_slices():
    B, Hkv, d, t = 2, 2, 64, 18001
    cfg = radar.Config(B, Hkv, Hkv, d, 64, 16, 16, t, torch.bfloat16, 4)
    K0, V0 = (torch.randn(B, Hkv, t, d, device="cuda").bfloat16() for _ in range(2))
    K, V, mass = K0.clone(), V0.clone(), torch.rand(B, Hkv, t, device="cuda")
    lens = torch.tensor([18001, 9000], device="cuda")
    new, kept = torch.empty_like(lens), torch.empty(B, Hkv, 5104, dtype=torch.int32, device="cuda")
    ws = torch.empty(radar.evict_workspace_bytes(cfg, t, 5000, 100), dtype=torch.uint8, device="cuda")

    def call():
        radar.evict(cfg, K, V, mass, t, 5000, 100, lens=lens, new_lens=new, kept=kept, workspace=ws)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(3):
        K.copy_(K0)
        V.copy_(V0)
        m0 = torch.rand(B, Hkv, t, device="cuda")
        mass.copy_(m0)
        lens.copy_(torch.tensor([18000 - rep, 4000 + 3000 * rep], device="cuda"))
        w = evicted(K0, V0, m0, t, lens.tolist(), 4, 5000, 100)
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        for got, ref in zip((K, V, mass, kept), w):
            assert torch.equal(got.cpu(), ref), rep
        assert new.tolist() == w[4]
