"""Eviction on the GPU against the definition: which rows stay (ties to the
lower row), their bits in K, V and the masses, and everything that has to be
left as it was. Nothing is rounded, so everything has to be equal."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from test_gpu_canaries import Guarded  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _bits(x):
    return x.view(torch.int16 if x.element_size() == 2 else torch.int32)


def _rows_kept(mass, n, sink, heavy, recent):
    """Rows of one head that stay, from its masses (a CPU list of floats)."""
    if n <= sink + heavy + recent:
        return list(range(n))
    key = lambda i: (mass[i] == mass[i], -mass[i] if mass[i] == mass[i] else 0.0, i)  # noqa: E731
    best = sorted(range(sink, n - recent), key=key)[:heavy]
    return list(range(sink)) + sorted(best) + list(range(n - recent, n))


def _want(K, V, mass, t, lens, sink, heavy, recent):
    K, V, mass = K.cpu().clone(), V.cpu().clone(), mass.cpu().clone()
    B, Hkv = mass.shape[:2]
    n = sink + heavy + recent
    kept = torch.full((B, Hkv, min(n, t)), -1, dtype=torch.int32)
    new = []
    for b in range(B):
        L = t if lens is None else lens[b]
        ok = 0 <= L <= t
        new.append(min(L, n) if ok else L)
        for h in range(Hkv):
            if not ok:
                continue
            at = _rows_kept(mass[b, h, :L].tolist(), L, sink, heavy, recent)
            kept[b, h, :len(at)] = torch.tensor(at, dtype=torch.int32)
            if L > n:
                k, v, m = K[b, h, at].clone(), V[b, h, at].clone(), mass[b, h, at].clone()
                K[b, h, :n], V[b, h, :n], mass[b, h, :n] = k, v, m
                mass[b, h, n:L] = 0
    return K, V, mass, kept, new


def _run(B, Hkv, d, t, sink, heavy, recent, lens=None, dtype="bf16", masses=None, spare=5, alias=False,
         pinned=False, seed=0):
    print(f"[case] evict B{B} Hkv{Hkv} d{d} t{t} {sink}+{heavy}+{recent} {lens} {dtype}", flush=True)
    g = torch.Generator().manual_seed(seed)
    cap = t + spare
    cfg = radar.Config(B, Hkv, Hkv, d, 64, 16, 16, cap, DT[dtype], sink)
    K, V = (torch.randn(B, Hkv, cap, d, generator=g).to(DT[dtype]) for _ in range(2))
    if masses is None:
        mass = torch.exp(3 * torch.randn(B, Hkv, cap, generator=g))
        mass *= torch.rand(B, Hkv, cap, generator=g) > 0.2
    else:
        mass = masses(B, Hkv, cap, g)
    want = _want(K, V, mass, t, lens, sink, heavy, recent)
    if pinned:
        Kd, Vd = K.pin_memory(), V.pin_memory()
    else:
        gk, gv = Guarded(K.shape, K.dtype), Guarded(V.shape, V.dtype)
        gk.t.copy_(K)
        gv.t.copy_(V)
        Kd, Vd = gk.t, gv.t
    gm = Guarded(mass.shape, torch.float32, init=mass)
    kept = Guarded(tuple(want[3].shape), torch.int32)
    ws = Guarded((radar.evict_workspace_bytes(cfg, t, heavy, recent),), torch.uint8)
    L = None if lens is None else torch.tensor(lens, device="cuda")
    new = L if alias else torch.empty(B, dtype=torch.int64, device="cuda")
    bound = radar.evict(cfg, Kd, Vd, gm.t, t, heavy, recent, lens=L, new_lens=new, kept=kept.t,
                        workspace=ws.t)
    torch.cuda.synchronize()
    assert bound == min(t, sink + heavy + recent)
    assert gm.intact() and ws.intact() and kept.intact()
    assert pinned or (gk.intact() and gv.intact())
    assert new.tolist() == want[4]
    if kept.t.numel():
        assert torch.equal(kept.t.cpu(), want[3])
    for got, ref in zip((Kd, Vd, gm.t), want):
        assert torch.equal(_bits(got.cpu()), _bits(ref))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,Hkv,d,t,sink,heavy,recent,lens", [
    (1, 1, 64, 1, 0, 0, 0, None),                 # nothing stays
    (1, 1, 64, 2, 0, 1, 0, None),
    (2, 3, 128, 100, 4, 20, 10, None),
    (2, 2, 64, 100, 0, 0, 7, None),               # a plain window
    (2, 2, 64, 100, 3, 0, 0, None),               # the sinks alone
    (1, 2, 128, 100, 0, 99, 0, None),             # one row leaves
    (1, 2, 128, 100, 4, 90, 6, None),             # none does
    (1, 2, 128, 100, 4, 900, 60, None),           # more room than rows
    (3, 2, 128, 3000, 4, 1500, 333, [3000, 1837, 1838]),
    (4, 1, 64, 1025, 1, 511, 1, [1025, 0, 1, 600]),
    (1, 2, 128, 20011, 4, 9001, 2001, None),
    (3, 2, 64, 50, 2, 10, 5, [51, -1, 40]),       # lengths that are none
])
def test_evict(B, Hkv, d, t, sink, heavy, recent, lens, dtype):
    _run(B, Hkv, d, t, sink, heavy, recent, lens, dtype)


@pytest.mark.parametrize("kind", ["zero", "one", "few", "signed", "special", "near"])
def test_ties_and_special_masses(kind):
    def masses(B, Hkv, cap, g):
        if kind == "zero":
            return torch.zeros(B, Hkv, cap)
        if kind == "one":
            return torch.full((B, Hkv, cap), 1.5)
        if kind == "few":                         # many equal ones
            return torch.randint(0, 3, (B, Hkv, cap), generator=g).float()
        if kind == "signed":                      # -0 equals 0
            return torch.randint(-2, 3, (B, Hkv, cap), generator=g).float() * 0.0 + \
                torch.randint(0, 2, (B, Hkv, cap), generator=g).float().neg()
        if kind == "near":                        # neighbours in the last bit
            x = torch.randint(0, 40, (B, Hkv, cap), generator=g, dtype=torch.int32) + 0x3f800000
            return x.view(torch.float32)
        v = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-42, 3e38, 1.0])
        return v[torch.randint(0, 8, (B, Hkv, cap), generator=g)]

    for heavy in (1, 37, 1000, 1900):
        _run(2, 2, 64, 2100, 4, heavy, 50, [2100, 2003], "f32", masses=masses)


@pytest.mark.parametrize("t", [8191, 8192, 8193, 16385])
def test_around_a_slice(t):
    _run(2, 2, 64, t, 4, t // 3, 100, [t, t - 1], "bf16")


def test_slices_of_ragged_sequences():
    """Sequences that end in the first slice, at a slice's end, behind it."""
    for heavy, recent in ((3000, 900), (0, 40), (5, 0), (0, 0)):
        _run(5, 1, 64, 20000, 4, heavy, recent, [20000, 4500, 8192, 16384, 8193], "bf16")
    _run(2, 1, 64, 9000, 0, 0, 0, [9000, 8000], "f32")


@pytest.mark.parametrize("kind", ["zero", "few", "near"])
def test_ties_across_slices(kind):
    def masses(B, Hkv, cap, g):
        if kind == "zero":
            return torch.zeros(B, Hkv, cap)
        if kind == "few":
            return torch.randint(0, 3, (B, Hkv, cap), generator=g).float()
        x = torch.randint(0, 3000, (B, Hkv, cap), generator=g, dtype=torch.int32) + 0x3f800000
        return x.view(torch.float32)

    for heavy in (1, 5000, 17000):
        _run(1, 2, 64, 18001, 4, heavy, 50, None, "bf16", masses=masses)


def test_long_cache():
    _run(1, 1, 64, 270001, 4, 100000, 5000, None, "bf16")          # slices of two steps
    _run(1, 1, 64, 131077, 4, 60000, 5000, None, "bf16")


@pytest.mark.parametrize("d,dtype,t", [(64, "bf16", 27000), (128, "bf16", 13500), (128, "f32", 6900)])
def test_large_move(d, dtype, t):
    """More than 768 MB moved, whose stores pass the caches by."""
    cfg = radar.Config(8, 8, 8, d, 64, 16, 16, t, DT[dtype], 4)
    K, V = (torch.randn(8, 8, t, d, device="cuda").to(DT[dtype]) for _ in range(2))
    mass = torch.rand(8, 8, t, device="cuda")
    K0, V0, mass0 = K.clone(), V.clone(), mass.clone()
    heavy = t - 600
    kept = torch.empty(8, 8, heavy + 104, dtype=torch.int32, device="cuda")
    n = radar.evict(cfg, K, V, mass, t, heavy, 100, kept=kept)
    assert n == heavy + 104 and 4 * n * 64 * d * K.element_size() > 768 << 20
    at = kept.long()
    assert bool((at[..., 1:] > at[..., :-1]).all())
    rows = at[..., None].expand(-1, -1, -1, d)
    assert torch.equal(K[:, :, :n], K0.gather(2, rows)) and torch.equal(V[:, :, :n], V0.gather(2, rows))
    assert torch.equal(K[:, :, n:], K0[:, :, n:]) and torch.equal(V[:, :, n:], V0[:, :, n:])
    assert torch.equal(mass[..., :n], mass0.gather(2, at)) and not bool(mass[..., n:].any())


def test_new_lengths_in_place_of_the_old():
    _run(5, 4, 64, 400, 2, 100, 30, [400, 133, 132, 7, 401], "bf16", alias=True)


def test_host_cache():
    _run(2, 2, 128, 900, 4, 300, 99, [900, 500], "bf16", pinned=True)


def test_twice():
    """A second eviction of what the first left; n rows of n are left alone."""
    cfg = radar.Config(1, 2, 2, 64, 64, 16, 16, 600, torch.float32, 4)
    K, V = (torch.randn(1, 2, 600, 64, device="cuda") for _ in range(2))
    mass = torch.rand(1, 2, 600, device="cuda")
    K0, V0, m0 = K.cpu(), V.cpu(), mass.cpu()
    n = radar.evict(cfg, K, V, mass, 600, 300, 50)
    w = _want(K0, V0, m0, 600, None, 4, 300, 50)
    n2 = radar.evict(cfg, K, V, mass, n, 100, 20)
    w = _want(w[0], w[1], w[2], n, None, 4, 100, 20)
    assert (n, n2) == (354, 124)
    for got, ref in zip((K, V, mass), w):
        assert torch.equal(got.cpu(), ref)
    radar.evict(cfg, K, V, mass, n2, 100, 20)
    for got, ref in zip((K, V, mass), w):
        assert torch.equal(got.cpu(), ref)


def test_graph_replays():
    B, Hkv, d, t = 2, 2, 128, 1500
    cfg = radar.Config(B, Hkv, Hkv, d, 64, 16, 16, t, torch.bfloat16, 4)
    K0, V0 = (torch.randn(B, Hkv, t, d, device="cuda").bfloat16() for _ in range(2))
    K, V, mass = K0.clone(), V0.clone(), torch.rand(B, Hkv, t, device="cuda")
    lens = torch.tensor([1500, 900], device="cuda")
    ws = torch.empty(radar.evict_workspace_bytes(cfg, t, 500, 100), dtype=torch.uint8, device="cuda")
    radar.evict(cfg, K, V, mass, t, 500, 100, lens=lens, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        radar.evict(cfg, K, V, mass, t, 500, 100, lens=lens, workspace=ws)
    for rep in range(3):
        K.copy_(K0)
        V.copy_(V0)
        m0 = torch.rand(B, Hkv, t, device="cuda")
        mass.copy_(m0)
        lens.copy_(torch.tensor([1400 - rep, 700 + 300 * rep], device="cuda"))
        w = _want(K0, V0, m0, t, lens.tolist(), 4, 500, 100)
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        for got, ref in zip((K, V, mass), w):
            assert torch.equal(got.cpu(), ref), rep


def test_refusals():
    cfg = radar.Config(1, 2, 2, 64, 64, 16, 16, 100, torch.float32, 4)
    K, V = (torch.randn(1, 2, 100, 64, device="cuda") for _ in range(2))
    mass = torch.rand(1, 2, 100, device="cuda")
    before = [x.clone() for x in (K, V, mass)]
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.evict(cfg, K, V, mass, 101, 10, 10)
    with pytest.raises(radar.RadarError, match="invalid"):
        radar.evict(cfg, K, V, mass, 100, -1, 10)
    with pytest.raises(radar.RadarError, match="instantiated"):
        radar.evict(cfg, K, V, mass, 100, 1 << 31, 10)
    with pytest.raises(radar.RadarError, match="workspace"):
        radar.evict(cfg, K, V, mass, 100, 10, 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="kept"):
        radar.evict(cfg, K, V, mass, 100, 10, 10, kept=torch.empty(1, 2, 23, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="int64"):
        radar.evict(cfg, K, V, mass, 100, 10, 10, lens=torch.tensor([50], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for x, y in zip((K, V, mass), before):
        assert torch.equal(x, y)
