"""Attention over a shared prefix and attention that accumulates the rows'
weights, on the GPU against 64 bits (tolerances: _cache_ref.py). Rows behind
the lengths hold NaN: nothing of them may reach a result."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
import _cache_ref as R  # noqa: E402
from test_gpu_canaries import Guarded  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DTYPES = pytest.mark.parametrize("dtype", list(DT))


def _cfg(B, Hq, Hkv, d, cap, dtype):
    return radar.Config(B, Hq, Hkv, d, 64, 16, 16, cap, DT[dtype])


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(DT[dtype])


def _inputs(B, Hq, Hkv, d, P, t, lens, dtype, seed=0, qscale=2.0, spare=3):
    """q, Kp, Vp, K, V: filled to P and lens, NaN behind."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = _randn(g, B, Hq, d, dtype=dtype, scale=qscale)
    Kp, Vp = (_randn(g, Hkv, P + spare, d, dtype=dtype) for _ in range(2))
    K, V = (_randn(g, B, Hkv, max(t, 1) + spare, d, dtype=dtype) for _ in range(2))
    for x in (Kp, Vp):
        x[:, P:] = float("nan")
    for b in range(B):
        n = t if lens is None else lens[b]
        for x in (K, V):
            x[b, :, max(0, n):] = float("nan")
    return q, Kp, Vp, K, V


def _check_prefix(out, q, Kp, Vp, P, K, V, t, lens, dtype, B, Hq, Hkv):
    G = Hq // Hkv
    assert not bool(out.isnan().any())
    for b in range(B):
        n = t if lens is None else lens[b]
        for h in range(Hkv):
            k = torch.cat([Kp[h, :P], K[b, h, :n]])
            v = torch.cat([Vp[h, :P], V[b, h, :n]])
            got = out[b, h * G:(h + 1) * G].double()
            if k.shape[0] == 0:
                assert bool((got == 0).all())
                continue
            # (a partial of the prefix has B G rows, of a sequence's own rows G)
            ref, tol, _, _ = R.attend(q[b, h * G:(h + 1) * G], k, v, DT[dtype], B * G)
            assert bool(((got - ref).abs() <= tol).all()), (b, h, float(((got - ref).abs() / tol).max()))


PREFIX = [  # B, Hq, Hkv, d, P, t, lens
    (1, 1, 1, 64, 1, 0, None),                 # one row
    (1, 8, 1, 128, 127, 1, None),              # a tile that ends early, one own row
    (2, 2, 2, 64, 0, 33, None),                # no prefix
    (3, 8, 2, 64, 128, 5, [5, 0, 3]),          # a whole tile, an empty sequence
    (3, 4, 4, 128, 0, 70, [0, 70, 1]),         # nothing at all to attend
    (4, 32, 4, 128, 129, 0, None),             # 32 rows a kv head
    (16, 2, 2, 128, 300, 140, None),           # 16 rows
    (17, 2, 2, 64, 300, 140, None),            # 17
    (5, 16, 2, 128, 1000, 77, [77, 0, 1, 64, 65]),   # 40
    (16, 32, 8, 64, 260, 130, None),           # 64
    (17, 8, 2, 128, 193, 20, None),            # 68
    (40, 64, 8, 64, 700, 200, "ragged"),       # 320: row tiles that end early
    (100, 8, 8, 128, 64, 300, "ragged"),       # own rows outweigh the prefix
    (2, 16, 2, 128, 40001, 9, None),           # many splits
    (33, 4, 1, 64, 20011, 1500, "ragged"),
]


@DTYPES
@pytest.mark.parametrize("B,Hq,Hkv,d,P,t,lens", PREFIX)
def test_prefix(B, Hq, Hkv, d, P, t, lens, dtype):
    print(f"[case] prefix B{B} Hq{Hq}/{Hkv} d{d} P{P} t{t} {lens} {dtype}", flush=True)
    if lens == "ragged":
        lens = [(t * b) // (B - 1) for b in range(B)]
    q, Kp, Vp, K, V = _inputs(B, Hq, Hkv, d, P, t, lens, dtype, seed=P + t)
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    L = None if lens is None else torch.tensor(lens, device="cuda")
    ws = Guarded((radar.attend_prefix_workspace_bytes(cfg, P, t),), torch.uint8)
    out = Guarded(q.shape, q.dtype)
    got = radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, t, out=out.t, lens=L, workspace=ws.t)
    torch.cuda.synchronize()
    assert ws.intact() and out.intact()
    _check_prefix(got, q, Kp, Vp, P, K, V, t, lens, dtype, B, Hq, Hkv)
    again = radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, t, lens=L)
    assert torch.equal(got, again)


@DTYPES
@pytest.mark.parametrize("P,t", [(1, 0), (0, 1), (64, 64), (65, 128), (512, 128), (512, 129),
                                 (640, 0), (0, 640), (0, 641), (33, 500), (192, 1), (129, 63)])
def test_prefix_few_rows(P, t, dtype):
    """Sizes on both sides of where one workgroup attends all of a pair's rows, with
    lengths down to none and two that are none."""
    lens = [t, t // 2, 0, 1 if t else 0, t + 1, -1]
    q, Kp, Vp, K, V = _inputs(6, 4, 2, 128, P, t, [min(max(n, 0), t) for n in lens], dtype, seed=P)
    cfg = _cfg(6, 4, 2, 128, K.shape[2], dtype)
    out = Guarded(q.shape, q.dtype)
    radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, t, out=out.t, lens=torch.tensor(lens, device="cuda"))
    torch.cuda.synchronize()
    assert out.intact() and bool(out.t[4:].isnan().all())
    _check_prefix(out.t[:4], q[:4], Kp, Vp, P, K[:4], V[:4], t, lens[:4], dtype, 4, 4, 2)


@DTYPES
def test_prefix_more_pairs_than_slots(dtype):
    q, Kp, Vp, K, V = _inputs(520, 2, 1, 64, 40, 9, None, dtype)
    cfg = _cfg(520, 2, 1, 64, K.shape[2], dtype)
    out = radar.attend_prefix(cfg, q, Kp, Vp, 40, K, V, 9)
    _check_prefix(out, q, Kp, Vp, 40, K, V, 9, None, dtype, 520, 2, 1)


@DTYPES
@pytest.mark.parametrize("B,G", [(16, 2), (33, 1), (60, 1), (17, 4), (64, 2), (33, 4), (193, 1), (40, 8)])
def test_prefix_row_tiles(B, G, dtype):
    """Query rows of a kv head around what one workgroup holds."""
    q, Kp, Vp, K, V = _inputs(B, G, 1, 64, 1000, 20, None, dtype, seed=B)
    cfg = _cfg(B, G, 1, 64, K.shape[2], dtype)
    out = radar.attend_prefix(cfg, q, Kp, Vp, 1000, K, V, 20)
    _check_prefix(out, q, Kp, Vp, 1000, K, V, 20, None, dtype, B, G, 1)


@DTYPES
@pytest.mark.parametrize("B", [1, 20])
def test_prefix_sharp_and_flat(B, dtype):
    """Logits of some hundreds (one row takes all) and all equal."""
    for qscale in (60.0, 0.0):
        q, Kp, Vp, K, V = _inputs(B, 4, 2, 128, 333, 50, None, dtype, qscale=qscale)
        cfg = _cfg(B, 4, 2, 128, K.shape[2], dtype)
        out = radar.attend_prefix(cfg, q, Kp, Vp, 333, K, V, 50)
        _check_prefix(out, q, Kp, Vp, 333, K, V, 50, None, dtype, B, 4, 2)


@DTYPES
def test_prefix_invalid_lengths(dtype):
    lens = [4, -1, 8, 9, 0]
    q, Kp, Vp, K, V = _inputs(5, 4, 2, 64, 100, 8, [4, 0, 8, 8, 0], dtype)
    cfg = _cfg(5, 4, 2, 64, K.shape[2], dtype)
    out = radar.attend_prefix(cfg, q, Kp, Vp, 100, K, V, 8, lens=torch.tensor(lens, device="cuda"))
    assert bool(out[[1, 3]].isnan().all())
    good = [0, 2, 4]
    _check_prefix(out[good], q[good], Kp, Vp, 100, K[good], V[good], 8, [4, 8, 0], dtype, 3, 4, 2)


@DTYPES
def test_prefix_workspace_of_the_largest(dtype):
    """One workspace for the largest call serves every smaller one."""
    B, Hq, Hkv, d = 6, 8, 2, 64
    cfg = _cfg(B, Hq, Hkv, d, 603, dtype)
    ws = radar.attend_prefix_workspace_bytes(cfg, 9000, 600)
    for P, t in ((9000, 600), (1, 600), (9000, 0), (130, 1), (4000, 300)):
        assert radar.attend_prefix_workspace_bytes(cfg, P, t) <= ws
        q, Kp, Vp, K, V = _inputs(B, Hq, Hkv, d, P, t, None, dtype)
        w = Guarded((ws,), torch.uint8)
        K2, V2 = (torch.full((B, Hkv, 603, d), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2))
        K2[:, :, :t], V2[:, :, :t] = K[:, :, :t], V[:, :, :t]
        out = radar.attend_prefix(cfg, q, Kp, Vp, P, K2, V2, t, workspace=w.t)
        torch.cuda.synchronize()
        assert w.intact()
        _check_prefix(out, q, Kp, Vp, P, K, V, t, None, dtype, B, Hq, Hkv)


def test_prefix_host_cache():
    """The sequences' rows in pinned host memory, the prefix too."""
    q, Kp, Vp, K, V = _inputs(3, 8, 2, 128, 200, 90, None, "bf16")
    cfg = _cfg(3, 8, 2, 128, K.shape[2], "bf16")
    want = radar.attend_prefix(cfg, q, Kp, Vp, 200, K, V, 90)
    host = [x.cpu().pin_memory() for x in (Kp, Vp, K, V)]
    got = radar.attend_prefix(cfg, q, host[0], host[1], 200, host[2], host[3], 90)
    assert torch.equal(got, want)


# ---- accumulated weights ---------------------------------------------------------
def _check_mass(out, mass, mass0, q, K, V, t, lens, dtype, B, Hq, Hkv):
    G = Hq // Hkv
    for b in range(B):
        n = t if lens is None else lens[b]
        for h in range(Hkv):
            ref, tol, w, wt = R.attend(q[b, h * G:(h + 1) * G], K[b, h, :n], V[b, h, :n], DT[dtype], G)
            got = out[b, h * G:(h + 1) * G].double()
            assert bool(((got - ref).abs() <= tol).all()), (b, h, float(((got - ref).abs() / tol).max()))
            want = mass0[b, h, :n].double() + w.sum(0)
            lim = wt.sum(0) + 16 * R.U * want.abs()
            err = (mass[b, h, :n].double() - want).abs()
            assert bool((err <= lim).all()), (b, h, float((err / lim).max()))
            assert torch.equal(mass[b, h, n:], mass0[b, h, n:])


MASS = [  # B, Hq, Hkv, d, t, lens
    (1, 1, 1, 64, 1, None), (1, 8, 1, 128, 31, None), (2, 4, 4, 64, 128, None),
    (2, 16, 2, 128, 129, [129, 1]), (3, 8, 4, 64, 2049, [2049, 2048, 5]),
    (1, 32, 8, 128, 30001, None), (6, 8, 8, 128, 700, [700, 3, 512, 513, 640, 1]),
]


@DTYPES
@pytest.mark.parametrize("B,Hq,Hkv,d,t,lens", MASS)
def test_accumulate(B, Hq, Hkv, d, t, lens, dtype):
    print(f"[case] accumulate B{B} Hq{Hq}/{Hkv} d{d} t{t} {lens} {dtype}", flush=True)
    q, _, _, K, V = _inputs(B, Hq, Hkv, d, 0, t, lens, dtype, seed=t)
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    L = None if lens is None else torch.tensor(lens, device="cuda")
    mass = Guarded((B, Hkv, cfg.capacity), torch.float32)
    mass.t.copy_(torch.rand(B, Hkv, cfg.capacity, device="cuda"))
    mass0 = mass.t.clone()
    ws = Guarded((radar.attend_accumulate_workspace_bytes(cfg, t),), torch.uint8)
    out = radar.attend_accumulate(cfg, q, K, V, mass.t, t, lens=L, workspace=ws.t)
    torch.cuda.synchronize()
    assert ws.intact() and mass.intact()
    _check_mass(out, mass.t, mass0, q, K, V, t, lens, dtype, B, Hq, Hkv)
    # the same inputs give the same bits
    again = mass0.clone()
    assert torch.equal(radar.attend_accumulate(cfg, q, K, V, again, t, lens=L), out)
    assert torch.equal(again, mass.t)


@DTYPES
def test_accumulate_sharp(dtype):
    q, _, _, K, V = _inputs(2, 4, 2, 128, 0, 400, None, dtype, qscale=60.0)
    cfg = _cfg(2, 4, 2, 128, K.shape[2], dtype)
    mass = radar.new_mass(cfg, "cuda")
    out = radar.attend_accumulate(cfg, q, K, V, mass, 400)
    _check_mass(out, mass, torch.zeros_like(mass), q, K, V, 400, None, dtype, 2, 4, 2)


def test_accumulate_invalid_lengths():
    lens = [5, 0, 9, -3, 8]
    q, _, _, K, V = _inputs(5, 4, 2, 64, 0, 8, [5, 0, 8, 0, 8], "f32")
    cfg = _cfg(5, 4, 2, 64, K.shape[2], "f32")
    mass = torch.rand(5, 2, cfg.capacity, device="cuda")
    before = mass.clone()
    out = radar.attend_accumulate(cfg, q, K, V, mass, 8, lens=torch.tensor(lens, device="cuda"))
    assert bool(out[[1, 2, 3]].isnan().all())
    assert torch.equal(mass[[1, 2, 3]], before[[1, 2, 3]])
    good = [0, 4]
    _check_mass(out[good], mass[good], before[good], q[good], K[good], V[good], 8, [5, 8], "f32", 2, 4, 2)


def test_accumulate_agrees_with_decode():
    """The same output as the decode that selects every segment, to both sides'
    roundings."""
    t = 700
    q, _, _, K, V = _inputs(2, 8, 2, 128, 0, t, None, "f32")
    cfg = radar.Config(2, 8, 2, 128, 64, 16, 16, K.shape[2], torch.float32)
    out = radar.attend_accumulate(cfg, q, K, V, radar.new_mass(cfg, "cuda"), t)
    every = radar.decode_exact(cfg, q, K, V, t, 64)
    _, tol, _, _ = R.attend(q[0, :4], K[0, 0, :t], V[0, 0, :t], torch.float32)
    assert float((out - every).abs().max()) <= 4 * float(tol.max())


# ---- streams, graphs ---------------------------------------------------------------
@pytest.mark.parametrize("op", ["prefix", "accumulate"])
def test_graph_replays(op):
    """Captured once, replayed with other inputs and lengths, eager work between:
    the eager result's bits every time."""
    B, Hq, Hkv, d, P, t = 4, 8, 2, 128, 500, 300
    q, Kp, Vp, K, V = _inputs(B, Hq, Hkv, d, P, t, None, "bf16")
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], "bf16")
    lens = torch.tensor([300, 2, 100, 299], device="cuda")
    out, mass = torch.empty_like(q), radar.new_mass(cfg, "cuda")
    ws = torch.empty(max(radar.attend_prefix_workspace_bytes(cfg, P, t),
                         radar.attend_accumulate_workspace_bytes(cfg, t)), dtype=torch.uint8, device="cuda")

    def call(out, mass, ws):
        if op == "prefix":
            radar.attend_prefix(cfg, q, Kp, Vp, P, K, V, t, out=out, lens=lens, workspace=ws)
        else:
            radar.attend_accumulate(cfg, q, K, V, mass, t, out=out, lens=lens, workspace=ws)

    call(out, mass, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, mass, ws)
    for rep in range(3):
        q.mul_(0.9)
        lens.copy_(torch.tensor([300 - 7 * rep, 1, 128, 129 + rep], device="cuda"))
        want, wmass = torch.empty_like(q), mass.clone()
        call(want, wmass, None)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        assert torch.equal(out, want) and torch.equal(mass, wmass), rep


def test_graph_of_a_short_call():
    """One launch, its output and workspace the graph's own."""
    q, Kp, Vp, K, V = _inputs(3, 8, 2, 128, 200, 80, None, "bf16")
    cfg = _cfg(3, 8, 2, 128, K.shape[2], "bf16")
    lens = torch.tensor([80, 0, 33], device="cuda")
    radar.attend_prefix(cfg, q, Kp, Vp, 200, K, V, 80, lens=lens)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = radar.attend_prefix(cfg, q, Kp, Vp, 200, K, V, 80, lens=lens)
    for rep in range(3):
        q.mul_(0.9)
        lens.copy_(torch.tensor([79 - rep, 1, 0], device="cuda"))
        want = radar.attend_prefix(cfg, q, Kp, Vp, 200, K, V, 80, lens=lens)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.randn(1 << 20, device="cuda").sum().item()
        assert torch.equal(out, want), rep


def test_two_streams():
    """Two calls at once on streams of their own, each with its workspace."""
    ins = [_inputs(4, 8, 2, 128, 3000, 300, None, "bf16", seed=i) for i in range(2)]
    cfg = _cfg(4, 8, 2, 128, ins[0][3].shape[2], "bf16")
    want = [radar.attend_prefix(cfg, q, Kp, Vp, 3000, K, V, 300) for q, Kp, Vp, K, V in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    outs = [torch.empty_like(x[0]) for x in ins]
    n = radar.attend_prefix_workspace_bytes(cfg, 3000, 300)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in ins]
    for rep in range(5):
        for s, o, w, (q, Kp, Vp, K, V) in zip(streams, outs, ws, ins):
            with torch.cuda.stream(s):
                radar.attend_prefix(cfg, q, Kp, Vp, 3000, K, V, 300, out=o, workspace=w)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_refusals():
    q, Kp, Vp, K, V = _inputs(2, 4, 2, 64, 50, 20, None, "f32")
    cfg = _cfg(2, 4, 2, 64, K.shape[2], "f32")
    mass = radar.new_mass(cfg, "cuda")
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.attend_prefix(cfg, q, Kp, Vp, Kp.shape[1] + 1, K, V, 20)
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.attend_prefix(cfg, q, Kp, Vp, 50, K, V, cfg.capacity + 1)
    with pytest.raises(radar.RadarError, match="workspace"):
        radar.attend_prefix(cfg, q, Kp, Vp, 50, K, V, 20,
                            workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="n_kv_heads"):
        radar.attend_prefix(cfg, q, Kp[:1], Vp[:1], 50, K, V, 20)
    with pytest.raises(ValueError, match="same number"):
        radar.attend_prefix(cfg, q, Kp, Vp[:, :51].contiguous(), 50, K, V, 20)
    with pytest.raises(ValueError, match="needed"):
        radar.attend_prefix(cfg, q, Kp, Vp, 50, t=20)
    with pytest.raises(ValueError, match="float32"):
        radar.attend_prefix(cfg, q.bfloat16(), Kp, Vp, 50, K, V, 20)
    with pytest.raises(ValueError, match="elements"):
        radar.attend_accumulate(cfg, q, K, V, mass[:, :, 1:].contiguous(), 20)
    with pytest.raises(radar.RadarError, match="capacity"):
        radar.attend_accumulate(cfg, q, K, V, mass, 0)
    with pytest.raises(ValueError, match="contiguous"):
        radar.attend_accumulate(cfg, q, K, V, mass.transpose(0, 1), 20)
    odd = radar.Config(2, 6, 2, 64, 64, 16, 16, K.shape[2], torch.float32)
    with pytest.raises(radar.RadarError, match="instantiated"):
        radar.attend_prefix(odd, torch.randn(2, 6, 64, device="cuda"), Kp, Vp, 50, K, V, 20,
                            workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert bool((mass == 0).all())
