"""Attention of drafted tokens over the cache, on the GPU against 64 bits
(tolerances: _cache_ref.py). Rows that nobody attends hold NaN, and so do rows of
other branches where a test says so: nothing of them may reach a result."""
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


def _tree(N, seed, spread):
    """Parents drawn from the `spread` nodes before (0: a chain, None: all roots)."""
    if spread is None:
        return [-1] * N
    r = torch.Generator().manual_seed(seed)
    return [i - 1 - int(torch.randint(0, min(i, spread) + 1, (1,), generator=r)) for i in range(N)]


def _above(parent, m):
    """Each node's own and the nodes above it, None where the parents leave the tree."""
    out = []
    for i in range(m):
        seen, p = [i], parent[i]
        while p >= 0 and p < seen[-1]:
            seen.append(p)
            p = parent[p]
        out.append(sorted(seen) if p == -1 else None)
    return out


def _inputs(B, Hq, Hkv, d, t, N, lens, counts, dtype, seed=0, qscale=2.0, spare=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    q = (torch.randn(B, N, Hq, d, generator=g, device="cuda") * qscale).to(dt)
    K, V = (torch.randn(B, Hkv, t + N + spare, d, generator=g, device="cuda").to(dt) for _ in range(2))
    for b in range(B):
        n = max(0, lens[b]) + max(0, counts[b])
        K[b, :, n:], V[b, :, n:] = float("nan"), float("nan")
    return q, K, V


def _check(out, q, K, V, parents, lens, counts, dtype, Hkv, worst=None):
    B, N, Hq, d = q.shape
    G = Hq // Hkv
    for b in range(B):
        above = _above(parents[b], counts[b])
        for i, seen in enumerate(above):
            rows = list(range(lens[b])) if lens[b] < 0 else None
            assert rows is None
            for h in range(Hkv):
                got = out[b, i, h * G:(h + 1) * G].double()
                if seen is None:
                    assert bool(got.isnan().all()), (b, i)
                    continue
                k = torch.cat([K[b, h, :lens[b]], K[b, h, [lens[b] + j for j in seen]]])
                v = torch.cat([V[b, h, :lens[b]], V[b, h, [lens[b] + j for j in seen]]])
                ref, tol, _, _ = R.attend(q[b, i, h * G:(h + 1) * G], k, v, DT[dtype], N * G)
                bad = (got - ref).abs() > tol
                assert not bool(got.isnan().any()) and not bool(bad.any()), (
                    b, i, h, float(((got - ref).abs() / tol).max()))


def _run(B, Hq, Hkv, d, t, N, lens, counts, spread, dtype, shared=False, qscale=2.0, check=None, seed=None):
    print(f"[case] tree B{B} Hq{Hq}/{Hkv} d{d} t{t} N{N} spread{spread} {lens} {counts} {dtype}", flush=True)
    if lens == "ragged":
        lens = [t * ((7 * b) % B) // B for b in range(B)]
    if counts == "ragged":
        counts = [(5 * b) % (N + 1) for b in range(B)]
    L, C = lens or [t] * B, counts or [N] * B
    q, K, V = _inputs(B, Hq, Hkv, d, t, N, L, C, dtype, seed=t + N if seed is None else seed, qscale=qscale)
    parents = [_tree(N, 0 if shared else b, spread) for b in range(B)]
    P = None
    if spread != 0:
        P = torch.tensor(parents[0] if shared else parents, dtype=torch.int32, device="cuda")
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    ws = Guarded((radar.attend_tree_workspace_bytes(cfg, N, t),), torch.uint8)
    out = Guarded(q.shape, q.dtype, init=torch.full_like(q, 7.0))
    kw = dict(parent=P, lens=None if lens is None else torch.tensor(lens, device="cuda"),
              counts=None if counts is None else torch.tensor(counts, device="cuda"))
    radar.attend_tree(cfg, q, K, V, t, out=out.t, workspace=ws.t, **kw)
    torch.cuda.synchronize()
    assert ws.intact() and out.intact()
    for b in range(B):
        assert bool((out.t[b, C[b]:] == 7.0).all())
    _check(out.t, q, K, V, parents, L, C, dtype, Hkv)
    new = radar.attend_tree(cfg, q, K, V, t, **kw)
    for b in range(B):
        assert torch.equal(new[b, :C[b]], out.t[b, :C[b]]) and not bool(new[b, C[b]:].any())
    return q, K, V, out.t, cfg, kw


CASES = [  # B, Hq, Hkv, d, t, N, lens, counts, spread
    (1, 1, 1, 64, 0, 1, None, None, 0),                     # one row, itself
    (1, 8, 1, 128, 1, 1, None, None, None),                 # a decode step
    (2, 4, 4, 64, 0, 5, None, None, 2),                     # no cache
    (3, 8, 2, 64, 31, 7, [31, 0, 5], None, 3),
    (3, 4, 1, 128, 33, 8, [0, 33, 1], [8, 0, 1], 2),
    (1, 8, 2, 64, 500, 7, None, None, 3),
    (2, 2, 2, 128, 127, 16, None, [16, 3], 4),              # 16 rows
    (2, 2, 2, 128, 127, 17, None, [17, 3], 4),              # 17
    (1, 8, 2, 64, 300, 8, None, None, 2),                   # 32
    (2, 8, 2, 128, 700, 9, [699, 1], None, 3),              # 36
    (1, 16, 2, 128, 1000, 8, None, None, None),             # 64: all roots
    (2, 4, 1, 64, 260, 17, None, None, 5),                  # 68
    (1, 32, 8, 128, 4100, 32, None, None, 6),               # 128
    (2, 8, 8, 64, 3000, 33, [3000, 77], [20, 33], 6),       # one head a group
    (1, 8, 1, 128, 900, 100, None, None, 9),                # 800: row tiles
    (1, 2, 2, 64, 64, 512, None, None, 40),                 # the largest tree
    (1, 1, 1, 128, 63, 512, None, None, 1),                 # and a deep one
    (5, 2, 1, 128, 9000, 3, [9000, 8191, 0, 4097, 128], None, 1),
    (1, 8, 8, 128, 40001, 2, None, None, None),             # many splits
    (1, 4, 4, 64, 0, 129, None, None, 0),                   # chains: a first chunk
    (2, 8, 2, 128, 77, 200, [77, 0], [200, 130], 0),
    (1, 4, 1, 64, 1000, 700, None, None, 0),
    (1, 1, 1, 128, 5, 1500, None, None, 0),
    (40, 4, 2, 64, 50, 6, None, None, 2),                   # more pairs than a wave of blocks needs
    (1, 32, 8, 128, 8161, 33, None, None, 6),               # eight waves to a workgroup
    (2, 32, 16, 128, 4100, 20, None, None, 4),              # the same, of 40 rows
    (2, 16, 4, 128, 9000, 40, None, None, 0),
    (17, 8, 8, 128, 1100, 66, None, None, 9),               # the same, whole
    (70, 2, 1, 64, 3000, 5, "ragged", None, 2),             # more lengths than lanes
    (130, 1, 1, 128, 700, 20, "ragged", "ragged", 3),
    (150, 4, 4, 64, 600, 3, "ragged", None, 1),             # more pairs than parts
    (3, 16, 4, 128, 2100, 40, [2100, 900, 5], [40, 31, 40], 5),      # cut, with row tiles
    (3, 32, 8, 128, 500, 130, [500, 17, 0], [130, 128, 129], 0),     # whole: the merge would cost more
    (2, 32, 8, 128, 400, 250, None, None, 0),
    (1, 8, 2, 128, 100, 30, None, None, 3),                 # parts of few steps in 32 bits
    (4, 4, 2, 64, 200, 8, "ragged", None, 2),
    (2, 32, 16, 128, 170, 150, [170, 3], [150, 149], 7),    # row tiles of one wave
    (1, 8, 2, 64, 800, 100, None, None, 0),
    (1, 8, 2, 64, 801, 100, None, None, 3),                 # and one row more: of four
    (5, 64, 8, 128, 60, 32, None, None, 3),                 # many short ones
    (7, 64, 8, 64, 60, 20, "ragged", None, 3),
    (30, 2, 1, 128, 1200, 80, "ragged", "ragged", 4),       # many parts of one head's rows
]


@DTYPES
@pytest.mark.parametrize("B,Hq,Hkv,d,t,N,lens,counts,spread", CASES)
def test_tree(B, Hq, Hkv, d, t, N, lens, counts, spread, dtype):
    _run(B, Hq, Hkv, d, t, N, lens, counts, spread, dtype)


@DTYPES
@pytest.mark.parametrize("M", [15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 193, 257])
def test_row_tiles(M, dtype):
    """Query rows of a kv head around what a workgroup holds, long enough to be split."""
    _run(1, 1, 1, 64, 2000, M, None, None, 5, dtype)


@DTYPES
@pytest.mark.parametrize("t", list(range(24, 42)) + [64, 95, 96, 97, 127, 128, 129, 255, 256, 257])
def test_where_the_drafted_rows_begin(t, dtype):
    """Every offset of the tree's bits in a step, and steps that begin with it."""
    _run(1, 4, 2, 64, t, 37, None, None, 6, dtype)
    _run(1, 2, 2, 128, t, 70, None, None, 0, dtype)


@DTYPES
@pytest.mark.parametrize("t", list(range(1024, 1042)) + [1055, 1056, 1057, 1087, 1088, 1089, 1151, 1153])
def test_where_the_drafted_rows_begin_in_longer_calls(t, dtype):
    """The same where a workgroup's waves share the rows (two and four row waves)."""
    _run(1, 16, 2, 64, t, 128, None, None, 6, dtype)
    _run(1, 1, 1, 64, t, 60, None, None, 4, dtype)
    if t % 4 == 0:
        _run(2, 16, 2, 64, t, 130, None, None, 3, dtype)
    _run(1, 8, 1, 128, t, 250, [t], None, 0, dtype)


@DTYPES
@pytest.mark.parametrize("t,N,G", [(5, 1, 1), (40, 9, 4), (900, 9, 4), (900, 30, 4), (30, 130, 4), (2500, 130, 1)])
def test_zeros_behind_the_nodes(t, N, G, dtype):
    """A new out where another tensor was: zeros from the counts on, of sequences with
    none too, whether blocks or the merge write the outputs."""
    B, Hkv, d = 5, 2, 128
    counts = torch.tensor([N, 0, N // 2, 1, max(0, N - 1)], device="cuda")
    lens = torch.tensor([t, t, t // 2, 0, 1], device="cuda")
    q, K, V = _inputs(B, Hkv * G, Hkv, d, t, N, lens.tolist(), [N] * B, dtype)
    cfg = _cfg(B, Hkv * G, Hkv, d, K.shape[2], dtype)
    ws = torch.empty(radar.attend_tree_workspace_bytes(cfg, N, t), dtype=torch.uint8, device="cuda")
    given = torch.full_like(q, 5.0)
    radar.attend_tree(cfg, q, K, V, t, lens=lens, counts=counts, workspace=ws, out=given)
    old = torch.full_like(q, float("nan"))
    at = old.data_ptr()
    del old
    out = radar.attend_tree(cfg, q, K, V, t, lens=lens, counts=counts, workspace=ws)
    assert out.data_ptr() == at
    for b, n in enumerate(counts.tolist()):
        assert torch.equal(out[b, :n], given[b, :n]) and bool((out[b, n:] == 0).all()) and bool((given[b, n:] == 5).all())


@DTYPES
def test_shared_tree(dtype):
    _run(3, 8, 2, 64, 100, 20, [100, 50, 0], [20, 7, 19], 4, dtype, shared=True)


@DTYPES
@pytest.mark.parametrize("N", [3, 40])
def test_sharp_and_flat(N, dtype):
    for qscale in (60.0, 0.0):
        _run(2, 4, 2, 128, 333, N, None, None, 3, dtype, qscale=qscale)


@DTYPES
@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("N,t", [(6, 40), (30, 1000), (90, 2500), (40, 17000), (12, 33000)])
def test_other_branches_do_not_matter(N, t, chain, dtype):
    """NaN and infinities in the rows of some nodes: those who attend them get values
    that are no finite numbers in those dims, the others what they get without."""
    B, Hq, Hkv, d = 2, 8, 2, 128
    parents = [[i - 1 for i in range(N)]] * B if chain else [_tree(N, b, 4) for b in range(B)]
    P = None if chain else torch.tensor(parents, dtype=torch.int32, device="cuda")
    q, K, V = _inputs(B, Hq, Hkv, d, t, N, [t] * B, [N] * B, dtype, seed=N)
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    clean = radar.attend_tree(cfg, q, K, V, t, parent=P)
    bad = [N // 2, N - 2]
    above = [_above(p, N) for p in parents]
    hit = torch.tensor([[any(j in seen for j in bad) for seen in a] for a in above], device="cuda")
    assert 0 < int(hit.sum()) < B * N
    for kind in ("K", "V"):
        for value in (float("nan"), float("inf"), -float("inf")):
            K2, V2 = K.clone(), V.clone()
            X = K2 if kind == "K" else V2
            for j in bad:
                X[:, :, t + j, 5] = value
                X[:, :, t + j, 100:] = value
            out = radar.attend_tree(cfg, q, K2, V2, t, parent=P)
            assert torch.equal(out[~hit], clean[~hit]), (kind, value)
            if kind == "V":
                dims = [5] + list(range(100, d))
                rest = [i for i in range(d) if i not in dims]
                assert not bool(out[hit][..., dims].isfinite().any())
                assert torch.equal(out[hit][..., rest], clean[hit][..., rest])
            elif value != value:
                assert bool(out[hit].isnan().all())


@DTYPES
def test_invalid(dtype):
    """Lengths and counts outside their ranges, parents that leave the tree."""
    B, t, N, Hq, Hkv, d, cap = 8, 50, 9, 4, 2, 64, 60
    for rows in (1, 30):                               # one block of a pair, and several
        T = t * rows
        lens = [T, -1, T + 1, T, T, T, 3, T]
        counts = [9, 9, 9, -1, 10, 4, 9, 9]
        good = [max(0, min(x, T)) for x in lens]
        q, K, V = _inputs(B, Hq, Hkv, d, T, N, good, [N] * B, dtype)
        K, V = K[:, :, :T + N].contiguous(), V[:, :, :T + N].contiguous()
        parents = [_tree(N, b, 3) for b in range(B)]
        parents[6] = [-1, 1, 0, -2, 3, 2, 1 << 30, 6, 5]
        P = torch.tensor(parents, dtype=torch.int32, device="cuda")
        cfg = _cfg(B, Hq, Hkv, d, T + N, dtype)
        L, C = torch.tensor(lens, device="cuda"), torch.tensor(counts, device="cuda")
        out = radar.attend_tree(cfg, q, K, V, T, parent=P, lens=L, counts=C)
        assert bool(out[1:5].isnan().all())
        ok = [0, 5, 6, 7]
        _check(out[ok], q[ok], K[ok], V[ok], [parents[b] for b in ok], [good[b] for b in ok], [counts[b] for b in ok],
               dtype, Hkv)
        # a length and a count that pass the capacity together
        small = _cfg(B, Hq, Hkv, d, T + 4, dtype)
        out = radar.attend_tree(small, q, K[:, :, :T + 4].contiguous(), V[:, :, :T + 4].contiguous(), T, parent=P,
                                lens=torch.full_like(L, T), counts=torch.tensor([4, 5, 9, 0, 4, 1, 9, 5], device="cuda"))
        assert bool(out[[1, 2, 6, 7]].isnan().all()) and not bool(out[[0, 3, 4, 5]].isnan().any())


@DTYPES
@pytest.mark.parametrize("N,t", [(1, 300), (20, 3000), (200, 77)])
def test_strides_and_in_place(N, t, dtype):
    """q as a slice of a projection, out the same place; one token without its axis."""
    B, Hq, Hkv, d = 2, 8, 2, 64
    q, K, V = _inputs(B, Hq, Hkv, d, t, N, [t] * B, [N] * B, dtype)
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], dtype)
    want = radar.attend_tree(cfg, q, K, V, t)
    x = torch.full((B, N, Hq + 2 * Hkv, d), 3.0, dtype=q.dtype, device="cuda")
    x[:, :, Hkv:Hkv + Hq] = q
    view = x[:, :, Hkv:Hkv + Hq]
    assert torch.equal(radar.attend_tree(cfg, view, K, V, t), want)
    assert radar.attend_tree(cfg, view, K, V, t, out=view) is view
    assert torch.equal(view, want)
    x[:, :, Hkv:Hkv + Hq] = 3.0
    assert bool((x == 3.0).all())
    heads = q.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(radar.attend_tree(cfg, heads, K, V, t), want)
    if N == 1:
        assert torch.equal(radar.attend_tree(cfg, q[:, 0], K, V, t), want[:, 0])


@DTYPES
def test_workspace_of_the_largest(dtype):
    """One workspace for the largest call serves every smaller one."""
    B, Hq, Hkv, d, cap = 2, 8, 2, 64, 6200
    cfg = _cfg(B, Hq, Hkv, d, cap, dtype)
    ws = radar.attend_tree_workspace_bytes(cfg, 200, 6000)
    K, V = (torch.randn(B, Hkv, cap, d, device="cuda").to(DT[dtype]) for _ in range(2))
    for N, t in ((200, 6000), (1, 6000), (200, 0), (8, 5999), (33, 6000), (16, 3000)):
        assert radar.attend_tree_workspace_bytes(cfg, N, t) <= ws
        q = torch.randn(B, N, Hq, d, device="cuda").to(DT[dtype])
        w = Guarded((ws,), torch.uint8)
        for lens in (None, torch.tensor([t, t // 3], device="cuda")):
            out = radar.attend_tree(cfg, q, K, V, t, lens=lens, workspace=w.t)
            torch.cuda.synchronize()
            assert w.intact()
            L = [t, t] if lens is None else lens.tolist()
            _check(out, q, K, V, [_tree(N, 0, 0)] * B, L, [N] * B, dtype, Hkv)


def test_host_cache():
    q, K, V = _inputs(2, 8, 2, 128, 400, 20, [400] * 2, [20] * 2, "bf16")
    cfg = _cfg(2, 8, 2, 128, K.shape[2], "bf16")
    P = torch.tensor(_tree(20, 0, 3), dtype=torch.int32, device="cuda")
    want = radar.attend_tree(cfg, q, K, V, 400, parent=P)
    got = radar.attend_tree(cfg, q, K.cpu().pin_memory(), V.cpu().pin_memory(), 400, parent=P)
    assert torch.equal(got, want)


@DTYPES
@pytest.mark.parametrize("N", [1, 20, 100])
def test_rows_behind_2_31_elements(N, dtype):
    """A cache whose rows lie past 32-bit offsets: one of the first rows and one of the
    last take all the weight of a query each, and its value is their mean."""
    d, G = 64, 2
    t = (1 << 25) + 77 if dtype == "bf16" else (1 << 24) + 77
    K = torch.zeros(1, 1, t + N, d, dtype=DT[dtype], device="cuda")
    V = torch.zeros_like(K)
    g = torch.Generator(device="cuda").manual_seed(N)
    q = torch.randn(1, N, G, d, generator=g, device="cuda").sign().to(DT[dtype])
    at = [3, t - 5]
    K[0, 0, at] = q[0, 0, 0] * 8                           # logits of 64 for the first query row
    V[0, 0, at] = torch.randn(2, d, generator=g, device="cuda").to(DT[dtype])
    V[0, 0, t:] = 5.0
    cfg = _cfg(1, G, 1, d, t + N, dtype)
    out = radar.attend_tree(cfg, q, K, V, t)
    # the others' weights together: 2^25 e^-64 of a row's
    want = V[0, 0, at].double().mean(0)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    lim = (2 * half + 1e-5) * V[0, 0, at].double().abs().sum(0) + 1e-18
    assert bool(((out[0, 0, 0].double() - want).abs() <= lim).all())


@DTYPES
def test_agrees_with_the_other_attentions(dtype):
    """One token over t rows: what attend_prefix gives for its t + 1."""
    q, K, V = _inputs(3, 8, 2, 128, 2000, 1, [2000] * 3, [1] * 3, dtype)
    cfg = _cfg(3, 8, 2, 128, K.shape[2], dtype)
    a = radar.attend_tree(cfg, q[:, 0], K, V, 2000)
    b = radar.attend_prefix(cfg, q[:, 0].contiguous(), None, None, 0, K, V, 2001)
    lim = 2 * torch.finfo(DT[dtype]).eps if dtype == "bf16" else 1e-4
    assert float((a.double() - b.double()).abs().max()) <= lim * float(b.abs().max())


def test_replayed_and_other_stream():
    B, Hq, Hkv, d, t, N = 2, 8, 2, 64, 3000, 24
    q, K, V = _inputs(B, Hq, Hkv, d, t, N, [t] * B, [N] * B, "bf16")
    cfg = _cfg(B, Hq, Hkv, d, K.shape[2], "bf16")
    P = torch.tensor([_tree(N, b, 3) for b in range(B)], dtype=torch.int32, device="cuda")
    lens, counts = torch.tensor([t, 50], device="cuda"), torch.tensor([N, 5], device="cuda")
    ws = torch.empty(radar.attend_tree_workspace_bytes(cfg, N, t), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    kw = dict(parent=P, lens=lens, counts=counts, workspace=ws, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        radar.attend_tree(cfg, q, K, V, t, **kw)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        radar.attend_tree(cfg, q, K, V, t, **kw)
    for i in range(5):
        n = torch.tensor([[t, 50], [7, t], [0, 0], [t, t], [1500, 2999]][i])
        m = torch.tensor([[N, 5], [1, 2], [N, N], [0, N], [13, 24]][i])
        K.copy_(torch.randn(K.shape, device="cuda"))
        V.copy_(torch.randn(K.shape, device="cuda"))
        q.copy_(torch.randn(q.shape, device="cuda"))
        P.copy_(torch.tensor([_tree(N, 10 * i + b, 4) for b in range(B)]))
        lens.copy_(n)
        counts.copy_(m)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, radar.attend_tree(cfg, q, K, V, t, parent=P, lens=lens, counts=counts)), i


def test_two_streams_at_once():
    """Two calls with workspaces of their own, at the same time."""
    q, K, V = _inputs(1, 8, 2, 128, 20000, 40, [20000], [40], "bf16")
    cfg = _cfg(1, 8, 2, 128, K.shape[2], "bf16")
    want = radar.attend_tree(cfg, q, K, V, 20000)
    want2 = radar.attend_tree(cfg, q, K, V, 9000)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            got.append(radar.attend_tree(cfg, q, K, V, 20000 if i % 2 else 9000))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want if i % 2 else want2)


def test_binding_refuses():
    cfg = _cfg(2, 8, 2, 64, 100, "f32")
    q, K = torch.zeros(2, 5, 8, 64, device="cuda"), torch.zeros(2, 2, 100, 64, device="cuda")
    P = torch.full((5,), -1, dtype=torch.int32, device="cuda")
    one = torch.tensor([1, 2], device="cuda")
    for bad in (dict(parent=P.long()), dict(parent=P[:4]), dict(parent=P.expand(3, 5).contiguous()), dict(parent=P.cpu()),
                dict(counts=one.int()), dict(counts=one[:1]), dict(lens=one[:1]), dict(out=q[:, :4]),
                dict(out=q.bfloat16()), dict(workspace=torch.zeros(9, device="cuda")), dict(q=q[..., :32]),
                dict(q=q[:, :, :4]), dict(q=q.bfloat16()), dict(K=K[:, :, :99].contiguous())):
        kw = dict(q=q, K=K, V=K, t=20)
        kw.update(bad)
        with pytest.raises(ValueError):
            radar.attend_tree(cfg, **kw)
    for bad, status in ((dict(t=96), 2), (dict(t=-1), 2), (dict(workspace=torch.zeros(9, dtype=torch.uint8, device="cuda")), 5)):
        kw = dict(q=q, K=K, V=K, t=20)
        kw.update(bad)
        with pytest.raises(radar.RadarError) as e:
            radar.attend_tree(cfg, **kw)
        assert e.value.status == status
    with pytest.raises(RuntimeError):
        radar.attend_tree(cfg, q.clone().requires_grad_(), K, K, 20)
