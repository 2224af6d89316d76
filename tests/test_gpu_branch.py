"""What moves rows when sequences branch, on the GPU: the acceptance of a path of
drafted tokens, given paths, the index of the rows that joined, and forking. All
of it is moves: every result is held to equality with a plain program's."""
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


def _cfg(B, Hkv, d, cap, dtype, c=16, n=64, sink=0):
    return radar.Config(B, Hkv, Hkv, d, n, c, c, cap, DT[dtype], sink)


def _caches(B, Hkv, cap, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [Guarded((B, Hkv, cap, d), DT[dtype], init=torch.randn(B, Hkv, cap, d, generator=g, device="cuda"))
            for _ in range(2)]


def _walk(parent, tokens, first, choice, m):
    """The path of one sequence's m nodes, and the last choice."""
    cur, want, path = -1, first, []
    while True:
        fits = [i for i in range(cur + 1, m) if parent[i] == cur and tokens[i] == want]
        if not fits:
            return path, want
        cur = fits[0]
        path.append(cur)
        want = choice[cur]


def _int(x, dtype=torch.int64):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _drafts(B, N, seed, chain=False, hit=0.85):
    """Random trees whose choices mostly name a child: parents, tokens, first, choice."""
    r = torch.Generator().manual_seed(seed)

    def below(n):
        return int(torch.randint(0, n, (1,), generator=r))

    out = []
    for _ in range(B):
        parent = [i - 1 if chain else i - 1 - below(min(i, 6) + 1) for i in range(N)]
        tokens = [below(5) for _ in range(N)]            # siblings often agree: the lowest counts
        want = [below(5) for _ in range(N + 1)]
        for i in range(-1, N):
            kids = [j for j in range(N) if parent[j] == i]
            if kids and float(torch.rand(1, generator=r)) < hit:
                want[i + 1] = tokens[kids[below(len(kids))]]
        out.append((parent, tokens, want[0], want[1:]))
    return out


ACCEPT = [  # B, Hkv, d, N, t
    (1, 1, 64, 1, 0),
    (1, 8, 128, 26, 100),
    (3, 2, 64, 64, 33),
    (2, 17, 128, 65, 5),
    (5, 3, 128, 200, 70),
    (2, 2, 64, 512, 9),
    (70, 1, 64, 7, 3),
]


@DTYPES
@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("B,Hkv,d,N,t", ACCEPT)
def test_accept(B, Hkv, d, N, t, chain, dtype):
    print(f"[case] accept B{B} Hkv{Hkv} d{d} N{N} t{t} chain={chain} {dtype}", flush=True)
    drafts = _drafts(B, N, N + t, chain)
    lens = [max(0, t - b % 5) for b in range(B)]
    counts = [max(0, N - 3 * (b % 4)) for b in range(B)]
    cap = t + N + 2
    K, V = _caches(B, Hkv, cap, d, dtype)
    wantK, wantV = K.t.clone(), V.t.clone()
    paths, nexts = [], []
    for b, (parent, tokens, first, choice) in enumerate(drafts):
        path, nxt = _walk(parent, tokens, first, choice, counts[b])
        paths.append(path)
        nexts.append(nxt)
        rows = [lens[b] + i for i in path]
        for want, x in ((wantK, K), (wantV, V)):
            want[b, :, lens[b]:lens[b] + len(path)] = x.t[b][:, rows]
    assert N < 20 or max(len(p) for p in paths) > 1
    path = Guarded((B, N), torch.int32)
    new = _int([0] * B)
    cfg = _cfg(B, Hkv, d, cap, dtype)
    got, n, nxt = radar.accept_tree(cfg, K.t, V.t, t, _int([x[1] for x in drafts]), _int([x[2] for x in drafts]),
                                    _int([x[3] for x in drafts]),
                                    parent=None if chain else _int([x[0] for x in drafts], torch.int32),
                                    counts=_int(counts), lens=_int(lens), new_lens=new, path=path.t)
    torch.cuda.synchronize()
    assert K.intact() and V.intact() and path.intact()
    assert got.tolist() == [p + [-1] * (N - len(p)) for p in paths]
    assert n.tolist() == [len(p) for p in paths] and nxt.tolist() == nexts
    assert new.tolist() == [a + len(p) for a, p in zip(lens, paths)]
    assert torch.equal(K.t, wantK) and torch.equal(V.t, wantV)


def test_accept_shared_tree_in_place():
    """One tree for the batch, no lengths; and new lengths and the next token in the
    places of the old ones."""
    B, N, t = 4, 9, 12
    parent, _, _, _ = _drafts(1, N, 3)[0]
    cfg = _cfg(B, 2, 64, 40, "bf16")
    K, V = _caches(B, 2, 40, 64, "bf16")
    rows = [_drafts(1, N, 10 + b)[0] for b in range(B)]
    tokens, first, choice = _int([r[1] for r in rows]), _int([r[2] for r in rows]), _int([r[3] for r in rows])
    walks = [_walk(parent, r[1], r[2], r[3], N) for r in rows]
    P = _int(parent, torch.int32)
    before = K.t.clone()
    path, n, nxt = radar.accept_tree(cfg, K.t, V.t, t, tokens, first, choice, parent=P)
    assert n.tolist() == [len(w[0]) for w in walks] and nxt.tolist() == [w[1] for w in walks]
    K.t.copy_(before)
    lens, f = _int([t] * B), first.clone()
    p2, n2, _ = radar.accept_tree(cfg, K.t, V.t, t, tokens, f, choice, parent=P, lens=lens, new_lens=lens, next_token=f)
    assert torch.equal(path, p2) and torch.equal(n, n2)
    assert lens.tolist() == [t + len(w[0]) for w in walks] and f.tolist() == [w[1] for w in walks]


def test_accept_invalid():
    """Lengths and counts outside their ranges, and parents that are no nodes before."""
    B, N, t, cap = 7, 6, 10, 16
    cfg = _cfg(B, 2, 64, cap, "f32")
    K, V = _caches(B, 2, cap, 64, "f32")
    wantK, wantV = K.t.clone(), V.t.clone()
    lens, counts = [11, -1, 10, 10, 10, 4, 10], [6, 6, 7, -1, 6, 6, 0]
    parent = [[-1, 0, 1, 2, 3, 4]] * B
    parent[4], parent[5] = [-1, 1, 7, -2, 0, 4], [0, 5, 1 << 30, -(1 << 31), 4, 5]
    tokens = _int([[1] * N] * B)
    new = _int([5] * B)
    path, n, nxt = radar.accept_tree(cfg, K.t, V.t, t, tokens, _int([1] * B), tokens.clone(), lens=_int(lens),
                                     parent=_int(parent, torch.int32), counts=_int(counts), new_lens=new)
    wantK[4, :, 11:13] = wantK[4][:, [14, 15]]
    wantV[4, :, 11:13] = wantV[4][:, [14, 15]]
    assert n.tolist() == [0, 0, 0, 0, 3, 0, 0]
    assert nxt.tolist() == [-1, -1, -1, -1, 1, 1, 1]
    assert new.tolist() == [11, -1, 10, 10, 13, 4, 10]
    assert path[4].tolist() == [0, 4, 5, -1, -1, -1]
    assert bool((path[[0, 1, 2, 3, 5, 6]] == -1).all())
    assert torch.equal(K.t, wantK) and torch.equal(V.t, wantV)


def test_accept_large_tokens():
    """Tokens that differ in their upper 32 bits only."""
    cfg = _cfg(1, 1, 64, 8, "f32")
    K, V = _caches(1, 1, 8, 64, "f32")
    big = 1 << 40
    path, n, nxt = radar.accept_tree(cfg, K.t, V.t, 0, _int([[3, big + 3, 3]]), _int([big + 3]),
                                     _int([[0, 3, -big]]), parent=_int([-1, -1, 1], torch.int32))
    assert path.tolist() == [[1, 2, -1]] and n.tolist() == [2] and nxt.tolist() == [-big]


@DTYPES
@pytest.mark.parametrize("n", [0, 1, 5, 16, 17, 100, 700])
def test_keep_path(n, dtype):
    B, Hkv, d, t = 5, 3, 128, 20
    cap = t + 2 * n + 8
    K, V = _caches(B, Hkv, cap, d, dtype)
    r = torch.Generator().manual_seed(n)
    path = torch.stack([torch.randperm(2 * n + 1, generator=r)[:n].sort()[0] for _ in range(B)]) if n else torch.zeros(B, 0)
    path = path.to(torch.int32)
    lens, counts = [20, 0, 7, 20, 11], [n, n, n // 2, n, 0]
    wantK, wantV, new = K.t.clone(), V.t.clone(), [a + c for a, c in zip(lens, counts)]
    if n > 1:
        path[3, n - 1] = path[3, n - 2]               # the same row twice: refused
        new[3], counts_ok = -1, [0, 1, 2, 4]
    else:
        counts_ok = range(B)
    for b in counts_ok:
        rows = [lens[b] + int(i) for i in path[b, :counts[b]]]
        for want, x in ((wantK, K), (wantV, V)):
            want[b, :, lens[b]:lens[b] + len(rows)] = x.t[b][:, rows]
    L = _int(lens)
    radar.keep_path(_cfg(B, Hkv, d, cap, dtype), K.t, V.t, t, path.cuda(), counts=_int(counts), lens=L, new_lens=L)
    torch.cuda.synchronize()
    assert K.intact() and V.intact()
    assert L.tolist() == new
    assert torch.equal(K.t, wantK) and torch.equal(V.t, wantV)


def test_keep_path_refused_ones_stay():
    B, cap, t = 6, 30, 20
    K, V = _caches(B, 1, cap, 64, "f32")
    want = K.t.clone()
    path = _int([[0, 2], [-1, 3], [4, 10], [3, 2], [1, 2], [0, 1]], torch.int32)
    new = _int([0] * B)
    radar.keep_path(_cfg(B, 1, 64, cap, "f32"), K.t, V.t, t, path, lens=_int([21, 20, 20, 20, 20, -1]), new_lens=new)
    want[4, :, 20:22] = want[4][:, [21, 22]]
    assert new.tolist() == [-1, -1, -1, -1, 22, -1]
    assert torch.equal(K.t, want)
    radar.keep_path(_cfg(B, 1, 64, cap, "f32"), K.t, V.t, t, path, counts=_int([3, -1, 0, 1, 1, 2]), new_lens=new)
    assert new.tolist() == [-1, -1, 20, 21, 21, 22]


# ---- the index of the rows that joined ------------------------------------------
@DTYPES
@pytest.mark.parametrize("c,sink", [(16, 0), (7, 3), (64, 1)])
def test_extend_index(c, sink, dtype):
    """Bit for bit what the whole build gives, and nothing else is written."""
    B, Hkv, d, n, cap = 3, 2, 64, 64, 300
    cfg = _cfg(B, Hkv, d, cap, dtype, c, n, sink)
    K, _ = _caches(B, Hkv, cap, d, dtype)
    omega = torch.randn(n, d, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16().float()
    full = radar.new_summaries(cfg, "cuda")
    radar.build_index(cfg, K.t, omega, cap, full)
    rows = full.shape[2]
    done = [max(0, r - sink) // c for r in range(cap + 1)]
    for t0, t in ((0, 0), (0, 1), (0, 130), (5, 90), (c + sink - 1, c + sink), (100, 100), (40, 300)):
        s = Guarded(full.shape, torch.float32, init=torch.full_like(full, -7.0))
        radar.extend_index(cfg, K.t, omega, t0, t, s.t)
        torch.cuda.synchronize()
        assert s.intact()
        want = torch.full_like(full, -7.0)
        want[:, :, done[t0]:done[t]] = full[:, :, done[t0]:done[t]]
        assert torch.equal(s.t, want), (t0, t)
    for most in (0, 1, c - 1, c, 3 * c + 1, 200):
        lens0 = [max(0, 150 - most), 37, 250]
        lens = [150, 37 + min(most, 60), min(251, 250 + most)]
        ws = Guarded((radar.extend_index_workspace_bytes(cfg, most),), torch.uint8)
        s = Guarded(full.shape, torch.float32, init=torch.full_like(full, -7.0))
        radar.extend_index(cfg, K.t, omega, 0, 299, s.t, lens0=_int(lens0), lens=_int(lens), most=most, workspace=ws.t)
        torch.cuda.synchronize()
        assert s.intact() and ws.intact()
        want = torch.full_like(full, -7.0)
        for b in range(B):
            want[b, :, done[lens0[b]]:done[lens[b]]] = full[b, :, done[lens0[b]]:done[lens[b]]]
        assert torch.equal(s.t, want), most
    s = torch.full_like(full, -7.0)                    # invalid pairs, and rows behind `most`
    radar.extend_index(cfg, K.t, omega, 0, 200, s, lens0=_int([-1, 90, 0]), lens=_int([50, 80, 200]), most=2 * c)
    want = torch.full_like(full, -7.0)
    want[2, :, :done[2 * c]] = full[2, :, :done[2 * c]]
    assert rows >= 4 and torch.equal(s, want)
    s.fill_(-7.0)
    radar.extend_index(cfg, K.t, omega, 0, 200, s, lens0=_int([0, 0, 0]), lens=_int([201, 0, 1]), most=200)
    assert bool((s[:2] == -7.0).all())


# ---- forking -----------------------------------------------------------------------
def _forked(x, src, lens, first, old):
    """x [B][..][rows][..] after the fork, rows on axis 2."""
    out = x.clone()
    for b, s in enumerate(src):
        if 0 <= s < len(src) and 0 <= old[s]:
            out[b, :, first:max(first, lens[s])] = x[s, :, first:max(first, lens[s])]
    return out


def _check_fork(src, lens, t, first, dtype, Hkv=2, d=64, c=16, n=64, sink=0, extra=True, in_place=False, spare=5):
    B, cap = len(src), t + spare
    print(f"[case] fork B{B} t{t} first{first} {dtype} sink{sink} src{src[:12]}", flush=True)
    cfg = _cfg(B, Hkv, d, cap, dtype, c, n, sink)
    K, V = _caches(B, Hkv, cap, d, dtype, seed=t)
    g = torch.Generator(device="cuda").manual_seed(t + 1)
    mass = Guarded((B, Hkv, cap), torch.float32, init=torch.rand(B, Hkv, cap, generator=g, device="cuda"))
    S = max(1, cap // c)
    summ = Guarded((B, Hkv, S, n), torch.float32, init=torch.rand(B, Hkv, S, n, generator=g, device="cuda"))
    old = [t] * B if lens is None else lens
    old = [x if 0 <= x <= t else -1 for x in old]
    raw = [t] * B if lens is None else lens
    wantK, wantV = (_forked(x.t, src, old, first, old) for x in (K, V))
    wantM, wantS = mass.t.clone(), summ.t.clone()
    new = []
    for b, s in enumerate(src):
        new.append(0 if s == -1 else raw[s] if 0 <= s < B else -1)
        if s == b or s < -1 or s >= B or s >= 0 and old[s] < 0:
            continue
        m = 0 if s == -1 else old[s]
        wantM[b, :, m:max(m, old[b])] = 0
        if s >= 0:
            wantM[b, :, :m] = mass.t[s, :, :m]
            a, e = max(0, first - sink) // c, max(0, m - sink) // c
            wantS[b, :, a:max(a, e)] = summ.t[s, :, a:max(a, e)]
    L = None if lens is None else _int(lens)
    N = L if in_place else _int([77] * B)
    radar.fork(cfg, K.t, V.t, _int(src), t, first=first, lens=L, new_lens=N, mass=mass.t if extra else None,
               summaries=summ.t if extra else None)
    torch.cuda.synchronize()
    assert K.intact() and V.intact() and mass.intact() and summ.intact()
    assert N.tolist() == new
    assert torch.equal(K.t, wantK) and torch.equal(V.t, wantV)
    if extra:
        assert torch.equal(mass.t, wantM) and torch.equal(summ.t, wantS)


MAPS = {
    "one": [0],
    "none": [0, 1, 2, 3],
    "samples": [0] * 9,
    "last": [4] * 5,
    "swap": [1, 0],
    "cycles": [1, 2, 0, 4, 3, 5],
    "chain": [1, 2, 3, 4, 4],
    "back": [0, 0, 1, 2, 3],
    "tree into a cycle": [1, 2, 0, 0, 3, 3, 2],
    "freed": [-1, 2, -1, 0, 3],
    "freed in use": [3, -1, 1, 1, -1],
    "all freed": [-1, -1, -1],
    "invalid": [5, -2, 0, 1 << 40, 3],
    "shift by one": [(b + 1) % 40 for b in range(40)],
    "reversed": list(range(32, -1, -1)),
    "long chain": [min(b + 1, 99) for b in range(100)],
    "zeros between": [0, -1, 0, -1, 0, -1, 0, 3],
}


@DTYPES
@pytest.mark.parametrize("name", list(MAPS))
def test_fork_maps(name, dtype):
    src = MAPS[name]
    B = len(src)
    _check_fork(src, None, 37, 0, dtype)
    _check_fork(src, [(13 * b + 5) % 41 for b in range(B)], 40, 0, dtype, sink=3, c=7)
    _check_fork(src, [(29 * b + 7) % 41 for b in range(B)], 40, 18, dtype, in_place=True)


@DTYPES
@pytest.mark.parametrize("seed", range(6))
def test_fork_random_maps(seed, dtype):
    r = torch.Generator().manual_seed(seed)
    B = [2, 3, 17, 64, 255, 300][seed]
    src = torch.randint(-1, B, (B,), generator=r).tolist()
    perm = torch.randperm(B, generator=r).tolist()
    lens = torch.randint(0, 51, (B,), generator=r).tolist()
    for s in (src, perm):
        _check_fork(s, lens, 50, 0, dtype, Hkv=1, c=9)
        _check_fork(s, lens, 50, 11, dtype, Hkv=1, extra=False, in_place=True)


@DTYPES
@pytest.mark.parametrize("d,t,first", [(128, 0, 0), (128, 1, 0), (128, 1, 1), (64, 5, 9), (128, 2000, 3), (64, 4097, 4000)])
def test_fork_sizes(d, t, first, dtype):
    _check_fork([1, 0, 0, 2], [t, t // 2, 0, min(t, 3)], t, min(first, t), dtype, Hkv=3, d=d, spare=0 if t else 1)
    _check_fork([1, 0, 0, 2], None, t, min(first, t), dtype, Hkv=3, d=d, spare=3)


@DTYPES
def test_fork_invalid_lengths(dtype):
    """From a sequence of no valid length nothing is copied; onto one it is."""
    _check_fork([1, 2, 0, 4, 3, 0], [10, 21, -1, 20, -5, 7], 20, 0, dtype)
    _check_fork([1, 2, 0, 4, 3, 0], [10, 21, -1, 20, -5, 7], 20, 0, dtype, in_place=True)


def test_fork_most_sequences():
    B = 2048
    r = torch.Generator().manual_seed(0)
    _check_fork(torch.randperm(B, generator=r).tolist(), None, 9, 0, "f32", Hkv=1, spare=1)
    _check_fork([min(b + 1, B - 1) for b in range(B)], None, 3, 0, "bf16", Hkv=1, extra=False, in_place=False)
    cfg = _cfg(B + 1, 1, 64, 4, "f32")
    K = torch.zeros(B + 1, 1, 4, 64, device="cuda")
    with pytest.raises(radar.RadarError) as e:
        radar.fork(cfg, K, K.clone(), torch.zeros(B + 1, dtype=torch.int64, device="cuda"), 4)
    assert e.value.status == 3


@pytest.mark.parametrize("src", [[1, 2, 0, 0], [3, 4, 0, 1, 5, 6, 3, 2]])
def test_fork_past_the_caches(src):
    """More than the Infinity Cache holds."""
    B = len(src)
    _check_fork(src, [64000 // B - 1000 * b for b in range(B)], 64000 // B, 7, "bf16", Hkv=8, d=128, c=512)


@DTYPES
def test_fork_behind_2_31_elements(dtype):
    """Sequences and rows that lie past 32-bit offsets; only the last rows move."""
    t = (1 << 25) + 40 if dtype == "bf16" else (1 << 24) + 40
    K = torch.zeros(2, 1, t, 64, dtype=DT[dtype], device="cuda")
    V = torch.zeros_like(K)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (K, V):
        x[:, :, -100:] = torch.randn(2, 1, 100, 64, generator=g, device="cuda").to(DT[dtype])
    want = [x[:, :, -100:].flip(0) for x in (K, V)]
    radar.fork(_cfg(2, 1, 64, t, dtype), K, V, _int([1, 0]), t, first=t - 60)
    for x, w, in zip((K, V), want):
        assert torch.equal(x[:, :, -60:], w[:, :, -60:])
        assert torch.equal(x[:, :, -100:-60], w[:, :, :40].flip(0)) and not bool(x[:, :, :1000].any())
    lens = _int([t - 50, t - 9])
    before = [x[:, :, -100:].clone() for x in (K, V)]
    radar.keep_path(_cfg(2, 1, 64, t, dtype), K, V, t, _int([[1, 3, 8], [0, 2, 8]], torch.int32), lens=lens, new_lens=lens)
    for x, w in zip((K, V), before):
        w[0, :, 50:53] = w[0][:, [51, 53, 58]]
        w[1, :, 91:94] = w[1][:, [91, 93, 99]]
        assert torch.equal(x[:, :, -100:], w)
    assert lens.tolist() == [t - 47, t - 6]


def test_paths_in_a_host_cache():
    K, V = (torch.randn(2, 3, 30, 64).pin_memory() for _ in range(2))
    want = [x.clone() for x in (K, V)]
    for w in want:
        w[:, :, 10:12] = w[:, :, [10, 13]]
    cfg = _cfg(2, 3, 64, 30, "f32")
    tokens = _int([[1, 2, 3, 4]] * 2)
    path, n, token = radar.accept_tree(cfg, K, V, 10, tokens, _int([1, 1]), _int([[4, 0, 0, 9]] * 2),
                                       parent=_int([-1, 0, 0, 0], torch.int32))
    torch.cuda.synchronize()
    assert path.tolist() == [[0, 3, -1, -1]] * 2 and token.tolist() == [9, 9]
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])
    for w in want:
        w[:, :, 12:14] = w[:, :, [14, 17]]
    radar.keep_path(cfg, K, V, 12, _int([[2, 5]] * 2, torch.int32))
    torch.cuda.synchronize()
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])


def test_fork_host_cache():
    K, V = (torch.randn(3, 2, 30, 64).pin_memory() for _ in range(2))
    want = [_forked(x, [1, 2, 2], [25] * 3, 0, [25] * 3) for x in (K, V)]
    radar.fork(_cfg(3, 2, 64, 30, "f32"), K, V, _int([1, 2, 2]), 25)
    torch.cuda.synchronize()
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])


# ---- as calls may come ----------------------------------------------------------------
def test_replayed():
    """Acceptance, the index and a fork in one graph, lengths in place, replayed with
    other inputs and eager work between."""
    B, Hkv, d, N, cap, c, n = 4, 2, 64, 9, 400, 16, 64
    cfg = _cfg(B, Hkv, d, cap, "bf16", c, n)
    g = torch.Generator(device="cuda").manual_seed(0)

    def fresh():
        return torch.randn(B, Hkv, cap, d, generator=g, device="cuda").bfloat16()

    omega = torch.randn(n, d, generator=g, device="cuda").bfloat16().float()
    state = dict(K=fresh(), V=fresh(), lens=_int([40, 3, 77, 20]), first=_int([0] * B), tokens=_int([[0] * N] * B),
                 choice=_int([[0] * N] * B), parent=_int([[-1] * N] * B, torch.int32), src=_int([0] * B),
                 summ=radar.new_summaries(cfg, "cuda"))
    was = state["lens"].clone()
    ws = torch.empty(radar.extend_index_workspace_bytes(cfg, N), dtype=torch.uint8, device="cuda")

    def go(s, was, out):
        was.copy_(s["lens"])
        radar.accept_tree(cfg, s["K"], s["V"], 300, s["tokens"], s["first"], s["choice"], parent=s["parent"],
                          lens=s["lens"], new_lens=s["lens"], **out)
        radar.extend_index(cfg, s["K"], omega, 0, 300, s["summ"], lens0=was, lens=s["lens"], most=N, workspace=ws)
        radar.fork(cfg, s["K"], s["V"], s["src"], 300, lens=s["lens"], new_lens=s["lens"], summaries=s["summ"])

    def outs():
        return dict(path=_int([[0] * N] * B, torch.int32), accepted=_int([0] * B), next_token=_int([0] * B))

    out = outs()
    eager = {k: v.clone() for k, v in state.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go({k: v.clone() for k, v in state.items()}, was.clone(), outs())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(state, was, out)
    for i in range(5):
        drafts = _drafts(B, N, i)
        for name, j, dt in (("parent", 0, torch.int32), ("tokens", 1, torch.int64), ("first", 2, torch.int64),
                            ("choice", 3, torch.int64)):
            v = _int([x[j] for x in drafts], dt)
            state[name].copy_(v)
            eager[name].copy_(v)
        src = _int([[0, 1, 2, 3], [1, 0, 3, 2], [2, 2, 2, 2], [3, 0, 1, 2], [0, 0, 1, -1]][i])
        state["src"].copy_(src)
        eager["src"].copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        ref = outs()
        go(eager, was.clone(), ref)
        for k in state:
            assert torch.equal(state[k], eager[k]), (i, k)
        for k in out:
            assert torch.equal(out[k], ref[k]), (i, k)


def test_binding_refuses():
    cfg = _cfg(2, 1, 64, 20, "f32")
    K = torch.zeros(2, 1, 20, 64, device="cuda")
    i2 = _int([[1, 2], [3, 4]])
    one = _int([1, 2])
    for bad in (dict(tokens=i2.int()), dict(tokens=i2[0]), dict(first=one[:1]), dict(choice=i2[:1].contiguous()),
                dict(parent=i2), dict(parent=_int([-1], torch.int32)), dict(counts=one.int()), dict(lens=one[:1]),
                dict(new_lens=one.int()), dict(path=i2), dict(accepted=one[:1]), dict(next_token=one.cpu())):
        kw = dict(tokens=i2, first=one, choice=i2)
        kw.update(bad)
        with pytest.raises(ValueError):
            radar.accept_tree(cfg, K, K.clone(), 5, **kw)
    for bad in (i2, _int([1, 2], torch.int32), _int([[1]], torch.int32)):
        with pytest.raises(ValueError):
            radar.keep_path(cfg, K, K.clone(), 5, bad)
    for bad in (dict(src=one.int()), dict(src=one[:1]), dict(lens=one[:1]), dict(new_lens=one.int()),
                dict(mass=torch.zeros(2, 1, 19, device="cuda")), dict(summaries=torch.zeros(3, device="cuda"))):
        kw = dict(src=one)
        kw.update(bad)
        with pytest.raises(ValueError):
            radar.fork(cfg, K, K.clone(), t=5, **kw)
    with pytest.raises(ValueError):
        radar.extend_index(cfg, K, torch.zeros(64, 64, device="cuda"), 0, 5, radar.new_summaries(cfg, "cuda"), lens=one)
    with pytest.raises(radar.RadarError) as e:
        radar.accept_tree(cfg, K, K.clone(), 19, i2, one, i2)
    assert e.value.status == 2
    with pytest.raises(radar.RadarError) as e:
        radar.fork(cfg, K, K.clone(), one, 5, new_lens=one)
    assert e.value.status == 1
