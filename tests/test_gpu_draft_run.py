"""Drafting as a program does it, through RadarLayer and the calls below it: prompts,
trees of drafted tokens attended and accepted, decode steps, forks, positions on
several axes. The outputs are held to exact attention in 64 bits over the rows that
ought to be there, rotated in 64 bits from the unrotated inputs; the index, bit for
bit, to one built anew."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
import _cache_ref as R  # noqa: E402
from test_gpu_cache_run import _attend, _logit_step, _near, _turn  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu

# nodes, their parents and depths
PARENT = [-1, -1, 0, 0, 1, 2, 5, 3]
DEPTH = [0, 0, 1, 1, 1, 2, 3, 2]


def _above(i):
    out = [i]
    while PARENT[out[-1]] >= 0:
        out.append(PARENT[out[-1]])
    return out[::-1]


@pytest.mark.parametrize("schedule", ["fixed", "sqrt"])
@pytest.mark.parametrize("dtype,rope", [(torch.float32, True), (torch.bfloat16, True), (torch.bfloat16, False)])
def test_layer_drafts(dtype, rope, schedule):
    B, Hq, Hkv, d, T, N = 2, 4, 2, 64, 90, len(PARENT)
    G = Hq // Hkv
    print(f"[case] layer drafts {dtype} rope={rope} {schedule}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    f, m = radar.rope_frequencies(48, 10000.0, "yarn", 4.0, trained_len=64)
    rp = radar.Rope(f.cuda(), False, m) if rope else None
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, 160, dtype, 3)
    omega = torch.randn(64, d, generator=g, device="cuda").to(torch.bfloat16).float()
    layer = radar.RadarLayer(cfg, omega, top_k=64, schedule=schedule, rope=rp)
    r = torch.Generator().manual_seed(1)

    def rand(*s):
        return (0.5 * torch.randn(*s, generator=g, device="cuda")).to(dtype)

    rows = [[[] for _ in range(Hkv)] for _ in range(B)]        # key, value, position

    def exact(b, h, q, pos, extra=()):
        """q [G][d] at pos over the rows of (b, h) and `extra`."""
        all_rows = rows[b][h] + list(extra)
        k, v = (torch.stack([x[j] for x in all_rows]).double() for j in (0, 1))
        qq = q.double()
        if rope:
            k = _turn(k, rp, torch.tensor([x[2] for x in all_rows], device="cuda"))
            qq = _turn(q[None], rp, torch.tensor([pos], device="cuda"))[0]
        return _attend(qq, k, v)[0], v, _logit_step(qq, k, dtype)

    def index_is_right():
        fresh = torch.zeros_like(layer.summaries)
        radar.build_index(layer.cfg, layer.K, omega, layer.t, fresh)
        n = max(0, layer.t - 3) // layer.cfg.seg_len
        a, b = (x.flatten()[:B * Hkv * layer.cfg.summary_rows * 64].view(B, Hkv, -1, 64)[:, :, :n]
                for x in (layer.summaries, fresh))
        assert torch.equal(a, b)

    k, v = rand(B, T, Hkv, d), rand(B, T, Hkv, d)
    layer.prefill(k, v)
    for b in range(B):
        for h in range(Hkv):
            rows[b][h] = [(k[b, t, h], v[b, t, h], t) for t in range(T)]
    parent = torch.tensor(PARENT, dtype=torch.int32, device="cuda")
    depth = torch.tensor(DEPTH, device="cuda") if rope else None
    for turn in range(7):
        chain = turn == 3
        q, k, v = rand(B, N, Hq, d), rand(B, N, Hkv, d), rand(B, N, Hkv, d)
        out = layer.draft(q, k, v, parent=None if chain else parent, depth=None if chain else depth)
        at, pos0 = layer.t, layer.pos
        for b in range(B):
            for h in range(Hkv):
                for i in range(N):
                    seen = list(range(i + 1)) if chain else _above(i)
                    where = {j: pos0 + (j if chain else DEPTH[j]) for j in seen}
                    ref, vv, ds = exact(b, h, q[b, i, h * G:(h + 1) * G], where[i],
                                        [(k[b, j, h], v[b, j, h], where[j]) for j in seen])
                    _near(out[b, i, h * G:(h + 1) * G], ref, vv, dtype, ds)
        # the model's choices follow a leaf's path, for the second sequence less far
        leaf = N - 1 if chain else [6, 7, 4][turn % 3]
        path = list(range(leaf + 1)) if chain else _above(leaf)
        tokens = torch.randint(100, 200, (B, N), generator=r) * 8 + torch.arange(N)
        choice, first = torch.zeros(B, N, dtype=torch.int64), torch.zeros(B, dtype=torch.int64)
        for b in range(B):
            upto = max(1, len(path) - b * (turn % 2))
            first[b] = tokens[b, path[0]]
            for x, y in zip(path[:upto], path[1:upto]):
                choice[b, x] = tokens[b, y]
            choice[b, path[upto - 1]] = 7 + b
        n, after = layer.accept(tokens.cuda(), first.cuda(), choice.cuda(), parent=None if chain else parent)
        assert n == max(1, len(path) - turn % 2) and layer.t == at + n and layer.pos == pos0 + n
        assert after.tolist() == [7 if n == len(path) else int(tokens[0, path[n]]), 8]
        for b in range(B):
            for h in range(Hkv):
                rows[b][h] += [(k[b, j, h], v[b, j, h], pos0 + i) for i, j in enumerate(path[:n])]
        index_is_right()
        if turn == 4:                                          # the second becomes the first
            layer.fork(torch.tensor([0, 0], device="cuda"))
            rows[1] = [list(x) for x in rows[0]]
            index_is_right()
        # a step over every segment, which reads the accepted rows' summaries
        q, kn, vn = rand(B, Hq, d), rand(B, Hkv, d), rand(B, Hkv, d)
        out = layer.step(q, kn, vn)
        for b in range(B):
            for h in range(Hkv):
                rows[b][h].append((kn[b, h], vn[b, h], layer.pos - 1))
                ref, vv, ds = exact(b, h, q[b, h * G:(h + 1) * G], layer.pos - 1)
                _near(out[b, h * G:(h + 1) * G], ref, vv, dtype, ds)
    assert layer.t > 110
    # nothing kept, and a path of one's own
    layer.draft(rand(B, 2, Hq, d), k := rand(B, 2, Hkv, d), rand(B, 2, Hkv, d))
    t = layer.t
    layer.keep(torch.zeros(B, 0, dtype=torch.int32, device="cuda"))
    assert layer.t == t
    K1 = layer.K[:, :, t + 1].clone()
    layer.keep(torch.ones(B, 1, dtype=torch.int32, device="cuda"))
    assert layer.t == t + 1 and torch.equal(layer.K[:, :, t], K1)
    with pytest.raises(radar.RadarError):
        layer.draft(rand(B, 90, Hq, d), rand(B, 90, Hkv, d), rand(B, 90, Hkv, d))
    t, pos = layer.t, layer.pos
    with pytest.raises(radar.RadarError):                      # more than the cache has room for
        layer.keep(torch.arange(160 - t + 1, dtype=torch.int32, device="cuda").expand(B, -1).contiguous())
    assert (layer.t, layer.pos) == (t, pos)


def test_layer_with_axes():
    """A picture's chunk at positions of its own, text behind it, a draft, a step."""
    B, Hq, Hkv, d = 1, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    freq, _ = radar.rope_frequencies(d)
    axis = radar.rope_axes((10, 11, 11), True)
    rope = radar.Rope(freq.cuda(), axis=axis.cuda())
    cfg = radar.Config(B, Hq, Hkv, d, 64, 16, 16, 128, torch.float32)
    omega = torch.randn(64, d, generator=g, device="cuda").bfloat16().float()
    layer = radar.RadarLayer(cfg, omega, top_k=64, rope=rope)

    def rand(*s):
        return 0.5 * torch.randn(*s, generator=g, device="cuda")

    def turned(x, pos):
        """x [n][d] at pos [3][n]."""
        ang = pos.double()[axis.long().cuda()].T * freq.cuda()
        c, s, y = torch.cos(ang), torch.sin(ang), x.double()
        a, b = y[:, :d // 2], y[:, d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    k, v = rand(B, 20, Hkv, d), rand(B, 20, Hkv, d)
    i = torch.arange(20, device="cuda")
    pos = torch.stack([torch.zeros_like(i), i // 5, i % 5])[:, None].contiguous()
    layer.prefill(k, v, pos=pos, next_pos=5)
    assert (layer.t, layer.pos) == (20, 5)
    q, kd, vd = rand(B, 3, Hq, d), rand(B, 3, Hkv, d), rand(B, 3, Hkv, d)
    out = layer.draft(q, kd, vd)
    layer.keep(torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"))
    q2, k2, v2 = rand(B, Hq, d), rand(B, Hkv, d), rand(B, Hkv, d)
    out2 = layer.step(q2, k2, v2)
    assert (layer.t, layer.pos) == (23, 8)

    def text(p, n=1):
        return (p + torch.arange(n, device="cuda")).expand(3, n)

    for h in range(Hkv):
        keys = torch.cat([turned(k[0, :, h], pos[:, 0]), turned(kd[0, :, h], text(5, 3))])
        vals = torch.cat([v[0, :, h], vd[0, :, h]]).double()
        for j in range(3):
            for gq in range(2):
                qq = turned(q[0, j, 2 * h + gq][None], text(5 + j))
                ref = _attend(qq, keys[:21 + j], vals[:21 + j])[0][0]
                _near(out[0, j, 2 * h + gq], ref, vals, torch.float32, _logit_step(qq, keys, torch.float32))
        keys = torch.cat([keys[:22], turned(k2[0, h][None], text(7))])
        vals = torch.cat([vals[:22], v2[0, h][None].double()])
        for gq in range(2):
            qq = turned(q2[0, 2 * h + gq][None], text(7))
            ref = _attend(qq, keys, vals)[0][0]
            _near(out2[0, 2 * h + gq], ref, vals, torch.float32, _logit_step(qq, keys, torch.float32))
    with pytest.raises(ValueError):
        layer.draft(q, kd, vd, parent=torch.full((3,), -1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        radar.RadarLayer(cfg, omega, top_k=64).prefill(k, v, pos=pos)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ragged_run(dtype):
    """A batch of different lengths, on the device throughout: positions by depth, the
    tree's rows behind each sequence, attention, acceptance, the index, a fork; twice."""
    B, Hq, Hkv, d, cap, c, N = 3, 4, 2, 64, 200, 16, len(PARENT)
    G = Hq // Hkv
    g = torch.Generator(device="cuda").manual_seed(9)
    freq, _ = radar.rope_frequencies(d)
    rope = radar.Rope(freq.cuda())
    cfg = radar.Config(B, Hq, Hkv, d, 64, c, c, cap, dtype)
    omega = torch.randn(64, d, generator=g, device="cuda").bfloat16().float()

    def rand(*s):
        return (0.5 * torch.randn(*s, generator=g, device="cuda")).to(dtype)

    K, V = (torch.zeros(B, Hkv, cap, d, dtype=dtype, device="cuda") for _ in range(2))
    summ = radar.new_summaries(cfg, "cuda")
    lens = torch.tensor([100, 1, 57], device="cuda")
    k, v = rand(B, 100, Hkv, d), rand(B, 100, Hkv, d)
    radar.rotary_fill(cfg, rope, K, V, k, v, 0, lens=lens)
    radar.extend_index(cfg, K, omega, 0, 100, summ, lens0=torch.zeros_like(lens), lens=lens, most=100)
    parent = torch.tensor(PARENT, dtype=torch.int32, device="cuda")
    depth = torch.tensor(DEPTH, device="cuda")
    for turn in range(2):
        q, k, v = rand(B, N, Hq, d), rand(B, N, Hkv, d), rand(B, N, Hkv, d)
        pos = lens[:, None] + depth
        qr = radar.rotary_fill(cfg, rope, K, V, k, v, lens, pos=pos, q=q)
        out = radar.attend_tree(cfg, qr, K, V, 150, parent=parent, lens=lens)
        for b in range(B):
            n = int(lens[b])
            for i in range(N):
                at = list(range(n)) + [n + j for j in _above(i)]
                for h in range(Hkv):
                    ref, tol, _, _ = R.attend(qr[b, i, h * G:(h + 1) * G], K[b, h, at], V[b, h, at], dtype, N * G)
                    assert bool(((out[b, i, h * G:(h + 1) * G].double() - ref).abs() <= tol).all())
        tokens = torch.arange(N, device="cuda").expand(B, N).contiguous()
        first = torch.tensor([0, 1, 9], device="cuda")
        choice = torch.full((B, N), 99, device="cuda")
        choice[0, 0], choice[0, 2], choice[0, 5], choice[1, 1] = 2, 5, 6, 4
        was, before = lens.clone(), K.clone()
        path, found, after = radar.accept_tree(cfg, K, V, 150, tokens, first, choice, parent=parent, lens=lens, new_lens=lens)
        assert found.tolist() == [4, 2, 0] and after.tolist() == [99, 99, 9]
        assert lens.tolist() == (was + found).tolist()
        for b, rows in enumerate(([0, 2, 5, 6], [1, 4], [])):
            n = int(was[b])
            assert torch.equal(K[b, :, n:n + len(rows)], before[b][:, [n + j for j in rows]])
        radar.extend_index(cfg, K, omega, 0, 150, summ, lens0=was, lens=lens, most=N)
        if turn == 0:
            radar.fork(cfg, K, V, torch.tensor([2, 1, 0], device="cuda"), 150, lens=lens, new_lens=lens, summaries=summ)
            assert lens.tolist() == [57, 3, 104]
        fresh = radar.new_summaries(cfg, "cuda")
        radar.build_index(cfg, K, omega, 150, fresh)
        for b in range(B):
            n = int(lens[b]) // c
            assert torch.equal(summ[b, :, :n], fresh[b, :, :n])
