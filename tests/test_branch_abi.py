"""The C ABI of the operators for drafted tokens, forking and positions on several
axes on the CPU: bad arguments get the documented status before anything reaches
the GPU, and the binding refuses tensors of the host."""
import ctypes
import os

import pytest
import torch

import paper_2503_10571_amd as radar
from paper_2503_10571_amd import _build, cache_ops

P = ctypes.c_void_p
GOOD, ODD, OFF = P(0x1000), P(0x1008), P(0x1002)
by = ctypes.byref


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(radar.LIB_PATH):
        _build.build_library()
    return radar.lib()


def _cfg(**kw):
    base = dict(batch=8, n_q_heads=32, n_kv_heads=8, head_dim=128, n_features=256, seg_len=256,
                window=256, capacity=4096)
    base.update(kw)
    return radar.Config(**base).c_struct()


BAD = [(dict(batch=0), 1), (dict(n_q_heads=30), 1), (dict(capacity=0), 1), (dict(n_sink=-1), 1),
       (dict(n_sink=4097), 1), (dict(n_q_heads=24), 3), (dict(head_dim=96), 3),
       (dict(capacity=1 << 31), 3), (dict(batch=9000), 3)]
BAD_INDEX = [(dict(seg_len=0), 1), (dict(n_features=100), 3), (dict(n_features=4096), 3)]


def test_axes_refusals(L):
    rope = cache_ops._Rope(128, 0, 1.0, 0x1000)
    rows = cache_ops._Rows(0x1000, 4096, 4096, 128)

    def call(rope=by(rope), axes=3, axis=GOOD, batch=2, tokens=3, d=128, dtype=1, hq=4, q=by(rows), qo=by(rows),
             hk=2, k=by(rows), ko=by(rows), pos=GOOD, lens=None):
        return L.radar_rotary_axes(rope, axes, axis, batch, tokens, d, dtype, hq, q, qo, hk, k, ko, pos, lens, 0, None)

    assert call(axes=0) == 1 and call(axes=-1) == 1
    assert call(axis=None) == 1 and call(axis=OFF) == 1 and call(pos=None) == 1 and call(pos=P(0x1004)) == 1
    assert call(rope=None) == 1 and call(dtype=2) == 1 and call(d=136) == 3 and call(d=272) == 3
    assert call(batch=0) == 1 and call(tokens=-1) == 1 and call(tokens=1 << 31) == 3
    assert call(q=None) == 1 and call(ko=None) == 1 and call(lens=ODD) == 1
    assert call(tokens=0) == 0

    def fill(cfg=_cfg(), axes=2, axis=GOOD, tokens=3, q=None, qo=None, k=by(rows), v=by(rows), K=GOOD, V=GOOD, row0=0,
             rows_=None, pos=GOOD, lens=None):
        return L.radar_rotary_fill_axes(by(cfg), by(rope), axes, axis, tokens, q, qo, k, v, K, V, row0, rows_, pos, lens,
                                        None)

    for kw, want in BAD:
        assert fill(cfg=_cfg(**kw)) == want, kw
    assert fill(axes=0) == 1 and fill(axis=OFF) == 1 and fill(pos=None) == 1
    assert fill(row0=-1) == 2 and fill(row0=4094) == 2 and fill(K=None) == 1 and fill(rows_=ODD) == 1
    assert fill(tokens=0) == 0


def test_tree_refusals(L):
    rows = by(cache_ops._Rows(0x1000, 32768, 4096, 128))

    def call(cfg=_cfg(), q=rows, K=GOOD, V=GOOD, t=100, lens=None, nodes=9, counts=None, parent=GOOD, out=rows, ws=GOOD,
             n=1 << 30):
        return L.radar_attend_tree(by(cfg), q, K, V, t, lens, nodes, counts, parent, 0, out, ws, n, None)

    for kw, want in BAD:
        assert call(cfg=_cfg(**kw)) == want, kw
    assert call(nodes=0) == 1 and call(nodes=513) == 3 and call(nodes=4097, parent=None) == 2
    assert call(cfg=_cfg(capacity=1 << 20), nodes=1 << 19, parent=None) == 3       # 2^27 query rows
    assert call(t=-1) == 2 and call(t=4097) == 2 and call(t=4090) == 2 and call(t=4097, lens=GOOD) == 2
    for name in ("q", "K", "V", "out"):
        assert call(**{name: None}) == 1, name
    for name in ("K", "V"):
        assert call(**{name: ODD}) == 1, name
    for name in ("lens", "counts", "parent"):
        assert call(**{name: OFF}) == 1, name
    for bad in ((0, 0, 0, 128), (0x1008, 4096, 4096, 128), (0x1000, 4, 4096, 128), (0x1000, 4096, 4, 128),
                (0x1000, 4096, 4096, 4)):
        assert call(q=by(cache_ops._Rows(*bad))) == 1 and call(out=by(cache_ops._Rows(*bad))) == 1, bad
    need = L.radar_attend_tree_workspace_bytes(by(_cfg()), 9, 100)
    assert need > 0 and call(n=need - 1) == 5 and call(ws=None) == 5 and call(ws=ODD) == 5
    for nodes, t in ((0, 100), (9, -1), (9, 4097), (4097, 0)):
        assert L.radar_attend_tree_workspace_bytes(by(_cfg()), nodes, t) == 0
    assert L.radar_attend_tree_workspace_bytes(by(_cfg(head_dim=96)), 9, 100) == 0


def test_tree_flags(L):
    """Shared, zeros behind the nodes, both; no others."""
    rows = by(cache_ops._Rows(0x1000, 32768, 4096, 128))
    for flags in (4, 8, 7, -1, 1 << 31 - 1):
        assert L.radar_attend_tree(by(_cfg()), rows, GOOD, GOOD, 100, None, 9, None, GOOD, flags, rows, GOOD, 1 << 30,
                                   None) == 1, flags
    for flags in (0, 1, 2, 3):                                   # (as far as the workspace)
        assert L.radar_attend_tree(by(_cfg()), rows, GOOD, GOOD, 100, None, 9, None, GOOD, flags, rows, GOOD, 0,
                                   None) == 5, flags


def test_accept_refusals(L):
    def call(cfg=_cfg(), K=GOOD, V=GOOD, t=100, lens=None, nodes=9, counts=None, parent=GOOD, tokens=GOOD, first=GOOD,
             choice=GOOD, path=GOOD, accepted=GOOD, nxt=GOOD, new=None):
        return L.radar_accept_tree(by(cfg), K, V, t, lens, nodes, counts, parent, 0, tokens, first, choice, path,
                                   accepted, nxt, new, None)

    for kw, want in BAD:
        assert call(cfg=_cfg(**kw)) == want, kw
    assert call(nodes=0) == 1 and call(nodes=513) == 3
    assert call(t=-1) == 2 and call(t=4097) == 2 and call(t=4090) == 2
    assert call(t=4097, lens=GOOD) == 2
    for name in ("tokens", "first", "choice", "path", "accepted", "nxt"):
        assert call(**{name: None}) == 1 and call(**{name: OFF}) == 1, name
    for name in ("lens", "counts", "parent", "new"):
        assert call(**{name: OFF}) == 1, name
    assert call(K=ODD) == 1 and call(tokens=P(0x1004)) == 1 and call(V=ODD) == 1
    assert call(K=None, V=GOOD) == 1 and call(V=None) == 1
    assert call(lens=GOOD, new=ODD) == 1 and call(nxt=ODD) == 1


def test_keep_refusals(L):
    def call(cfg=_cfg(), K=GOOD, V=GOOD, t=100, lens=None, path=GOOD, n=9, counts=None, new=None):
        return L.radar_keep_path(by(cfg), K, V, t, lens, path, n, counts, new, None)

    for kw, want in BAD:
        assert call(cfg=_cfg(**kw)) == want, kw
    assert call(n=-1) == 1 and call(n=4097) == 2 and call(t=-1) == 2 and call(t=4097) == 2
    for name in ("K", "V", "path"):
        assert call(**{name: None}) == 1 and call(**{name: OFF}) == 1, name
    for name in ("lens", "counts", "new"):
        assert call(**{name: OFF}) == 1, name
    assert call(V=ODD) == 1
    assert call(lens=GOOD, new=P(0x1038)) == 1 and call(lens=P(0x1038), new=GOOD) == 1   # over a part of the other


def test_extend_index_refusals(L):
    def call(cfg=_cfg(), K=GOOD, omega=GOOD, t0=0, t=100, lens0=None, lens=None, most=50, summ=GOOD, ws=GOOD, n=1 << 20):
        return L.radar_extend_index(by(cfg), K, omega, t0, t, lens0, lens, most, summ, ws, n, None)

    for kw, want in BAD + BAD_INDEX + [(dict(omega_dtype=torch.bfloat16, dtype=torch.float32), 1)]:
        assert call(cfg=_cfg(**kw)) == want, kw
    assert call(t0=-1) == 2 and call(t0=101) == 2 and call(t=4097) == 2
    for name in ("K", "omega", "summ"):
        assert call(**{name: None}) == 1 and call(**{name: ODD}) == 1, name
    assert call(lens=GOOD) == 1 and call(lens0=GOOD) == 1 and call(lens0=OFF, lens=GOOD) == 1
    assert call(t=255) == 0 and call(t0=256, t=511) == 0         # no segment ends there
    ragged = dict(lens0=GOOD, lens=GOOD)
    assert call(most=-1, **ragged) == 2 and call(most=4097, **ragged) == 2
    need = L.radar_extend_index_workspace_bytes(by(_cfg()), 600)
    assert need == 256                                           # 3 rows of 8 lengths
    assert L.radar_extend_index_workspace_bytes(by(_cfg(seg_len=1)), 600) == 600 * 8 * 8
    assert call(most=600, ws=None, **ragged) == 5 and call(most=600, ws=ODD, **ragged) == 5
    assert call(most=600, n=need - 1, **ragged) == 5
    assert call(most=0, **ragged) == 0
    assert L.radar_extend_index_workspace_bytes(by(_cfg()), -1) == 0
    assert L.radar_extend_index_workspace_bytes(by(_cfg(seg_len=0)), 1) == 0


def test_fork_refusals(L):
    def call(cfg=_cfg(), K=GOOD, V=GOOD, mass=None, summ=None, src=GOOD, first=0, t=100, lens=None, new=None):
        return L.radar_fork(by(cfg), K, V, mass, summ, src, first, t, lens, new, None)

    for kw, want in BAD:
        assert call(cfg=_cfg(**kw)) == want, kw
    for kw, want in BAD_INDEX:
        assert call(cfg=_cfg(**kw), summ=GOOD) == want, kw
    assert call(cfg=_cfg(batch=2049, n_kv_heads=8)) == 3
    assert call(first=-1) == 1 and call(t=-1) == 2 and call(t=4097) == 2
    for name in ("K", "V", "src"):
        assert call(**{name: None}) == 1 and call(**{name: OFF}) == 1, name
    for name in ("mass", "summ", "lens", "new"):
        assert call(**{name: OFF}) == 1, name
    assert call(K=ODD) == 1 and call(mass=ODD) == 1 and call(summ=ODD) == 1
    assert call(new=GOOD) == 1                                   # the new lengths over the map
    assert call(new=ODD) == 1 and call(src=P(0x2000), lens=GOOD, new=P(0x1038)) == 1     # or over a part of a list


def test_what_moves_in_place_shares_no_memory(L):
    """Caches, masses or summaries over one another, by one address or by the last 16
    bytes: refused, before a lane is sent over them."""
    n = 8 * 8 * 4096                                             # rows; 128 bf16 each
    far = 0x1000 + n * 256
    accept = dict(t=100, tail=(None, 9, None, GOOD, 0, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, None, None))
    for K, V in ((0x1000, 0x1000), (0x1000, far - 16), (far - 16, 0x1000)):
        assert L.radar_accept_tree(by(_cfg()), P(K), P(V), accept["t"], *accept["tail"]) == 1
        assert L.radar_keep_path(by(_cfg()), P(K), P(V), 100, None, GOOD, 9, None, None, None) == 1
        assert L.radar_fork(by(_cfg()), P(K), P(V), None, None, GOOD, 0, 100, None, None, None) == 1
    end = far + n * 256                                          # of V
    summ = 8 * 8 * 16 * 256 * 4
    for mass, at in ((0x1000, None), (far, None), (end - 16, None), (None, 0x1000), (None, end - 16), (end, end),
                     (end, end + n * 4 - 16), (end + summ - 16, end)):
        assert L.radar_fork(by(_cfg()), P(0x1000), P(far), P(mass), P(at), GOOD, 0, 100, None, None, None) == 1, (mass, at)


def test_binding_refuses_host_tensors(L):
    cfg = radar.Config(1, 1, 1, 64, 64, 16, 16, 32)
    K = torch.zeros(1, 1, 32, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, 1, dtype=torch.int64)
    with pytest.raises(ValueError):
        radar.accept_tree(cfg, K, K, 1, i, i[0], i)
    with pytest.raises(ValueError):
        radar.keep_path(cfg, K, K, 1, i.int())
    with pytest.raises(ValueError):
        radar.fork(cfg, K, K, i[0], 1)
    with pytest.raises(ValueError):
        radar.extend_index(cfg, K, torch.zeros(64, 64), 0, 1, torch.zeros(1, 1, 2, 64))
    with pytest.raises(ValueError):
        radar.Rope(torch.zeros(32, dtype=torch.float64), axis=torch.zeros(32, dtype=torch.int32))


@pytest.mark.parametrize("sections,cycled,want", [
    ((2, 3), False, [0, 0, 1, 1, 1]), ((2, 3), True, [0, 1, 0, 1, 1]), ((1, 0, 2), True, [0, 2, 2]),
    ((1, 0, 2), False, [0, 2, 2]), ((4,), True, [0, 0, 0, 0])])
def test_rope_axes(sections, cycled, want):
    got = radar.rope_axes(sections, cycled)
    assert got.dtype == torch.int32 and got.tolist() == want


@pytest.mark.parametrize("bad", [(), (0,), (2, -1)])
def test_rope_axes_refuses(bad):
    with pytest.raises(ValueError):
        radar.rope_axes(bad)
