"""RadarLayer.keep() and accept() take in tokens of the last draft only, along a path that
ascends; what they refuse changes nothing (on the CPU: the calls that reach the GPU are
replaced)."""
import pytest
import torch

import paper_2503_10571_amd as radar

B, CAP, T = 2, 40, 20


@pytest.fixture
def layer(monkeypatch):
    """A layer of T rows that notes its calls."""
    calls = []
    for name in ("keep_path", "extend_index", "append", "append_decode"):
        monkeypatch.setattr(radar, name, lambda *a, name=name, **kw: calls.append(name))
    monkeypatch.setattr(radar, "attend_tree", lambda cfg, q, *a, **kw: q)
    monkeypatch.setattr(radar, "evict", lambda cfg, K, V, mass, t, heavy, recent, **kw: heavy + recent)
    cfg = radar.Config(B, 4, 2, 64, 64, 16, 16, CAP, torch.bfloat16)
    out = radar.RadarLayer.__new__(radar.RadarLayer)
    out.cfg, out.schedule, out.rope, out.t, out.pos = cfg, "fixed", None, T, T
    out.omega = out.summaries = None
    out.mass = torch.zeros(1)
    out.K, out.V = (torch.zeros(B, 2, CAP, 64).bfloat16() for _ in range(2))
    out._reindex = out._fit_workspace = lambda: None
    out.k, out.workspace = 4, None
    out.calls = calls
    return out


def _draft(layer, n):
    x = torch.zeros(B, n, 2, 64).bfloat16()
    layer.draft(torch.zeros(B, n, 4, 64).bfloat16(), x, x)


def _path(*rows):
    return torch.tensor(rows, dtype=torch.int32)


def _refused(layer, path, match):
    t, pos = layer.t, layer.pos
    layer.calls.clear()
    with pytest.raises(ValueError, match=match):
        layer.keep(path)
    assert (layer.t, layer.pos, layer.calls) == (t, pos, [])


@pytest.mark.parametrize("path", [
    [[0, 0], [0, 1]],                    # an entry twice
    [[0, 1], [2, 1]],                    # descends
    [[0, 1], [-1, 0]],                   # below the first
    [[3, -1], [0, 1]],                   # the end of a shorter path
    [[5, -(1 << 31)], [0, 1]],
    [[0, 1], [4, 6]],                    # a token that was not drafted
    [[6], [0]],
    [[0, (1 << 31) - 1], [0, 1]],
    [list(range(7)), list(range(7))],    # more tokens than were
])
def test_keep_refuses(layer, path):
    _draft(layer, 6)
    _refused(layer, _path(*path), "path")
    layer.keep(_path([0, 5], [1, 2]))    # the draft is still there
    assert (layer.t, layer.pos, layer.calls) == (T + 2, T + 2, ["keep_path", "extend_index"])


def test_keep_needs_a_draft(layer):
    one = _path([0], [0])
    _refused(layer, one, "drafted")
    _draft(layer, 3)
    layer.keep(_path([], []))            # nothing taken in: the rows still lie there
    layer.keep(one)
    _refused(layer, one, "drafted")      # taken in already
    x = torch.zeros(B, 1, 2, 64).bfloat16()
    for other in (lambda: layer.append(x, x), lambda: layer.step(x, x, x), lambda: layer.prefill(x, x),
                  lambda: layer.evict(4, 8)):
        _draft(layer, 3)
        other()
        _refused(layer, one, "drafted")
    _draft(layer, 3)
    with pytest.raises(ValueError):      # a chunk that is refused leaves the draft
        layer.prefill(x[:1], x[:1])
    with pytest.raises(radar.RadarError):
        _draft(layer, CAP)
    layer.evict(layer.t - 8, 8)          # nothing to cut, and a chunk of no tokens
    layer.prefill(x[:, :0], x[:, :0])
    layer.keep(one)
    _draft(layer, 3)
    with pytest.raises(radar.RadarError):        # no room in the cache at all
        layer.keep(torch.arange(CAP, dtype=torch.int32).expand(B, -1))


def test_accept(layer, monkeypatch):
    path = _path([0, 2, -1, -1], [1, 2, 3, -1])
    monkeypatch.setattr(radar, "accept_tree", lambda *a, **kw: (path, torch.tensor([2, 3]), torch.tensor([7, 8])))
    tokens = torch.arange(8).view(2, 4)
    with pytest.raises(ValueError, match="drafted"):
        layer.accept(tokens, None, None)
    _draft(layer, 3)
    with pytest.raises(ValueError, match="drafted"):
        layer.accept(tokens, None, None)
    assert (layer.t, layer.calls) == (T, [])
    seen = []

    class Layer(radar.RadarLayer):       # a subclass's keep() is called
        def keep(self, path):
            seen.append(path.tolist())
            super().keep(path)

    layer.__class__ = Layer
    _draft(layer, 4)
    n, after = layer.accept(tokens, None, None)
    assert n == 2 and after.tolist() == [7, 7] and layer.t == T + 2
    assert seen == [[[0, 2], [1, 2]]] and layer.calls == ["keep_path", "extend_index"]
    _refused(layer, _path([0, 0], [0, 1]), "path")


def test_fork_takes_a_draft_along(layer, monkeypatch):
    seen = []
    monkeypatch.setattr(radar, "fork", lambda cfg, K, V, src, t, first=0, **kw: seen.append((t, first)))
    layer.fork("src")
    _draft(layer, 5)
    layer.fork("src", first=3)
    layer.fork("src", first=T + 2)       # rows below `first`: the cache's at most
    layer.keep(_path([0, 4], [1, 2]))
    layer.fork("src")
    assert seen == [(T, 0), (T + 5, 3), (T + 5, T), (T + 2, 0)]
