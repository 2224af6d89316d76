"""The operators around drafted tokens and branching sequences that speed is
measured on: rotary positions on several axes, attention of a tree (or chain)
of drafted tokens over the cache, the acceptance of one of its paths, and the
forking of the caches' sequences.

A case is one call. `own` False: the operators in elementary torch operations;
True: the calls of the package.

Fields of a case:
  op        "axes", "tree", "accept" or "fork"
  B, Hq, Hkv, d   batch, query heads, kv heads, head dim
  dtype     "bf16" or "f32" (everything but masses, summaries, positions, frequencies)
  ragged    sequences of different lengths
axes (q and k as slices of one projection; fill: q, k, v into the cache):
  T         tokens per sequence (ragged: of the longest)
  A         axes of the positions
  rot       rotated dims of the head
  cycled    pair i belongs to axis i mod A, instead of A runs of pairs
  inter     pairs (2i, 2i + 1) instead of (i, i + rot / 2)
  fill      into the cache
  inverse   rotate back (the gradient of the rotation)
tree, accept:
  t         rows in the cache before the drafted ones (ragged: of the longest)
  N         drafted tokens per sequence (ragged: the most)
  kind      "tree": one tree for the batch, "trees": one per sequence, "chain"
fork:
  t         rows in the cache (ragged: of the longest)
  first     rows that all sequences have in common, not moved
  kind      "samples": the first sequence's rows for all; "beams": each from any;
            "live": the ended ones' places are taken by those behind them
  extra     the rows' masses and the index's summaries move too
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0
SPARE = 64                                # free rows behind the filled ones
VOCAB = 32000
SEG, FEATURES = 256, 256                  # segment length and features of the summaries


def _axes(name, B, T, Hq, Hkv, d, rot, A, cycled=False, inter=False, fill=False, inverse=False,
          ragged=False, dtype="bf16"):
    c = dict(op="axes", B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, rot=rot, A=A, cycled=cycled, inter=inter,
             fill=fill, inverse=inverse, ragged=ragged, dtype=dtype)
    return dict(c, name=name) if name else c


def _tree(name, B, Hq, Hkv, d, t, N, kind, ragged=False, dtype="bf16"):
    c = dict(op="tree", B=B, Hq=Hq, Hkv=Hkv, d=d, t=t, N=N, kind=kind, ragged=ragged, dtype=dtype)
    return dict(c, name=name) if name else c


def _accept(name, B, Hkv, d, t, N, kind, ragged=False, dtype="bf16"):
    c = dict(op="accept", B=B, Hkv=Hkv, d=d, t=t, N=N, kind=kind, ragged=ragged, dtype=dtype)
    return dict(c, name=name) if name else c


def _fork(name, B, Hkv, d, t, kind, first=0, extra=False, ragged=False, dtype="bf16"):
    c = dict(op="fork", B=B, Hkv=Hkv, d=d, t=t, kind=kind, first=first, extra=extra, ragged=ragged,
             dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step's new query and key behind a picture: latency
        _axes("axes_step", 1, 1, 32, 8, 128, 128, 3),
        # two clips of different lengths on their way into the cache
        _axes("axes_fill", 2, 8003, 32, 8, 128, 128, 3, cycled=True, fill=True, ragged=True),
        # the gradient over a batch of pictures, 32 bits, part of the head, odd length
        _axes("axes_back_f32", 2, 4095, 16, 4, 64, 48, 2, inter=True, inverse=True, dtype="f32"),
        # a few guesses behind a short prompt: the smallest attention, latency
        _tree("tree_small", 1, 8, 2, 64, 500, 7, "tree"),
        # eight conversations, each with a tree of its own
        _tree("tree_gqa", 8, 32, 8, 128, 16411, 32, "trees", ragged=True),
        # one long context and a large tree: many query rows, matrix-bound
        _tree("tree_long", 1, 32, 8, 128, 65536, 64, "tree"),
        # multi-head in 32 bits, odd sizes
        _tree("tree_f32", 2, 16, 16, 128, 4097, 25, "trees", ragged=True, dtype="f32"),
        # a chunk of a prompt behind what is in the cache: the largest product
        _tree("chain_chunk", 1, 32, 8, 128, 8000, 1500, "chain"),
        # one sequence's step: the path and its few rows, latency
        _accept("accept_one", 1, 8, 128, 3000, 26, "tree"),
        # a batch with large trees
        _accept("accept_batch", 64, 8, 128, 1001, 63, "trees", ragged=True),
        # one prompt's cache for eight samples
        _fork("fork_samples", 8, 8, 128, 16411, "samples"),
        # beams behind a common prompt, with masses and summaries
        _fork("fork_beams", 16, 16, 64, 3001, "beams", first=1000, extra=True, ragged=True, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call over the ranges of the listed ones: one to 32K new tokens
    of one to four axes, caches of one to 64K rows, trees of one to 256 nodes,
    chains of up to 2000, batches of 1 to 64, groups of 1 to 8; most of it in
    bf16 at head dim 128."""
    while True:
        op = rng.choice(["axes", "tree", "tree", "tree", "accept", "fork"])
        dtype = rng.choice(["bf16"] * 4 + ["f32"])
        d = rng.choice([128, 128, 128, 64])
        G, Hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([1, 2, 4, 8, 8, 16, 32])
        ragged = rng.random() < 0.4
        if op == "axes":
            fill = rng.random() < 0.5
            c = _axes(None, _log_uniform(rng, 1, 16), _log_uniform(rng, 1, 32768), G * Hkv, Hkv, d,
                      rng.choice([d, d, d // 2, d * 3 // 4, d // 4]), rng.choice([1, 2, 2, 3, 3, 3, 4]),
                      rng.random() < 0.5, rng.random() < 0.5, fill, not fill and rng.random() < 0.5,
                      fill and ragged, dtype)
        elif op == "tree":
            kind = rng.choice(["tree", "trees", "trees", "chain"])
            c = _tree(None, _log_uniform(rng, 1, 32), G * Hkv, Hkv, d, _log_uniform(rng, 1, 65536),
                      _log_uniform(rng, 1, 2000 if kind == "chain" else 256), kind, ragged, dtype)
            if c["B"] * c["Hq"] * c["N"] * (c["t"] + c["N"]) > (32 * 1500 * 9500 if dtype == "bf16" else 1 << 26):
                continue
        elif op == "accept":
            c = _accept(None, _log_uniform(rng, 1, 64), Hkv, d, _log_uniform(rng, 1, 16384),
                        _log_uniform(rng, 1, 256), rng.choice(["tree", "trees", "chain"]), ragged, dtype)
        else:
            t = _log_uniform(rng, 1, 65536)
            c = _fork(None, _log_uniform(rng, 2, 64), Hkv, d, t, rng.choice(["samples", "beams", "live"]),
                      rng.choice([0, 0, t // 3]), rng.random() < 0.5, ragged, dtype)
        if work(c)["bytes"] > 5.3e8 or c["B"] * Hkv * d * c.get("t", 0) > 3e8:
            continue
        return c


# ---- shapes -----------------------------------------------------------------
def _lengths(case):
    """Tokens (rows) of every sequence."""
    B, n = case["B"], case.get("T") or case["t"]
    if not case["ragged"]:
        return [n] * B
    return [max(1, n - (n * b) // B) for b in range(B)]


def _counts(case):
    """Drafted tokens of every sequence."""
    B, N = case["B"], case["N"]
    if not case["ragged"] or case["kind"] != "trees":
        return [N] * B
    return [max(1, N - (N * ((5 * b + 3) % B)) // (2 * B)) for b in range(B)]


def _sources(case):
    """The sequence that each one's rows come from, -1: it has ended."""
    B, rng = case["B"], random.Random(case["B"] * 65537 + case["t"])
    if case["kind"] == "samples":
        return [0] * B
    if case["kind"] == "beams":
        return [rng.randrange(B) for _ in range(B)]
    live = [b for b in range(B) if rng.random() < 0.6]
    return live + [-1] * (B - len(live))


def work(case):
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    Hq, size = case.get("Hq", 0), 2 if case["dtype"] == "bf16" else 4
    lens = _lengths(case)
    if case["op"] == "axes":
        n = sum(lens)
        rows = n * (Hq + Hkv * (2 if case["fill"] else 1))
        return {"bytes": 2 * rows * d * size + 8 * case["A"] * n,
                "flops": 3.0 * n * (Hq + Hkv) * case["rot"]}
    if case["op"] == "tree":
        counts = _counts(case)
        seen = sum(n * m + (m * (m + 1) // 2 if case["kind"] == "chain" else m)
                   for n, m in zip(lens, counts))
        return {"bytes": 2 * sum(Hkv * (n + m) + Hq * m for n, m in zip(lens, counts)) * d * size,
                "flops": 4.0 * Hq * d * seen}
    if case["op"] == "accept":
        # parents, tokens and choices read, paths written; an accepted row or two moved
        return {"bytes": B * (case["N"] * (4 + 8 + 8 + 4) + 2 * 2 * 2 * Hkv * d * size), "flops": float(B * case["N"])}
    src, per = _sources(case), Hkv * 2 * d * size
    moved = [s for b, s in enumerate(src) if s >= 0 and s != b]
    total = sum(max(0, lens[s] - case["first"]) * per for s in moved + sorted(set(moved)))
    if case["extra"]:
        each = {s: Hkv * (lens[s] * 4 + max(0, lens[s] // SEG - case["first"] // SEG) * FEATURES * 4)
                for s in set(moved)}
        total += sum(each[s] for s in moved + sorted(set(moved)))
    return {"bytes": total + 8 * B, "flops": 0.0}


# ---- inputs -----------------------------------------------------------------
def _frequencies(case):
    """Angle per position of every pair, in 64 bits."""
    r = case["rot"]
    return BASE ** (-2.0 * torch.arange(r // 2, dtype=torch.float64) / r)


def _axis_of(case):
    """The axis of every pair: in turn, or runs whose lengths differ by one at most."""
    pairs, A = case["rot"] // 2, case["A"]
    return [i % A if case["cycled"] else i * A // pairs for i in range(pairs)]


def _parents(case, g):
    """[B][N] int32: node i hangs on one of the few before it, or is a root (-1)."""
    B, N = case["B"], case["N"]
    rows = 1 if case["kind"] == "tree" else B
    i = torch.arange(N, device="cuda")
    if case["kind"] == "chain":
        return (i - 1).int().expand(B, N).contiguous()
    back = torch.rand(rows, N, generator=g, device="cuda") * torch.clamp(i + 1, max=2 * math.isqrt(N) + 2)
    return (i - 1 - back.long()).int().expand(B, N).contiguous()


def prepare(case, seed):
    B, Hkv, d, dtype = case["B"], case["Hkv"], case["d"], DTYPES[case["dtype"]]
    Hq, op = case.get("Hq", case["Hkv"]), case["op"]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=dtype)
        return x * scale if scale != 1.0 else x

    s = dict(case=case)
    lens = _lengths(case)
    s["lens"] = torch.tensor(lens, device="cuda") if case["ragged"] else None
    if op == "axes":
        # q, k (and v): slices of one projection's output, as it leaves a product
        T, heads = case["T"], Hq + Hkv * (2 if case["fill"] else 1)
        qkv = normal(B, T, heads, d)
        s["q"], s["k"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
        s["freq"] = _frequencies(case).cuda()
        s["axis"] = torch.tensor(_axis_of(case), dtype=torch.int32, device="cuda")
        # frames of up to 1000 places, one after the other
        side = [1 << 30, 31, 33, 7]
        at = torch.arange(T, device="cuda") + torch.randint(0, 100000, (B, 1), generator=g, device="cuda")
        pos = [at // 1023] + [at // (1 if a == 1 else 31 if a == 2 else 5) % side[a] for a in range(1, case["A"])]
        s["pos"] = torch.stack(pos).contiguous()
        cap = T + SPARE
        if case["fill"]:
            s["v"] = qkv[:, :, Hq + Hkv:]
            s["K"], s["V"] = normal(B, Hkv, cap, d), normal(B, Hkv, cap, d)
            s["qo"] = torch.zeros(B, T, Hq, d, device="cuda", dtype=dtype)
    else:
        cap = case["t"] + case.get("N", 0) + SPARE
        s["K"], s["V"] = normal(B, Hkv, cap, d), normal(B, Hkv, cap, d)
    if op in ("tree", "accept"):
        s["parent"] = _parents(case, g)
        counts = _counts(case)
        s["counts"] = torch.tensor(counts, device="cuda") if min(counts) < case["N"] else None
        # as the calls take it: one list for the batch, one for each sequence, or none
        s["links"] = {"tree": s["parent"][0], "trees": s["parent"], "chain": None}[case["kind"]]
    if op == "tree":
        # logits of standard deviation 2: weights from nothing to some percent
        s["q"] = normal(B, case["N"], Hq, d, scale=2.0)
    elif op == "accept":
        # tokens guessed, and the model's own: often that of a guess behind it
        N, parent = case["N"], s["parent"].long()
        s["tokens"] = torch.randint(0, VOCAB, (B, N), generator=g, device="cuda")
        child = torch.full((B, N + 1), -1, device="cuda").scatter_reduce(
            1, parent + 1, torch.arange(N, device="cuda").expand(B, N), "amax")
        hit = (torch.rand(B, N + 1, generator=g, device="cuda") < 0.8) & (child >= 0)
        other = torch.randint(0, VOCAB, (B, N + 1), generator=g, device="cuda")
        picked = torch.where(hit, s["tokens"].gather(1, child.clamp(min=0)), other)
        s["first"], s["choice"] = picked[:, 0].contiguous(), picked[:, 1:].contiguous()
    elif op == "fork":
        s["src"] = torch.tensor(_sources(case), device="cuda")
        s["mass"] = s["summ"] = None
        if case["extra"]:
            s["mass"] = torch.rand(B, Hkv, cap, generator=g, device="cuda")
            s["summ"] = torch.rand(B, Hkv, max(1, cap // SEG), FEATURES, generator=g, device="cuda")
    if own:                               # what a program holds beside its tensors
        import paper_2503_10571_amd as radar
        s["cfg"] = radar.Config(B, Hq, Hkv, d, FEATURES, SEG, SEG, cap, dtype)
        if op == "axes":
            s["rope"] = radar.Rope(s["freq"], interleaved=case["inter"], axis=s["axis"])
    return s


# ---- the plain forms ----------------------------------------------------------
def _turned(x, s):
    """x [B][T][H][d] rotated, in 32 bits; the angles in 64."""
    c, freq = s["case"], s["freq"]
    rot = 2 * freq.numel()
    angle = s["pos"][s["axis"].long()].permute(1, 2, 0).double() * freq          # [B][T][pairs]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if c["inverse"]:
        sin = -sin
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["inter"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if c["inter"] else torch.cat((u, w), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _plain_axes(s):
    c = s["case"]
    q, k = _turned(s["q"], s), _turned(s["k"], s)
    if not c["fill"]:
        return {"q": q, "k": k}
    T = c["T"]
    K, V, qo = s["K"][:, :, :T], s["V"][:, :, :T], s["qo"]
    k, v = k.transpose(1, 2), s["v"].transpose(1, 2)
    if s["lens"] is not None:
        on = torch.arange(T, device="cuda") < s["lens"][:, None]
        k, v = torch.where(on[:, None, :, None], k, K), torch.where(on[:, None, :, None], v, V)
        q = torch.where(on[:, :, None, None], q, qo)
    K.copy_(k)
    V.copy_(v)
    qo.copy_(q)
    return {"q": qo, "K": s["K"], "V": s["V"]}


def _ancestors(parent):
    """[B][N][N]: whether node j is node i or above it. In each round the set of
    a node takes in that of the node that it points to, and the pointer doubles."""
    B, N = parent.shape
    up = torch.eye(N, device="cuda", dtype=torch.bool).expand(B, N, N)
    # a place behind the nodes stands for none: its set is empty, it points to itself
    up = torch.cat([up, up.new_zeros(B, 1, N)], 1)
    at = torch.cat([torch.where(parent < 0, N, parent.long()), parent.new_full((B, 1), N).long()], 1)
    for _ in range(max(1, (N - 1).bit_length())):
        up = up | up.gather(1, at[..., None].expand(-1, -1, N))
        at = at.gather(1, at)
    return up[:, :N]


def _plain_tree(s):
    c = s["case"]
    B, Hq, Hkv, d, t, N = c["B"], c["Hq"], c["Hkv"], c["d"], c["t"], c["N"]
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), t, device="cuda")
    at = torch.arange(t + N, device="cuda")
    node = at - lens[:, None]                                   # of a row, [B][t + N]
    if c["kind"] == "chain":
        mine = node[:, None] <= torch.arange(N, device="cuda")[:, None]
    else:
        up = _ancestors(s["parent"])
        mine = up.gather(2, node.clamp(0, N - 1)[:, None].expand(B, N, t + N)) & (node < N)[:, None]
    on = (node < 0)[:, None] | mine                             # [B][N][t + N]
    q = s["q"].view(B, N, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    K, V = s["K"][:, :, :t + N], s["V"][:, :, :t + N]
    x = torch.matmul(q.float(), K.float().transpose(-1, -2).contiguous()) / math.sqrt(d)
    x = x.view(B, Hkv, -1, N, t + N).masked_fill(~on[:, None, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, -1, t + N), V.float())
    out = out.view(B, Hkv, -1, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, Hq, d).to(s["q"].dtype)
    if s["counts"] is not None:                                 # nothing behind the last node
        here = torch.arange(N, device="cuda") < s["counts"][:, None]
        out = torch.where(here[..., None, None], out, torch.zeros_like(out))
    return out


def _plain_accept(s):
    c = s["case"]
    B, t, N, d = c["B"], c["t"], c["N"], c["d"]
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), t, device="cuda")
    counts = s["counts"] if s["counts"] is not None else torch.full((B,), N, device="cuda")
    node = torch.arange(N, device="cuda")
    real, parent = node < counts[:, None], s["parent"].long()
    cur, want = torch.full((B,), -1, device="cuda"), s["first"]
    path, going = [], torch.ones(B, dtype=torch.bool, device="cuda")
    for _ in range(N):
        fits = real & (parent == cur[:, None]) & (s["tokens"] == want[:, None])
        got = torch.where(fits, node, N).amin(1)
        going = going & (got < N)
        cur = torch.where(going, got, cur)
        want = torch.where(going, s["choice"].gather(1, cur.clamp(min=0)[:, None])[:, 0], want)
        path.append(torch.where(going, cur, -1))
    path = torch.stack(path, 1)
    n = (path >= 0).sum(1)
    # rows of the path to the front of the drafted ones
    at = lens[:, None] + node
    frm = torch.where(path >= 0, lens[:, None] + path, at)
    to = at[:, None, :, None].expand(-1, c["Hkv"], -1, d)
    frm = frm[:, None, :, None].expand(-1, c["Hkv"], -1, d)
    for x in (s["K"], s["V"]):
        x.scatter_(2, to, x.gather(2, frm))
    return {"K": s["K"], "V": s["V"], "path": path.int(), "accepted": n, "next": want, "lens": lens + n}


def _plain_fork(s):
    c = s["case"]
    B, t = c["B"], c["t"]
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), t, device="cuda")
    src = s["src"]
    frm = torch.where(src >= 0, src, torch.arange(B, device="cuda"))
    n = torch.where(src >= 0, lens[frm], 0)                     # new lengths
    rows = torch.arange(t, device="cuda")
    on = ((rows < n[:, None]) & (rows >= c["first"]))[:, None, :, None]
    for x in (s["K"], s["V"]):
        x[:, :, :t] = torch.where(on, x[frm, :, :t], x[:, :, :t])
    if c["extra"]:
        mass, on = s["mass"], (rows < n[:, None])[:, None]
        gone = ((rows >= n[:, None]) & (rows < lens[:, None]))[:, None]
        moved = torch.where(on, mass[frm, :, :t], mass[:, :, :t])
        mass[:, :, :t] = torch.where(gone, 0.0, moved)
        m = s["summ"].shape[2]
        seg = torch.arange(m, device="cuda")
        on = ((seg >= c["first"] // SEG) & (seg < n[:, None] // SEG))[:, None, :, None]
        s["summ"].copy_(torch.where(on, s["summ"][frm], s["summ"]))
    return {"K": s["K"], "V": s["V"], "mass": s["mass"], "summ": s["summ"], "lens": n}


# ---- the package's calls --------------------------------------------------------
def _own(s):
    import paper_2503_10571_amd as radar
    c, cfg = s["case"], s["cfg"]
    if c["op"] == "axes":
        if c["fill"]:
            q = radar.rotary_fill(cfg, s["rope"], s["K"], s["V"], s["k"], s["v"], 0, pos=s["pos"],
                                  q=s["q"], q_out=s["qo"], lens=s["lens"])
            return {"q": q, "K": s["K"], "V": s["V"]}
        q, k = radar.rotary_qk(s["rope"], s["q"], s["k"], s["pos"], inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "tree":
        return radar.attend_tree(cfg, s["q"], s["K"], s["V"], c["t"], parent=s["links"], counts=s["counts"],
                                 lens=s["lens"])
    if c["op"] == "accept":
        lens = torch.empty(c["B"], dtype=torch.int64, device="cuda")
        path, n, token = radar.accept_tree(cfg, s["K"], s["V"], c["t"], s["tokens"], s["first"],
                                           s["choice"], parent=s["links"], counts=s["counts"],
                                           lens=s["lens"], new_lens=lens)
        return {"K": s["K"], "V": s["V"], "path": path, "accepted": n, "next": token, "lens": lens}
    lens = torch.empty(c["B"], dtype=torch.int64, device="cuda")
    radar.fork(cfg, s["K"], s["V"], s["src"], c["t"], first=c["first"], lens=s["lens"], new_lens=lens,
               mass=s["mass"], summaries=s["summ"])
    return {"K": s["K"], "V": s["V"], "mass": s["mass"], "summ": s["summ"], "lens": lens}


PLAIN = {"axes": _plain_axes, "tree": _plain_tree, "accept": _plain_accept, "fork": _plain_fork}


def run(s):
    if own:
        return _own(s)
    return PLAIN[s["case"]["op"]](s)


# ---- what the outputs are, in 64 bits -------------------------------------------
def _exact_turn(x, s):
    """One complex product per pair."""
    case = s["case"]
    r = case["rot"]
    f = _frequencies(case).cuda()
    turn = torch.empty(*x.shape[:2], r // 2, dtype=torch.complex128, device="cuda")
    for i, a in enumerate(_axis_of(case)):
        p = s["pos"][a].double() * f[i]
        turn[..., i] = torch.polar(torch.ones_like(p), -p if case["inverse"] else p)
    turn = turn[:, :, None]
    out = x.double()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if case["inter"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(out[..., one], out[..., two]) * turn
    out[..., one], out[..., two] = z.real, z.imag
    return out


def _exact_axes(case, s):
    q, k = _exact_turn(s["q"], s), _exact_turn(s["k"], s)
    if not case["fill"]:
        return {"q": q, "k": k}
    K, V, qo = s["K"].double(), s["V"].double(), s["qo"].double()
    for b, n in enumerate(_lengths(case)):
        K[b, :, :n], V[b, :, :n] = k[b, :n].transpose(0, 1), s["v"][b, :n].double().transpose(0, 1)
        qo[b, :n] = q[b, :n]
    return {"q": qo, "K": K, "V": V}


def _chains(parent):
    """Every node's list of itself and the nodes above it."""
    out = []
    for i, p in enumerate(parent):
        out.append([i] if p < 0 else out[p] + [i])
    return out


def _exact_tree(case, s):
    Hkv, d, N = case["Hkv"], case["d"], case["N"]
    G = case["Hq"] // Hkv
    if case["B"] * case["Hq"] * N * (case["t"] + N) * d > 3e11:
        return None
    out = torch.zeros(case["B"], N, case["Hq"], d, device="cuda", dtype=torch.float64)
    parents = s["parent"].tolist()
    for b, (n, m) in enumerate(zip(_lengths(case), _counts(case))):
        off = torch.ones(m, n + m, dtype=torch.bool)
        off[:, :n] = False
        for i, seen in enumerate(_chains(parents[b][:m])):
            off[i, [n + j for j in seen]] = False
        off = off.cuda()
        for h in range(Hkv):
            k, v = s["K"][b, h, :n + m].double(), s["V"][b, h, :n + m].double()
            for g in range(h * G, (h + 1) * G):
                x = s["q"][b, :m, g].double() @ k.T / math.sqrt(d)
                out[b, :m, g] = torch.softmax(x.masked_fill(off, -math.inf), -1) @ v
    return out


def _exact_accept(case, s):
    K, V = s["K"].double(), s["V"].double()
    parents, tokens, choice = s["parent"].tolist(), s["tokens"].tolist(), s["choice"].tolist()
    first = s["first"].tolist()
    for b, (n, m) in enumerate(zip(_lengths(case), _counts(case))):
        cur, want, rows = -1, first[b], []
        for i in range(m):                # a node's children all come behind it
            if parents[b][i] == cur and tokens[b][i] == want:
                cur, want = i, choice[b][i]
                rows.append(n + i)
        if rows:
            K[b, :, n:n + len(rows)] = s["K"][b][:, rows].double()
            V[b, :, n:n + len(rows)] = s["V"][b][:, rows].double()
    return {"K": K, "V": V, "path": None, "accepted": None, "next": None, "lens": None}


def _exact_fork(case, s):
    K, V = s["K"].double(), s["V"].double()
    mass, summ = (s[n].double() if case["extra"] else None for n in ("mass", "summ"))
    lens, lo = _lengths(case), case["first"]
    for b, a in enumerate(_sources(case)):
        n = lens[a] if a >= 0 else 0
        if case["extra"]:
            mass[b, :, n:lens[b]] = 0
            mass[b, :, :n] = s["mass"][a, :, :n].double()
            summ[b, :, lo // SEG:n // SEG] = s["summ"][a, :, lo // SEG:n // SEG].double()
        if n > lo:
            K[b, :, lo:n], V[b, :, lo:n] = s["K"][a, :, lo:n].double(), s["V"][a, :, lo:n].double()
    return {"K": K, "V": V, "mass": mass, "summ": summ, "lens": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"axes": _exact_axes, "tree": _exact_tree, "accept": _exact_accept, "fork": _exact_fork}[case["op"]](case, s)
