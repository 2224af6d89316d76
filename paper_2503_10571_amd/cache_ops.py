"""The cache operators beside the decode path (include/radar_cache.h): rotary
positions, attention over a shared prefix, attention that accumulates the
rows' weights, eviction by those weights. Like the rest of the binding this
only marshals arguments; the package re-exports every public name.
"""
from __future__ import annotations

import ctypes
import dataclasses
import math

import torch

from . import (RADAR_BF16, RADAR_F32, Config, RadarError, _cache, _check, _Config,
               _need, _query, lib)

_P = ctypes.c_void_p
_DTYPES = {torch.float32: RADAR_F32, torch.bfloat16: RADAR_BF16}
ROPE_MAX_DIM = 256


class _Rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("mscale", ctypes.c_float), ("inv_freq", ctypes.c_void_p)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq", ctypes.c_int64),
                ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


def declare(L) -> None:
    """Argument types of the calls, for the library the package loaded."""
    cfgp, ropep, rowsp = (ctypes.POINTER(x) for x in (_Config, _Rope, _Rows))
    i64, i32, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    L.radar_rotary.argtypes = [ropep, i32, i64, i32, ctypes.c_int, i32, rowsp, rowsp,
                               i32, rowsp, rowsp, i64, _P, i32, _P, i32, _P]
    L.radar_rotary_fill.argtypes = [cfgp, ropep, i64, rowsp, rowsp, rowsp, rowsp, _P, _P,
                                    i64, _P, i64, _P, i32, _P, _P]
    L.radar_attend_prefix.argtypes = [cfgp, _P, _P, _P, i64, i64, _P, _P, i64, _P, _P, _P,
                                      sz, _P]
    L.radar_attend_accumulate.argtypes = [cfgp, _P, _P, _P, _P, i64, _P, _P, _P, sz, _P]
    L.radar_attend_prefix_workspace_bytes.argtypes = [cfgp, i64, i64]
    L.radar_attend_accumulate_workspace_bytes.argtypes = [cfgp, i64]
    L.radar_evict.argtypes = [cfgp, _P, _P, _P, i64, _P, i64, i64, _P, _P, _P, sz, _P]
    L.radar_evict_workspace_bytes.argtypes = [cfgp, i64, i64, i64]
    for fn in ("radar_attend_prefix_workspace_bytes",
               "radar_attend_accumulate_workspace_bytes", "radar_evict_workspace_bytes"):
        getattr(L, fn).restype = sz
    for fn in ("radar_rotary", "radar_rotary_fill", "radar_attend_prefix",
               "radar_attend_accumulate", "radar_evict"):
        getattr(L, fn).restype = ctypes.c_int


def _ptr(x):
    return None if x is None else x.data_ptr()


def _one_device(x, *others):
    """Every device tensor of a call lies on x's GPU."""
    d = x.get_device()
    for o in others:
        if o is not None and o.get_device() not in (d, -1):
            raise ValueError(f"tensors on different devices: {x.device} and {o.device}")


def _call(fn, x, *args):
    """lib().fn(*args, stream) with x's device current (a stream takes launches
    from its own device only). Device and stream are asked for as torch's own
    generated code asks: the stream's handle alone, 2 us less than an object."""
    f = getattr(lib(), fn)
    i = x.get_device()
    if i == torch._C._cuda_getDevice():
        st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    if st != 0:
        _check(fn, st)


# ---- rotary positions --------------------------------------------------------
@dataclasses.dataclass(frozen=True, eq=False)
class Rope:
    """Rotary positions of a head: inv_freq, a device float64 tensor
    [rot_dim / 2] of angles per position (see rope_frequencies); interleaved:
    pairs (2 i, 2 i + 1) instead of (i, i + rot_dim / 2); mscale: a factor on
    the rotated dims."""
    inv_freq: torch.Tensor
    interleaved: bool = False
    mscale: float = 1.0

    def __post_init__(self):
        _need(self.inv_freq, torch.float64, "inv_freq")
        object.__setattr__(self, "_c", _Rope(2 * self.inv_freq.numel(),
                                             1 if self.interleaved else 0, self.mscale,
                                             self.inv_freq.data_ptr()))

    # (the same frequencies are the same tensor: two of equal values have no truth value)
    def _key(self):
        return id(self.inv_freq), self.interleaved, self.mscale

    def __eq__(self, other):
        return self._key() == other._key() if isinstance(other, Rope) else NotImplemented

    def __hash__(self):
        return hash(self._key())

    def __reduce__(self):                          # the pointer is not copied
        return Rope, (self.inv_freq, self.interleaved, self.mscale)

    @property
    def rot_dim(self) -> int:
        return 2 * self.inv_freq.numel()


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none",
                     factor: float = 1.0, trained_len: int = 0, alpha: float = 1.0,
                     beta: float = 32.0):
    """(inv_freq, mscale) of rot_dim rotated dims: inv_freq a float64 CPU tensor
    f_i = base^(-2 i / rot_dim), and, for contexts longer than the trained one
    by `factor`,
      "linear"  f_i / factor (positions interpolated);
      "ntk"     the base times factor^(rot_dim / (rot_dim - 2)), which leaves
                the fastest pair as it is and slows the slowest by `factor`;
      "yarn"    by parts: pairs that turn more than beta times over trained_len
                positions stay, those that turn less than alpha times are
                interpolated, linear in between; mscale = 0.1 ln(factor) + 1.
    mscale is 1 otherwise."""
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError(f"rot_dim must be even and positive, got {rot_dim}")
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor must be positive")
    if scaling == "ntk":
        if rot_dim < 4:
            raise ValueError("ntk scaling needs two pairs")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    f = torch.pow(torch.tensor(float(base), dtype=torch.float64), -2.0 * i / rot_dim)
    if scaling in ("none", "ntk"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "yarn":
        raise ValueError(f"scaling {scaling!r}: none, linear, ntk or yarn")
    if trained_len < 1 or not beta > alpha:
        raise ValueError("yarn needs trained_len >= 1 and beta > alpha")
    turns = f * (trained_len / (2 * math.pi))
    keep = ((turns - alpha) / (beta - alpha)).clamp(0.0, 1.0)
    return keep * f + (1 - keep) * f / factor, 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0


def _rows(x, name, dtype):
    """(struct, B, T, heads, d) of x, [B][T][heads][d] or [B][heads][d] (one
    token): a dense last axis, the address and the other strides on 16 bytes."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) == 4:
        B, T, H, d = shape
        sb, st, sh, sd = stride
    elif len(shape) == 3:
        (B, H, d), (sb, sh, sd), T, st = shape, stride, 1, 0
    else:
        raise ValueError(f"{name} must be [B][T][heads][d] or [B][heads][d]")
    # (the stride of an axis of one element is not used and may be anything)
    if B <= 1:
        sb = 0
    if T <= 1:
        st = 0
    if H <= 1:
        sh = 0
    ptr, per = x.data_ptr(), 16 // x.element_size()
    if sd != 1 and d > 1 or ptr & 15 or sb % per or st % per or sh % per:
        raise ValueError(f"{name} needs a dense last axis and other strides and an address "
                         "that are multiples of 16 bytes")
    return _Rows(ptr, sb, st, sh), B, T, H, d


def _out_rows(x, out, name, lens):
    """(out, struct) for the input x: the given tensor, or a new dense one (zeros
    where lengths leave tokens unwritten)."""
    if out is None:
        new = torch.empty_like if lens is None else torch.zeros_like
        out = new(x, memory_format=torch.contiguous_format)
        H, d = x.shape[-2:]
        if d * out.element_size() % 16 == 0:
            T = x.shape[1] if x.dim() == 4 else 1
            return out, _Rows(out.data_ptr(), T * H * d, H * d, d)
    else:
        if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device:
            raise ValueError(f"{name} must have the input's shape, type and device")
        if any(s == 0 and n > 1 for s, n in zip(out.stride(), out.shape)):
            raise ValueError(f"{name} has elements that share a place")
        if out.data_ptr() == x.data_ptr() and out.stride() != x.stride():
            raise ValueError(f"{name} starts at its input with other strides")
    return out, _rows(out, name, x.dtype)[0]


def _positions(pos, B, T, name="pos"):
    """(first position, device tensor or None, one per token) of an int, an
    int64 [B] (first tokens) or an int64 [B][T] (each token)."""
    if isinstance(pos, int):
        return pos, None, 0
    _need(pos, torch.int64, name)
    if pos.dim() == 1 and pos.numel() == B:
        return 0, pos, 0
    if tuple(pos.shape) == (B, T):
        return 0, pos, 1
    raise ValueError(f"{name} must be an int, int64 [B] or int64 [B][T]")


def _lens_of(lens, B):
    if lens is not None:
        _need(lens, torch.int64, "lens", B)
    return lens


def _float_type(x, name):
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, got {x.dtype}")


def _records(rope, x, y=None):
    """Whether autograd records a call on x (and y)."""
    if not torch.is_grad_enabled():
        return False
    if rope.inv_freq.requires_grad:
        raise RuntimeError("inv_freq has no gradient here: detach it")
    return x.requires_grad or y is not None and y.requires_grad


def _no_gradient(fn, *xs):
    """For the calls that autograd does not know: refuses operands whose gradient
    would be lost without a word."""
    if torch.is_grad_enabled():
        for x in xs:
            if x is not None and x.requires_grad:
                raise RuntimeError(f"{fn} has no gradient: call it under torch.no_grad(), or "
                                   "detach its operands")


class _Rotate(torch.autograd.Function):
    """rotary (one operand) and rotary_qk (two) for autograd: the gradient is the
    inverse rotation of the outputs' gradients."""

    @staticmethod
    def forward(ctx, rope, pos, inverse, lens, *xs):
        ctx.set_materialize_grads(False)
        ctx.rope, ctx.pos, ctx.inverse = rope, pos, inverse
        # (saved so that a change in place before the backward pass is found)
        ctx.save_for_backward(rope.inv_freq, lens, None if isinstance(pos, int) else pos)
        if len(xs) == 1:
            return rotary(rope, *xs, pos, inverse=inverse, lens=lens)
        return rotary_qk(rope, *xs, pos, inverse=inverse, lens=lens)

    @staticmethod
    def backward(ctx, *grads):
        _, lens, pos = ctx.saved_tensors
        kw = dict(pos=ctx.pos if pos is None else pos, inverse=not ctx.inverse, lens=lens)
        want = [g if need else None for g, need in zip(grads, ctx.needs_input_grad[4:])]
        # gradients of any layout; the kernel takes dense rows on 16 bytes
        want = [g if g is None else g.contiguous() for g in want]
        want = [g.clone() if g is not None and g.data_ptr() & 15 else g for g in want]
        if len(want) == 2 and want[0] is not None and want[1] is not None:
            got = rotary_qk(ctx.rope, *want, **kw)
        else:
            got = [g if g is None else rotary(ctx.rope, g, **kw) for g in want]
        return (None, None, None, None, *got)


def rotary(rope: Rope, x, pos, out=None, inverse: bool = False, lens=None):
    """radar_rotary of one tensor x, [B][T][heads][d] or [B][heads][d] (one
    token), strided as it comes out of a projection. pos: the position of the
    first token (an int, or an int64 [B]) or of every token (int64 [B][T]).
    out may be x. inverse: the gradient of the rotation. lens (int64 [B]): only
    tokens t < lens[b] are touched (the others are 0 in a new out). Autograd
    differentiates it in x, where out is not given. Returns out."""
    _float_type(x, "x")
    if _records(rope, x):
        if out is not None:
            raise RuntimeError("rotary takes no out where a gradient is recorded")
        return _Rotate.apply(rope, pos, inverse, lens, x)
    rx, B, T, H, d = _rows(x, "x", x.dtype)
    out, ro = _out_rows(x, out, "out", lens)
    p0, p, each = _positions(pos, B, T)
    lens = _lens_of(lens, B)
    _one_device(x, p, lens, rope.inv_freq)
    if x.numel():
        by = ctypes.byref
        _call("radar_rotary", x, by(rope._c), B, T, d, _DTYPES[x.dtype], H, by(rx), by(ro),
              0, None, None, p0, _ptr(p), each, _ptr(lens), 1 if inverse else 0)
    return out


def rotary_qk(rope: Rope, q, k, pos, q_out=None, k_out=None, inverse: bool = False,
              lens=None):
    """rotary() of q and k in one launch; either may have no heads. Returns
    (q_out, k_out)."""
    _float_type(q, "q")
    if _records(rope, q, k):
        if q_out is not None or k_out is not None:
            raise RuntimeError("rotary_qk takes no q_out and k_out where a gradient is recorded")
        return _Rotate.apply(rope, pos, inverse, lens, q, k)
    rq, B, T, Hq, d = _rows(q, "q", q.dtype)
    rk, Bk, Tk, Hk, dk = _rows(k, "k", q.dtype)
    if (Bk, Tk, dk) != (B, T, d):
        raise ValueError("q and k must agree in batch, tokens and head_dim")
    q_out, qo = _out_rows(q, q_out, "q_out", lens)
    k_out, ko = _out_rows(k, k_out, "k_out", lens)
    p0, p, each = _positions(pos, B, T)
    lens = _lens_of(lens, B)
    _one_device(q, k, p, lens, rope.inv_freq)
    if B * T * d and (Hq or Hk):
        by = ctypes.byref
        first, second = (Hq, by(rq), by(qo)), (Hk, by(rk), by(ko))
        if not Hq:                             # k is the only operand
            first, second = second, first
        if not second[0]:
            second = (0, None, None)
        _call("radar_rotary", q, by(rope._c), B, T, d, _DTYPES[q.dtype], *first, *second,
              p0, _ptr(p), each, _ptr(lens), 1 if inverse else 0)
    return q_out, k_out


def rotary_fill(cfg: Config, rope: Rope, K, V, k, v, row, pos=None, q=None, q_out=None,
                lens=None):
    """radar_rotary_fill: the chunk k, v [B][T][Hkv][d] (or [B][Hkv][d], one
    token) into rows row + t of K and V, k rotated; with q, its rotation too,
    in the same launch. row: an int, or an int64 [B] (rows outside the capacity
    are skipped); pos: as for rotary(), the row itself if None. lens: as for
    rotary(). No gradient goes through the cache: operands that want one are
    refused. Returns q_out (None without q)."""
    _no_gradient("rotary_fill", k, v, q, rope.inv_freq)
    _cache(cfg, K, V)
    rk, B, T, Hk, d = _rows(k, "k", cfg.dtype)
    rv, *shape_v = _rows(v, "v", cfg.dtype)
    if [B, T, Hk, d] != shape_v or (B, Hk, d) != (cfg.batch, cfg.n_kv_heads, cfg.head_dim):
        raise ValueError("k and v must be [batch][T][n_kv_heads][head_dim], the config's "
                         f"{cfg.batch}, {cfg.n_kv_heads} heads of {cfg.head_dim}")
    rq = qo = None
    by = ctypes.byref
    if q is not None:
        rq, *shape_q = _rows(q, "q", cfg.dtype)
        if shape_q != [B, T, cfg.n_q_heads, d]:
            raise ValueError("q must be [batch][T][n_q_heads][head_dim] with k's tokens")
        q_out, qo = _out_rows(q, q_out, "q_out", lens)
        rq, qo = by(rq), by(qo)
    elif q_out is not None:
        raise ValueError("q_out without q")
    r0, rows, each = _positions(row, B, T, "row")
    if each:
        raise ValueError("row must be an int or int64 [B]")
    p0, p, each = (r0, rows, 0) if pos is None else _positions(pos, B, T)
    lens = _lens_of(lens, B)
    _one_device(k, v, q, rows, p, lens, rope.inv_freq, K, V)
    if T:
        _call("radar_rotary_fill", k, by(cfg.c_struct()), by(rope._c), T, rq, qo, by(rk), by(rv),
              _ptr(K), _ptr(V), r0, _ptr(rows), p0, _ptr(p), each, _ptr(lens))
    return q_out


# ---- attention over a shared prefix, and with accumulated weights --------------
def attend_prefix_workspace_bytes(cfg: Config, prefix_len: int, t: int) -> int:
    """Scratch for every call with this config, at most this prefix_len and t."""
    return int(lib().radar_attend_prefix_workspace_bytes(ctypes.byref(cfg.c_struct()),
                                                         prefix_len, t))


def attend_accumulate_workspace_bytes(cfg: Config, t: int) -> int:
    """Scratch for every call with this config and at most this t."""
    return int(lib().radar_attend_accumulate_workspace_bytes(ctypes.byref(cfg.c_struct()), t))


def _workspace(given, nbytes, device):
    """The given workspace, or a new one (none where the size is 0: the call
    refuses its arguments)."""
    if given is not None:
        _need(given, torch.uint8, "workspace")
        return given, given.numel()
    if nbytes == 0:
        return None, 0
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def _attended(cfg, q, out, lens):
    _query(cfg, q)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, cfg.dtype, "out", cfg.batch * cfg.n_q_heads * cfg.head_dim)
    return out, _lens_of(lens, cfg.batch)


def attend_prefix(cfg: Config, q, Kp, Vp, prefix_len: int, K=None, V=None, t: int = 0,
                  out=None, lens=None, workspace=None):
    """radar_attend_prefix: exact attention of every sequence's query (q
    [B][Hq][d]) over rows [0, prefix_len) of Kp, Vp [Hkv][rows][d], which the
    batch shares, and rows [0, t) (or [0, lens[b])) of its own K, V (None with
    t = 0). Has no gradient: operands that want one are refused. Returns out."""
    _no_gradient("attend_prefix", q, Kp, Vp, K, V)
    out, lens = _attended(cfg, q, out, lens)
    prefix_cap = 0
    if prefix_len > 0:
        for x, name in ((Kp, "Kp"), (Vp, "Vp")):
            if x is None or x.dim() != 3 or x.shape[0] != cfg.n_kv_heads or x.shape[2] != cfg.head_dim:
                raise ValueError(f"{name} must be [n_kv_heads][rows][head_dim]")
            _need(x, cfg.dtype, name, host_ok=True)
        prefix_cap = Kp.shape[1]
        if Vp.shape[1] != prefix_cap:
            raise ValueError("Kp and Vp must hold the same number of rows")
    if t > 0 or K is not None:
        if K is None or V is None:
            raise ValueError("K and V are needed with t > 0")
        _cache(cfg, K, V)
    _one_device(q, Kp, Vp, K, V, out, lens, workspace)
    c = ctypes.byref(cfg.c_struct())
    need = lib().radar_attend_prefix_workspace_bytes(c, prefix_len, t) if workspace is None else 0
    workspace, n = _workspace(workspace, need, q.device)
    _call("radar_attend_prefix", q, c, _ptr(q), _ptr(Kp), _ptr(Vp), prefix_len, prefix_cap,
          _ptr(K), _ptr(V), t, _ptr(lens), _ptr(out), _ptr(workspace), n)
    return out


def _mass(cfg, mass):
    _need(mass, torch.float32, "mass", cfg.batch * cfg.n_kv_heads * cfg.capacity)


def new_mass(cfg: Config, device) -> torch.Tensor:
    """The weights of the rows of an empty cache, [B][Hkv][capacity] fp32."""
    return torch.zeros(cfg.batch, cfg.n_kv_heads, cfg.capacity, dtype=torch.float32,
                       device=device)


def attend_accumulate(cfg: Config, q, K, V, mass, t: int, out=None, lens=None,
                      workspace=None):
    """radar_attend_accumulate: exact attention over rows [0, t) (or
    [0, lens[b])) of K and V; the softmax weight of every row, summed over the
    query heads of its kv head, is added to mass [B][Hkv][capacity] (fp32).
    Has no gradient: operands that want one are refused. Returns out."""
    _no_gradient("attend_accumulate", q, K, V)
    out, lens = _attended(cfg, q, out, lens)
    _cache(cfg, K, V)
    _mass(cfg, mass)
    _one_device(q, K, V, mass, out, lens, workspace)
    c = ctypes.byref(cfg.c_struct())
    need = lib().radar_attend_accumulate_workspace_bytes(c, t) if workspace is None else 0
    workspace, n = _workspace(workspace, need, q.device)
    _call("radar_attend_accumulate", q, c, _ptr(q), _ptr(K), _ptr(V), _ptr(mass), t,
          _ptr(lens), _ptr(out), _ptr(workspace), n)
    return out


# ---- eviction ---------------------------------------------------------------------
def evict_workspace_bytes(cfg: Config, t: int, heavy: int, recent: int) -> int:
    """Scratch for every call with this config, at most this t and at most as
    many kept rows."""
    return int(lib().radar_evict_workspace_bytes(ctypes.byref(cfg.c_struct()), t, heavy,
                                                 recent))


def evict(cfg: Config, K, V, mass, t: int, heavy: int, recent: int, lens=None,
          new_lens=None, kept=None, workspace=None) -> int:
    """radar_evict: cut the cache of t rows (or lens[b]) to n = cfg.n_sink +
    heavy + recent: the sinks, the last `recent` rows, and the `heavy` rows of
    the others with the largest mass move to the front of K, V and mass, in
    their order; the masses behind them become 0. new_lens (int64 [B], may be
    lens) receives the new lengths, kept (int32 [B][Hkv][min(n, t)]) the rows
    kept. The summaries hold for the old rows: build_index() follows. Returns
    the bound of the new lengths, min(t, n)."""
    _cache(cfg, K, V)
    _mass(cfg, mass)
    n = min(cfg.n_sink + heavy + recent, t)
    lens = _lens_of(lens, cfg.batch)
    if new_lens is not None:
        _need(new_lens, torch.int64, "new_lens", cfg.batch)
    if kept is not None:
        _need(kept, torch.int32, "kept", cfg.batch * cfg.n_kv_heads * n)
    _one_device(mass, K, V, lens, new_lens, kept, workspace)
    c = ctypes.byref(cfg.c_struct())
    need = (lib().radar_evict_workspace_bytes(c, t, heavy, recent)
            if workspace is None else 0)
    workspace, size = _workspace(workspace, need, mass.device)
    _call("radar_evict", mass, c, _ptr(K), _ptr(V), _ptr(mass), t, _ptr(lens), heavy, recent,
          _ptr(new_lens), _ptr(kept), _ptr(workspace), size)
    return n
