"""What the cache attention operators compute, in 64 bits, and how far 32-bit
arithmetic may be from it (shared by their tests).

With s = q.k / sqrt(d) off by at most ds, a weight is off by a factor of
1 +- 2 ds; the sums over n rows add at most n 2^-24 of their terms' size each.
ds: a sum of d products, each rounded and added, (d + 2) 2^-24 of |q| |k| /
sqrt(d), and the exponent's own rounding, 2^-23 of |s| and 2^-23. bf16: the
weights enter the product with V rounded to half a step (2^-8), or to 16 bits
(cut, 2^-15) where at most 16 query rows share a kv head's rows; the output is
rounded by half a step of its value."""
import math

import torch

U = 2.0 ** -24


def logit_error(q, k):
    """q [G][d], k [n][d] in 64 bits -> (s [G][n], ds [G][n])."""
    d = q.shape[-1]
    s = q @ k.T / math.sqrt(d)
    size = q.norm(dim=-1)[:, None] * k.norm(dim=-1)[None] / math.sqrt(d)
    return s, (d + 2) * U * size + 2 * U * (s.abs() + 1)


def attend(q, k, v, dtype, rows=1 << 30):
    """(out, tolerance, weights, their tolerance) of q [G][d] over n rows."""
    q, k, v = q.double(), k.double(), v.double()
    n = k.shape[0]
    s, ds = logit_error(q, k)
    w = torch.softmax(s, -1)
    ds = ds.max(-1, keepdim=True)[0]
    rel = 2 * ds + (n + 8) * U
    out = w @ v
    size = w @ v.abs()
    p = 0.0 if dtype == torch.float32 else (2.0 ** -15 if rows <= 16 else 2.0 ** -8)
    half = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2
    tol = (rel * 1.01 + p) * size
    return out, tol + half * (out.abs() + tol), w, w * rel * 1.01 + 1e-37
