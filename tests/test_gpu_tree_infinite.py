"""Infinities and NaN among the drafted rows that a node attends: what the definition
gives in 64 bits, whichever tile, part or wave the row falls to."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
import _cache_ref as R  # noqa: E402
from test_gpu_tree import DT, DTYPES, _above, _cfg, _inputs, _tree  # noqa: E402

import paper_2503_10571_amd as radar  # noqa: E402

pytestmark = pytest.mark.gpu

CASES = [  # Hq, Hkv, d, t, N, lens, spread (0: a chain)
    (4, 4, 64, 0, 5, None, 2),
    (2, 1, 64, 0, 300, None, None),      # all roots: the first wave's tiles hold nothing for most
    (8, 2, 128, 40, 7, None, 3),         # one row tile, a wave for each of its tiles
    (8, 2, 128, 40, 7, None, 0),
    (8, 2, 128, 900, 12, [900, 3], 3),   # 48 query rows, in parts of different lengths
    (8, 2, 64, 2500, 30, None, 0),       # 120, a chain, in parts
    (8, 2, 128, 130, 90, None, 0),       # row tiles, whole
    (8, 2, 128, 130, 90, [130, 0], 6),
    (1, 1, 64, 0, 200, None, 0),
    (32, 8, 128, 8161, 33, None, 6),     # eight waves to a workgroup
    (2, 2, 128, 17000, 3, None, None),   # many parts
    (8, 1, 64, 70, 40, None, None),
]


@DTYPES
@pytest.mark.parametrize("Hq,Hkv,d,t,N,lens,spread", CASES)
def test_attended(Hq, Hkv, d, t, N, lens, spread, dtype):
    B, G = 2, Hq // Hkv
    print(f"[case] infinite Hq{Hq}/{Hkv} d{d} t{t} N{N} {lens} spread{spread} {dtype}", flush=True)
    L = lens or [t] * B
    parents = [_tree(N, b, spread) for b in range(B)]
    P = None if spread == 0 else torch.tensor(parents, dtype=torch.int32, device="cuda")
    q, K, V = _inputs(B, Hq, Hkv, d, t, N, L, [N] * B, dtype, seed=N + t)
    q[..., 3] = q[..., 3].abs() + 0.5
    inf = float("inf")
    one, two, gone = N // 2, N - 1, N // 3
    for b in range(B):
        for j, dims in ((one, {5: inf, 6: -inf, 7: inf, 8: float("nan"), 20: inf}),
                        (two, {7: -inf, 20: inf, 21: -inf}), (gone, {30: inf, 31: float("nan")})):
            for dim, x in dims.items():
                V[b, :, L[b] + j, dim] = x
        K[b, :, L[b] + gone, 3] = -inf   # a logit of -inf: weight 0, and 0 times infinity
        if L[b]:
            V[b, :, L[b] // 2, 9] = inf  # of the sequence itself
    kw = dict(parent=P, lens=None if lens is None else torch.tensor(lens, device="cuda"))
    out = radar.attend_tree(_cfg(B, Hq, Hkv, d, K.shape[2], dtype), q, K, V, t, **kw)
    for b in range(B):
        for i, seen in enumerate(_above(parents[b], N)):
            for h in range(Hkv):
                at = list(range(L[b])) + [L[b] + j for j in seen]
                k, v = K[b, h, at].double(), V[b, h, at].double()
                qq = q[b, i, h * G:(h + 1) * G].double()
                live = [x for x in range(len(at)) if at[x] != L[b] + gone]
                got = out[b, i, h * G:(h + 1) * G].double()
                if not live:             # 0 / 0
                    assert bool(got.isnan().all())
                    continue
                # (logits and weights without the infinite key; its values times 0 then)
                lost = torch.nan_to_num(v[live], 0.0, 0.0, 0.0)
                want, tol, w, _ = R.attend(qq, k[live], lost, DT[dtype], N * G)
                odd = torch.where(v.isfinite(), 0.0, v)
                full = torch.zeros(G, len(at), dtype=torch.float64, device="cuda")
                full[:, live] = w
                assert bool((w > 1e-30).all())
                want = want + (full[:, :, None] * odd[None]).sum(1)
                fine = want.isfinite()
                assert torch.equal(got.isnan(), want.isnan()), (b, i, h)
                assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()]), (b, i, h)
                assert bool(((got - want).abs()[fine] <= tol[fine]).all()), (b, i, h)
