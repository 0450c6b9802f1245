"""rf_cross_attn: active rows keep their bits whatever stands beside them.

A tile of 128 rows can hold tokens of skipped frames, the padding of short frames, or what an earlier tile or
kernel left in shared memory.  None of that may reach a result, by not a bit.
"""
import math

import pytest
import torch

from ops_check import DEV, SENTINEL, lists, row_mask

H16 = torch.bfloat16
SHAPES = [  # F, N, frames, H, Hkv, d, L
    (6, 100, (0, 2, 5), 4, 4, 128, 700),
    (4, 200, (1,), 4, 2, 64, 900),
    (40, 1, (3, 7, 20, 39), 8, 8, 128, 3000),   # single tokens
    (9, 6, (0, 4, 8), 6, 2, 64, 1300),          # packed: tokens and query heads
    (5, 1003, (0, 3), 2, 2, 64, 1500),
    (3, 1560, (1, 2), 12, 12, 128, 512),
]


def _case(shape, keys):
    F, N, frames, H, Hkv, d, L = shape
    g = torch.Generator().manual_seed(N)
    Q = torch.randn(F * N, H, d, generator=g)
    K, V = (torch.randn(L, Hkv, d, generator=g) for _ in range(2))
    K = K * torch.linspace(0.05, 3.0, L)[:, None, None]  # a row's maximum grows from tile to tile
    kw = {}
    if keys == "ranges":
        kw["kv_range"] = torch.tensor([[f % 3, L - f] for f in range(F)], dtype=torch.int32, device=DEV)
    elif keys == "mask":
        kw["key_mask"] = (torch.rand(L, generator=g) < 0.7).to(torch.uint8).to(DEV)
    elif keys == "few":  # gathered
        kw["key_mask"] = (torch.rand(L, generator=g) < 0.3).to(torch.uint8).to(DEV)
    return Q, K.to(H16).to(DEV), V.to(H16).to(DEV), kw


@pytest.mark.gpu
@pytest.mark.parametrize("keys", ["all", "ranges", "mask", "few"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rows_beside(cuda_lib, shape, keys):
    F, N, frames, H, Hkv, d, L = SHAPES[shape]
    Q, K, V, kw = _case(SHAPES[shape], keys)
    act, cnt = lists(frames, F, N)
    rows = row_mask(frames, F, N)
    loud = (torch.randn(2048, 8, 128, generator=torch.Generator().manual_seed(1)) * 40).to(H16).to(DEV)
    first = None
    for fill in (0.0, 1.0, 40.0, -40.0, math.nan, math.inf):
        q = Q.clone()
        q[~rows] = q[~rows] * fill
        O = torch.full((F * N, H, d), SENTINEL, dtype=H16, device=DEV)
        lse = torch.full((H, F * N), SENTINEL, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        q = q.to(H16).to(DEV)
        if fill != 1.0:  # (once without) leaves every SM's shared memory full of large queries
            cuda_lib.rf_cross_attn(torch.empty_like(loud), None, loud, loud[:700], loud[:700], 1, 2048, 1.0)
        cuda_lib.rf_cross_attn(O, lse, q, K, V, F, N, d ** -0.5, active=act, counts=cnt, status=st, **kw)
        torch.cuda.synchronize()
        assert st.item() == 0
        got = (O.cpu()[rows], lse.cpu()[:, rows])
        assert (O.cpu()[~rows] == SENTINEL).all()
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first)), fill
