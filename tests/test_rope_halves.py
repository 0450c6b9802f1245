"""rf_rope in halves where R/2 is not a multiple of four, element by element: against the 64-bit statement,
in every type, forward and back.  The bound is test_rope.py's."""
import numpy as np
import pytest
import torch

from ops_check import DEV, DTYPES, SENTINEL, check, lists, row_mask
from oracle import ops_oracle
from test_rope import _bound, _tables

# F, gh, gw, frames, Hq, Hk, d, dims; R/2: 7, 45, 5, 1, 127, 46, 38
SHAPES = [
    (3, 2, 5, (0, 2), 2, 1, 16, (4, 6, 4)),
    (4, 7, 9, (1, 3), 5, 2, 128, (30, 30, 30)),
    (2, 1, 33, (0, 1), 9, 0, 8, (0, 0, 0)),      # (nothing rotates)
    (5, 3, 4, (0, 4), 1, 6, 40, (2, 4, 4)),
    (2, 1, 1, (1,), 1, 1, 256, (0, 2, 0)),
    (3, 5, 3, (0, 1, 2), 3, 3, 256, (86, 84, 84)),
    (2, 30, 52, (0, 1), 12, 12, 128, (32, 30, 30)),
    (3, 4, 4, (2,), 4, 4, 80, (0, 36, 40)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_halves_off_the_vectors(cuda_lib, shape, dtype):
    rf = cuda_lib
    F, gh, gw, frames, Hq, Hk, d, dims = SHAPES[shape]
    dt, N, R = DTYPES[dtype], gh * gw, sum(dims)
    g = torch.Generator().manual_seed(300 + shape)
    pos = [np.arange(F) * 0.75 - 1.0, np.arange(gh) + 3.0, np.arange(gw) * 2.0]
    fused = torch.randn(F * N, Hq + Hk + 1, d, generator=g).to(dt).to(DEV)
    Xq, Xk = fused[:, :Hq], fused[:, Hq:Hq + Hk] if Hk else None
    act, cnt = lists(frames, F, N)
    tables, rows = _tables(rf, pos, dims), row_mask(frames, F, N)
    for inverse in (False, True):
        Yq = torch.full((F * N, Hq, d), SENTINEL, dtype=dt, device=DEV)
        Yk = torch.full((F * N, Hk, d), SENTINEL, dtype=dt, device=DEV) if Hk else None
        rf.rf_rope(Yq, Xq, Yk, Xk, F, gh, gw, dims, tables, pairing="half", inverse=inverse, active=act,
                   counts=cnt)
        # the same in place
        both = fused.clone()
        rf.rf_rope(both[:, :Hq], both[:, :Hq], both[:, Hq:Hq + Hk] if Hk else None,
                   both[:, Hq:Hq + Hk] if Hk else None, F, gh, gw, dims, tables, pairing="half",
                   inverse=inverse, active=act, counts=cnt)
        torch.cuda.synchronize()
        on = rows.to(DEV)
        for X, Y, at in ((Xq, Yq, slice(0, Hq)), (Xk, Yk, slice(Hq, Hq + Hk))):
            if X is None:
                continue
            want = ops_oracle.rope(X, frames, pos, dims, pairing="half", inverse=inverse)
            check(Y, want, _bound(X, want, dims, "half", dt), rows, f"halves {shape} {dtype} {inverse}")
            assert torch.equal(Y[on][..., R:], X[on][..., R:])
            assert torch.equal(both[:, at][on], Y[on]) and torch.equal(both[:, at][~on], X[~on])
        assert torch.equal(both[:, Hq + Hk:], fused[:, Hq + Hk:])
