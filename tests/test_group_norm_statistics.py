"""Statistics of rf_group_norm far from zero, and the 64-bit statement of the norm against torch's own operator."""
import pytest
import torch

from ops_check import DEV, check, lists, row_mask, SENTINEL
from oracle import ops_oracle
from test_group_norm import ACTS, SHAPES, _forward, _inputs, _workspace


@pytest.mark.gpu
@pytest.mark.parametrize("in8", [False, True])
@pytest.mark.parametrize("shape", [2, 4, 5, 8, 10, 12, 17, 20, 23])
def test_statistics_far_from_zero(cuda_lib, shape, in8):
    """Mean and 1/deviation, which the gradients take, where channels lie a thousand deviations from zero and one row
    far from all others: within the bounds that test_group_norm.py derives."""
    F, N, frames, C, G = SHAPES[shape]
    X, w, b = _inputs(F, N, C, torch.float32, torch.float32, shape, far=0.1)
    X = X + 1000.0
    X[0] += 300.0
    st = torch.full((F, G, 2), SENTINEL, device=DEV)
    Y = torch.zeros(F * N, C, dtype=torch.int8 if in8 else torch.float32, device=DEV)
    scale = torch.zeros(F * N, device=DEV) if in8 else None
    a, cnt = lists(frames, F, N)
    cuda_lib.rf_group_norm(Y, X, F, N, G, weight=w, bias=b, stats=st, scale=scale, active=a, counts=cnt,
                           workspace=_workspace(cuda_lib, F, N, C, G, torch.float32))
    torch.cuda.synchronize()
    _, _, stats, dm, dr = _forward(X, w, b, frames, N, G, 1e-5, None)
    on = torch.zeros(F, dtype=torch.bool)
    on[list(frames)] = True
    check(st[:, :, 0], stats[:, :, 0], dm, on, "mean")
    check(st[:, :, 1], stats[:, :, 1], dr, on, "1/deviation")


@pytest.mark.parametrize("act", ACTS)
def test_oracle_agrees_with_torch(act):
    """The oracle's norm and gradients against torch's group_norm and autograd, both in 64 bits."""
    F, N, C, G, frames = 3, 11, 24, 4, (0, 2)
    g = torch.Generator().manual_seed(4)
    X, dY = (torch.randn(F * N, C, generator=g, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(C, generator=g, dtype=torch.float64) for _ in range(2))
    fn = {None: lambda t: t, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
          "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[act]
    leaves = [t.clone().requires_grad_() for t in (X, w, b)]
    x = leaves[0].view(F, N, C).transpose(1, 2)  # channels second
    y = fn(torch.nn.functional.group_norm(x, G, leaves[1], leaves[2], 1e-5)).transpose(1, 2).reshape(F * N, C)
    rows = row_mask(frames, F, N)
    gx, gw, gb = torch.autograd.grad((y * dY)[rows].sum(), leaves)
    Y, _, stats = ops_oracle.group_norm(X, frames, N, G, w, b, 1e-5, act)
    dX, dW, db, _ = ops_oracle.group_norm_bwd(dY, X, stats, frames, N, G, w, b, act)
    # (64 bits on both sides: some hundred roundings of 2^-53, on values of a few units)
    for got, want in ((Y[rows], y[rows]), (dX[rows], gx[rows]), (dW, gw), (db, gb)):
        assert (got - want).abs().max() <= 1e-12
