"""rf_quantize_rows where quotients land on halves, exactly or nearly, in every vector of a row, for largest values from
the smallest to the largest floats: the nearest whole number, ties to even, without exception."""
import math

import pytest
import torch

from ops_check import DEV, DTYPES, ROUND, TINY
from oracle import ops_oracle

MOST = [2.0 ** -120, 1e-30, 2.0 ** -100, 1.0, 127.0, 1e30, 2.0 ** 100, 127 * 2.0 ** 100, 2.6e36, 1e37, 127 * 2.0 ** 117,
        1e38, 2.0 ** 127, 3e38, 127 * 2.0 ** 121, torch.finfo(torch.float32).max]


def _halves(most, rows, d, dt):
    """Numbers at a half of the row's steps, next to one, or anywhere; the first is the largest value.  (In a type
    with few bits not every one is next to a half; all are of the type.)"""
    g = torch.Generator().manual_seed(int(math.frexp(most)[1]) + 2000)
    h = torch.randint(-127, 127, (rows, d), generator=g).double() + 0.5
    top = torch.tensor(most, dtype=torch.float64).to(dt)
    x = (h * top.double() / 127).to(dt)
    pick = torch.rand(rows, d, generator=g)
    x = torch.where(pick < 0.2, torch.nextafter(x, torch.full_like(x, 0.0)), x)
    x = torch.where(pick > 0.8, torch.nextafter(x, torch.full_like(x, math.inf).copysign(x)), x)
    away = ((torch.rand(rows, d, generator=g, dtype=torch.float64) * 2 - 1) * top.double()).to(dt)
    x = torch.where((pick > 0.4) & (pick < 0.5), away, x)
    x[:, 0] = top * (1 - 2 * (torch.arange(rows) % 2))
    x[0, 1] = top / 2  # 63.5 beside 127
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 1000, 77])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("most", MOST)
def test_halves_of_any_size(cuda_lib, most, dtype, d):
    if dtype == "bf16" and most > 3.38e38:
        pytest.skip("rounds to infinity")
    X = _halves(most, 24, d, DTYPES[dtype])
    assert torch.isfinite(X).all() and (X.abs() <= X[:, :1].abs()).all()
    Y, s = torch.full(X.shape, 77, dtype=torch.int8, device=DEV), torch.zeros(24, device=DEV)
    cuda_lib.rf_quantize_rows(Y, s, X.to(DEV), 1, 24)
    torch.cuda.synchronize()
    q, want = ops_oracle.quantize_rows(X, (0,), 24)
    assert torch.equal(Y.cpu().double(), q)
    assert ((s.cpu().double() - want).abs() <= ROUND[torch.float32] * want + TINY[torch.float32]).all()
