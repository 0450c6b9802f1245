"""rf_linear_i8 over many digits: sums below 2^24 come back bit for bit from every kernel, so a digit that is lost, taken
twice or from another row shows, whatever its weight in the sum."""
import math

import pytest
import torch

from ops_check import DEV
from oracle import ops_oracle

# rows, K, O: rows behind which pairs of CTAs, splits and dot products stand
SHAPES = [(1100, 5120, 1536), (700, 8192, 1920), (512, 13824, 5120), (513, 13823, 5117), (300, 8191, 1700),
          (16, 5120, 13824), (40, 5120, 1000), (200, 13824, 640), (4, 13824, 5120), (7, 13824, 200)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,K,O", SHAPES)
def test_long_sums_are_exact(cuda_lib, rows, K, O):
    g = torch.Generator().manual_seed(K + rows)
    most = min(127, math.isqrt((2 ** 24 - 1) // K))  # K most^2 < 2^24: no sum of some of the products is larger
    pad = (K + 15) // 16 * 16

    def digits(n):
        t = torch.full((n, pad), -77, dtype=torch.int8)
        t[:, :K] = torch.randint(-most, most + 1, (n, K), generator=g)
        return t

    X, W = digits(rows), digits(O)
    X[-1, :K], W[-1, :K] = most, most  # the largest sum there is
    one = torch.ones(max(rows, O), device=DEV)
    Y = torch.full((rows, O), math.nan, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    cuda_lib.rf_linear_i8(Y, X.to(DEV)[:, :K], one[:rows], W.to(DEV)[:, :K], one[:O], 1, rows, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    want, _, S = ops_oracle.linear_i8(X[:, :K], torch.ones(rows), W[:, :K], torch.ones(O), (0,), rows)
    assert S.max() < 2 ** 24 and torch.equal(Y.cpu().double(), want)
