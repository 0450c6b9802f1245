"""rf_linear_i8 where a token's scale is large and the columns' small, or the other way round: nothing overflows or is
lost that the three factors' product does not."""
import math

import pytest
import torch

from ops_check import DEV
from oracle import ops_oracle

# Of tokens and of columns (powers of two: products are exact).
SCALES = [(2.0 ** 116, 2.0 ** -100), (2.0 ** -100, 2.0 ** 116), (2.0 ** 64, 2.0 ** -120), (2.0 ** 65, 2.0 ** -120),
          (-2.0 ** 119, 2.0 ** -125), (2.0 ** -125, -2.0 ** 119), (2.0 ** 127, 2.0 ** -126), (2.0 ** -126, 2.0 ** 127),
          (2.0 ** -60, 2.0 ** -60), (2.0 ** 50, 2.0 ** 50)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 3, 6, 40, 600])
@pytest.mark.parametrize("scales", range(len(SCALES)))
def test_scales_far_apart(cuda_lib, rows, scales):
    """Sums below 2^24 times powers of two: exact, in rows of ordinary scales beside them too."""
    K, O = 80, 1600
    xs, ws = SCALES[scales]
    g = torch.Generator().manual_seed(rows)
    X, W = (torch.randint(-127, 128, (n, K), generator=g).to(torch.int8) for n in (rows, O))
    s = torch.full((rows,), xs)
    s[1::2] = 2.0 ** -max(-120, min(120, round(math.log2(abs(ws)))))
    if rows > 2:
        s[2] = math.nan
    u = torch.full((O,), ws)
    Y = torch.zeros(rows, O, device=DEV)
    cuda_lib.rf_linear_i8(Y, X.to(DEV), s.to(DEV), W.to(DEV), u.to(DEV), 1, rows)
    want, _, _ = ops_oracle.linear_i8(X, s, W, u, (0,), rows)
    got = Y.cpu().double()
    if rows > 2:
        assert torch.isnan(got[2]).all()
        got[2] = want[2] = 0.0
    # (the inputs are such that every product is a normal float)
    assert ((want == 0) | ((want.abs() >= 2.0 ** -126) & (want.abs() < 2.0 ** 128))).all()
    assert torch.equal(got, want)
