"""rf_linear on a single row of any length: its stride, which no second row shows, is none that could be
off a boundary.  Exact in whole numbers."""
import pytest
import torch

from ops_check import DEV

H16 = torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("K,O", [(17, 40), (1, 8), (333, 777), (1001, 1), (7, 1)])
def test_one_row(cuda_lib, K, O):
    g = torch.Generator().manual_seed(K)
    x, w = (torch.randint(-8, 9, shape, generator=g) for shape in ((1, K), (O, K)))
    b = torch.randint(-99, 100, (O,), generator=g)
    want = (x @ w.T + b).float()
    W = torch.zeros(O, (K + 7) // 8 * 8, dtype=H16, device=DEV)
    W[:, :K] = w.to(DEV)
    Y = torch.zeros(1, O, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = dict(bias=b.to(DEV).to(H16), status=st)
    X = x.to(DEV).to(H16)  # a stride of K elements
    cuda_lib.rf_linear(Y, X, W[:, :K], 1, 1, **kw)
    torch.cuda.synchronize()
    assert st.item() == 0 and torch.equal(Y.cpu(), want)
    if O == 1:  # and of W
        Y.zero_()
        cuda_lib.rf_linear(Y, X, w.to(DEV).to(H16), 1, 1, **kw)
        torch.cuda.synchronize()
        assert st.item() == 0 and torch.equal(Y.cpu(), want)


@pytest.mark.gpu
def test_rows_off_the_boundaries_are_refused(cuda_lib):
    z = lambda *s: torch.zeros(*s, dtype=H16, device=DEV)  # noqa: E731
    for x, w in ((z(2, 17), z(8, 24)[:, :17]), (z(2, 24)[:, :17], z(8, 17)), (z(25)[1:18][None], z(8, 24)[:, :17])):
        with pytest.raises(cuda_lib.RFError) as e:
            cuda_lib.rf_linear(z(x.shape[0], 8), x, w, 1, x.shape[0])
        assert e.value.status == 3
