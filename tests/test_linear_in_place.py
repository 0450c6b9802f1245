"""rf_linear refuses a residual that begins where Y does with another stride: rows would be read after
others were written over them."""
import torch


def test_refused_with_two_strides():
    import paper_2606_06309_gb300 as rf
    lib = rf.load()
    P = 256
    ok = [P, 256, 0, P, 128, P, 128, 0, 4, 64, 128, 256, P, 0, P, 256, P, 256, P, P, None, None]
    for y, r in ((256, 264), (512, 256)):
        args = list(ok)
        args[1], args[17] = y, r
        assert lib.rf_linear(*args) == 1
        assert b"two strides" in lib.rf_last_error()


def test_binding_refuses_views_of_one_buffer():
    import pytest

    import paper_2606_06309_gb300 as rf
    h = torch.bfloat16
    buf, X, W = torch.zeros(6, 32, dtype=h), torch.zeros(3, 16, dtype=h), torch.zeros(16, 16, dtype=h)
    with pytest.raises(rf.RFError, match="two strides"):
        rf.rf_linear(buf[:3, :16], X, W, 1, 3, residual=buf.view(3, 64)[:, :16], stream=0)
