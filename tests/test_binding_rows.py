"""The bindings' reading of strides: what a row's stride is where torch leaves it open."""
import pytest
import torch

import paper_2606_06309_gb300 as rf


def test_row_strides():
    rows = lambda t: rf._rows("f", "t", t, tuple(t.shape))  # noqa: E731
    assert rows(torch.zeros(4, 24)) == 24
    assert rows(torch.zeros(4, 32)[:, :24]) == 32
    assert rows(torch.zeros(1, 32)[:, :17]) == 32    # one row of a wider buffer keeps its stride
    assert rows(torch.zeros(1, 17)) == 17
    assert rows(torch.zeros(4, 3, 8)) == 24
    assert rows(torch.zeros(4, 5, 8)[:, :3]) == 40
    assert rows(torch.zeros(1, 5, 8)[:, :3]) == 40
    assert rows(torch.zeros(6, 2, 3, 8)[:, 1]) == 48
    assert rows(torch.zeros(0, 3, 8)) == 24
    for bad in (torch.zeros(24, 4).T, torch.zeros(4, 48)[:, ::2], torch.zeros(4, 3, 16)[..., :8]):
        with pytest.raises(ValueError):
            rows(bad)
    with pytest.raises(ValueError):
        rf._rows("f", "t", torch.zeros(4, 24), (4, 23))


def test_row_addresses():
    b = torch.zeros(32)
    assert rf._row("f", "b", b, 32) == b.data_ptr()
    assert rf._row("f", "b", b[5:9], 4) == b.data_ptr() + 20
    assert rf._row("f", "b", b[None], 32) == b.data_ptr()
    assert rf._row("f", "b", b[::32], 1) == b.data_ptr()
    for bad in (b[:31], b[::2], b[:16].view(2, 8)):
        with pytest.raises(ValueError):
            rf._row("f", "b", bad, bad.numel() if bad.dim() > 1 or bad.stride(0) > 1 else 32)
