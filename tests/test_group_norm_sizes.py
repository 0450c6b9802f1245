"""rf_group_norm, rf_group_norm_bwd and rf_group_norm_workspace_bytes agree on the sizes that there are."""
import pytest
import torch

import paper_2606_06309_gb300 as rf

MOST = 0x7FFFFFFF - 65536  # tokens
HUGE = 1 << 62             # bytes of workspace that a call is told of


def _norm(F, N, C, G, bytes_):
    P = 256  # not read: the calls are refused on the host
    return rf.load().rf_group_norm(P, C, None, 2 * P, C, 0, F, N, C, G, None, None, 0, 1e-5, 0, None, P, bytes_, None,
                                   None, None)


def _bwd(F, N, C, G, bytes_):
    P = 256
    return rf.load().rf_group_norm_bwd(P, C, None, None, 2 * P, C, 3 * P, C, P, 0, F, N, C, G, None, None, 0, 0, P, bytes_,
                                       None, None, None)


@pytest.mark.parametrize("F,N,C,G", [(1, MOST + 1, 8, 1), (1, 0x7FFFFFFF, 8, 1), (1 << 20, 1 << 20, 8, 1),
                                     (0x7FFFFFFF, 2, 64, 8), (MOST + 1, 1, 8, 8),
                                     (1 << 30, 1, 65536, 1)])  # pieces beyond a grid at any alignment
def test_no_workspace_for_refused_sizes(F, N, C, G):
    assert _norm(F, N, C, G, HUGE) == 1 and _bwd(F, N, C, G, HUGE) == 1
    for dtype in (0, 1, 2):
        assert rf.load().rf_group_norm_workspace_bytes(F, N, C, G, dtype) == -1
    with pytest.raises(ValueError):
        rf.rf_group_norm_workspace_bytes(F, N, C, G, torch.bfloat16)


@pytest.mark.parametrize("F,N,C,G", [(1, MOST, 8, 1), (MOST, 1, 8, 8), (1, 1, 65536, 1), (1 << 27, 1, 264, 33),
                                     (7, 1003, 960, 32)])
def test_workspace_of_the_largest_sizes(F, N, C, G):
    """One byte less than the gradients need is refused; no size in between overflows."""
    n = rf.load().rf_group_norm_workspace_bytes(F, N, C, G, 0)
    assert n >= 8 * F * G
    assert _bwd(F, N, C, G, n - 1) == 1 and _norm(F, N, C, G, 8 * F * G - 1) == 1


@pytest.mark.gpu
def test_more_pieces_than_a_grid_has(cuda_lib):
    """2^30 rows of 65,536 single elements are 2^32 pieces: refused on the host, whatever the pointers are."""
    P = 258  # rows off the 16-byte boundaries
    got = cuda_lib.load().rf_group_norm(P, 65536, None, 2 * P, 65536, 0, 1, 1 << 30, 65536, 1, None, None, 0, 1e-5, 0, None,
                                        256, HUGE, None, None, None)
    assert got == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", [19400, 65536])
def test_a_refused_call_writes_nothing(cuda_lib, C, dtype):
    """Rows of 8 bits with more channels than shared memory has factors for: digits, scales and statistics stay."""
    F, N, G = 2, 100, 8
    X = torch.ones(F * N, C, dtype=dtype, device="cuda")
    Y, s = torch.full((F * N, C), 77, dtype=torch.int8, device="cuda"), torch.full((F * N,), 7.0, device="cuda")
    st = torch.full((F, G, 2), 7.0, device="cuda")
    ws = torch.zeros(rf.rf_group_norm_workspace_bytes(F, N, C, G, dtype), dtype=torch.uint8, device="cuda")
    with pytest.raises(rf.RFError):
        rf.rf_group_norm(Y, X, F, N, G, stats=st, scale=s, workspace=ws)
    torch.cuda.synchronize()
    assert (Y == 77).all() and (s == 7.0).all() and (st == 7.0).all() and not ws.any()
