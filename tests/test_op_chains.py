"""Calls one behind the other on a stream, each from what the one before it wrote.

A launch may begin while the one before it ends; results must be the bits that a wait between the
calls gives, whatever kinds of calls, copies and torch operations follow one another.
"""
import math

import pytest
import torch

from ops_check import DEV, lists

H16 = torch.bfloat16


def _chain(rf, between, rounds, F, N, H, d, L, frames):
    g = torch.Generator().manual_seed(3)
    D, T = H * d, F * N
    act, cnt = lists(frames, F, N)
    W = [(torch.randn(D, D, generator=g) / math.sqrt(D)).to(H16).to(DEV) for _ in range(2)]
    E = (torch.randn(2 * D, D, generator=g) / math.sqrt(D)).to(H16).to(DEV)
    states = torch.randn(L, D, generator=g).to(H16).to(DEV)
    x = torch.randn(T, D, generator=g).to(H16).to(DEV)
    tables = [torch.from_numpy(rf.rf_rope_table(range(n), dim, 1e4)).to(DEV)
              for n, dim in ((F, 24), (1, 20), (N, 20))]
    y, o = torch.zeros_like(x), torch.zeros(T, H, d, dtype=H16, device=DEV)
    kv = torch.zeros(L, 2, H, d, dtype=H16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    on = dict(active=act, counts=cnt)
    for r in range(rounds):
        rf.rf_linear(kv.view(L, -1), states, E, 1, L, status=status)
        between()
        rf.rf_linear(y, x, W[0], F, N, status=status, act="silu", **on)
        between()
        q = y.view(T, H, d)
        rf.rf_rope(q, q, None, None, F, 1, N, (24, 20, 20), tables, **on)
        between()
        rf.rf_cross_attn(o, None, q, kv[:, 0], kv[:, 1], F, N, d ** -0.5, status=status, **on)
        between()
        rf.rf_linear(x, o.view(T, D), W[1], F, N, residual=x, status=status, **on)
        between()
        if r % 2:
            y.zero_()          # other kernels in the chain
            x.mul_(0.5)
        states = states.roll(1, 0)
    torch.cuda.synchronize()
    assert status.item() == 0
    return x, y, o


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 40, 4, 64, 50, (0, 2)), (5, 300, 8, 64, 700, (0, 1, 4)),
                                   (4, 1, 4, 64, 3000, (1, 3)), (2, 64, 4, 64, 64, ())])
def test_chain_needs_no_waits(cuda_lib, shape):
    F, N, H, d, L, frames = shape
    want = _chain(cuda_lib, torch.cuda.synchronize, 12, F, N, H, d, L, frames)
    for _ in range(3):
        got = _chain(cuda_lib, lambda: None, 12, F, N, H, d, L, frames)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
