"""A chain of the operators in a captured graph, replayed: the bits of the same calls with a wait after each.

A launch may begin while the one before it ends, in a graph as on a stream; copies and torch's kernels
stand between some of them.
"""
import math

import pytest
import torch

from ops_check import DEV, lists

H16 = torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 40, 4, 64, 50, (0, 2)), (5, 300, 8, 64, 700, (0, 1, 4)),
                                   (4, 1, 4, 64, 3000, (1, 3)), (2, 64, 4, 64, 64, ())])
def test_chain_in_a_graph(cuda_lib, shape):
    rf = cuda_lib
    F, N, H, d, L, frames = shape
    D, T = H * d, F * N
    g = torch.Generator().manual_seed(7)
    act, cnt = lists(frames, F, N)
    W = [(torch.randn(D, D, generator=g) / math.sqrt(D)).to(H16).to(DEV) for _ in range(2)]
    E = (torch.randn(2 * D, D, generator=g) / math.sqrt(D)).to(H16).to(DEV)
    states = torch.randn(L, D, generator=g).to(H16).to(DEV)
    x0 = torch.randn(T, D, generator=g).to(H16).to(DEV)
    tables = [torch.from_numpy(rf.rf_rope_table(range(n), dim, 1e4)).to(DEV)
              for n, dim in ((F, 24), (1, 20), (N, 20))]
    x, y = x0.clone(), torch.zeros_like(x0)
    o, kv = torch.zeros(T, H, d, dtype=H16, device=DEV), torch.zeros(L, 2, H, d, dtype=H16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    on = dict(active=act, counts=cnt)

    def chain(between=lambda: None, rounds=4):
        for r in range(rounds):
            q = y.view(T, H, d)
            for call in (lambda: rf.rf_linear(kv.view(L, -1), states, E, 1, L, status=status),
                         lambda: rf.rf_linear(y, x, W[0], F, N, act="gelu", status=status, **on),
                         lambda: rf.rf_rope(q, q, None, None, F, 1, N, (24, 20, 20), tables, **on),
                         lambda: rf.rf_cross_attn(o, None, q, kv[:, 0], kv[:, 1], F, N, d ** -0.5,
                                                  status=status, **on),
                         lambda: rf.rf_linear(x, o.view(T, D), W[1], F, N, residual=x, status=status, **on)):
                call()
                between()
            if r % 2:
                states.copy_(states.flip(0))
                x.mul_(0.5)

    chain(torch.cuda.synchronize)
    chain(torch.cuda.synchronize)
    want = [t.clone() for t in (x, y, o, states)]
    assert status.item() == 0
    states.copy_(states)
    x.copy_(x0)  # (two chains leave states in their first order)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for t in (y, o):
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert status.item() == 0
    assert all(torch.equal(a, b) for a, b in zip((x, y, o, states), want))
