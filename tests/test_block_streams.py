"""ActiveBlock with encode, run and the making of the block on streams of their own, none of which waits
for another: the bits of one stream.  A spinning kernel of some 50 ms holds a stream back."""
import math

import pytest
import torch

from ops_check import DEV

H16 = torch.bfloat16
F, GH, GW, H, D_HEAD, DE, DF, L, S = 3, 8, 9, 4, 64, 64, 512, 70, 4
N, D, SCALE = GH * GW, H * D_HEAD, D_HEAD ** -0.5


def _hold(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)


class Case:
    def __init__(self):
        from paper_2606_06309_gb300.block import BlockWeights
        from paper_2606_06309_gb300.stepcore import StepCore, upload_plan
        g = torch.Generator().manual_seed(5)

        def lin(o, i):
            return (torch.randn(o, i, generator=g) / math.sqrt(i)).to(H16).to(DEV), None

        self.w = BlockWeights(lin(3 * D, D), lin(D, D), lin(D, D), lin(2 * D, DE), lin(D, D),
                              lin(DF, D), lin(D, DF))
        self.x0 = torch.randn(F * N, D, generator=g).to(H16).to(DEV)
        self.enc = [torch.randn(L, DE, generator=g).to(H16).to(DEV) for _ in range(2)]
        self.core = StepCore(F, N, N * 16, H, D_HEAD, upload_plan(F, S, [1, 0, 1], [2] * S, 0, DEV), DEV)
        self.core.compact(0)
        torch.cuda.synchronize()

    def block(self, dims=(24, 20, 20)):
        from paper_2606_06309_gb300.block import ActiveBlock
        return ActiveBlock(self.core, GH, GW, self.w, dims, H)

    def plain(self, which, mask=None, **kw):
        """All on one stream, with waits."""
        b, x = self.block(**kw), self.x0.clone()
        b.encode(self.enc[which], mask=mask)
        torch.cuda.synchronize()
        b.run(0, x, SCALE)
        torch.cuda.synchronize()
        assert self.core.status.item() == 0
        return x


@pytest.fixture()
def case(cuda_lib):
    return Case()


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [False, True])
def test_run_waits_for_the_states(case, handle):
    want, x = case.plain(0), case.x0.clone()
    b = case.block()
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    _hold(a)
    b.encode(case.enc[0], stream=a.cuda_stream if handle else a)
    b.run(0, x, SCALE, stream=c.cuda_stream if handle else c)
    torch.cuda.synchronize()
    assert case.core.status.item() == 0
    assert torch.equal(x, want)


@pytest.mark.gpu
def test_run_waits_for_the_buffers(case):
    dims = (0, 0, 0)  # no tables, whose upload would wait
    want, x = case.plain(0, dims=dims), case.x0.clone()
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    _hold(a)
    with torch.cuda.stream(a):
        b = case.block(dims=dims)
    b.encode(case.enc[0], stream=c)
    b.run(0, x, SCALE, stream=c)
    torch.cuda.synchronize()
    assert case.core.status.item() == 0
    assert torch.equal(x, want)


@pytest.mark.gpu
def test_states_are_kept_until_they_are_read(case):
    """A second encode, and what is allocated on its stream, while a run with the first ones is held up."""
    mask = (torch.arange(L, device=DEV) % 3 != 0).to(torch.uint8)
    want = [case.plain(i, mask) for i in range(2)]
    x = [case.x0.clone() for _ in range(2)]
    b = case.block()
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        b.encode(case.enc[0], mask=mask.clone())
    first = b.enc.data_ptr()
    a.synchronize()
    _hold(c)
    b.run(0, x[0], SCALE, stream=c)
    with torch.cuda.stream(a):
        b.encode(case.enc[1], mask=mask.clone())
        junk = [torch.full((L, 2, H, D_HEAD), math.nan, dtype=H16, device=DEV) for _ in range(8)]
        junk += [torch.zeros(L, dtype=torch.uint8, device=DEV) for _ in range(8)]
    assert all(t.data_ptr() != first for t in junk)
    b.run(0, x[1], SCALE, stream=c)
    torch.cuda.synchronize()
    assert case.core.status.item() == 0
    for got, w in zip(x, want):
        assert torch.equal(got, w)
    b.encode(case.enc[0])  # the first ones are let go
    assert all(o[0].data_ptr() != first for o in b._enc_old)


@pytest.mark.gpu
@pytest.mark.parametrize("encode_inside", [False, True])
def test_block_in_a_graph(case, encode_inside):
    want, x = case.plain(0), case.x0.clone()
    b = case.block()
    b.encode(case.enc[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        if encode_inside:
            b.encode(case.enc[1])
        b.run(0, x, SCALE)
    case.enc[1].copy_(case.enc[0])
    g.replay()
    torch.cuda.synchronize()
    assert case.core.status.item() == 0
    assert torch.equal(x, want)
    y = case.x0.clone()  # and outside again, over the states that the graph left
    b.run(0, y, SCALE)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
