"""ActiveBlock on a stream other than the current one: the same bits as on the current one."""
import math

import pytest
import torch

from ops_check import DEV

H16 = torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [False, True])
def test_block_on_another_stream(cuda_lib, handle):
    from paper_2606_06309_gb300.block import ActiveBlock, BlockWeights
    from paper_2606_06309_gb300.stepcore import StepCore, upload_plan
    F, gh, gw, H, d, De, Df, L, S = 3, 8, 9, 4, 64, 64, 512, 70, 4
    N, D = gh * gw, H * d
    g = torch.Generator().manual_seed(5)

    def lin(o, i):
        return (torch.randn(o, i, generator=g) / math.sqrt(i)).to(H16).to(DEV), None

    w = BlockWeights(lin(3 * D, D), lin(D, D), lin(D, D), lin(2 * D, De), lin(D, D), lin(Df, D),
                     lin(D, Df))
    x0 = torch.randn(F * N, D, generator=g).to(H16).to(DEV)
    enc = torch.randn(L, De, generator=g).to(H16).to(DEV)
    K0, V0 = (torch.randn(F * N, H, d, generator=g).to(H16).to(DEV) for _ in range(2))

    def norm(h):  # on whatever stream is current where it is called
        return (h.float() * torch.rsqrt(h.float().square().mean(-1, keepdim=True) + 1e-6)).to(H16)

    def go(stream, arg):
        plan = upload_plan(F, S, [1, 0, 1], [2] * S, 0, DEV)
        core = StepCore(F, N, N * 16, H, d, plan, DEV)
        core.set_kv_cache(K0, V0)
        block = ActiveBlock(core, gh, gw, w, (24, 20, 20), H)
        x = x0.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            core.compact(0)
        block.encode(enc, stream=arg)
        for _ in range(4):
            block.run(0, x, d ** -0.5, norms=[norm] * 3, stream=arg)
        torch.cuda.synchronize()
        assert core.status.item() == 0
        return x

    want = go(torch.cuda.current_stream(), None)
    side = torch.cuda.Stream()
    got = go(side, side.cuda_stream if handle else side)
    assert torch.equal(got, want)
