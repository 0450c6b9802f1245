"""ActiveBlocks that share one set of buffers: the bits of blocks with their own, in the memory of one."""
from types import SimpleNamespace

import pytest
import torch

from ops_check import DEV
from test_block_layers import DIMS, GH, GW, HKV, H16, _case, _core, _trajectory


@pytest.mark.gpu
def test_shared_buffers(cuda_lib):
    from paper_2606_06309_gb300.block import ActiveBlock
    weights, kv, enc, _, x0 = _case(3)
    out = []
    for share in (False, True):
        core, blocks = _core(kv_cache=False), []
        for w in weights:
            blocks.append(ActiveBlock(core, GH, GW, w, DIMS, HKV, own_cache=True,
                                      buffers=blocks[0] if share and blocks else None))
        out.append(_trajectory(blocks, [core], kv, enc, x0))
        for name in ("qkv", "rows", "ffn"):
            assert len({getattr(b, name).data_ptr() for b in blocks}) == (1 if share else 3)
        assert len({b.cache[0].data_ptr() for b in blocks}) == 3
    assert torch.equal(*out)


@pytest.mark.gpu
def test_buffers_made_on_another_stream(cuda_lib):
    """The second block's run waits for the zeros that the first block's stream has still to write."""
    from paper_2606_06309_gb300.block import ActiveBlock
    weights, _, _, _, x0 = _case(2)
    core = _core(kv_cache=False)
    core.compact(0)
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    out = []
    for hold in (0, 100_000_000):
        x = x0.to(DEV)
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            torch.cuda._sleep(hold)
            first = ActiveBlock(core, GH, GW, weights[0], (0, 0, 0), HKV, own_cache=True)
        with torch.cuda.stream(c):
            b = ActiveBlock(core, GH, GW, weights[1], (0, 0, 0), HKV, own_cache=True, buffers=first)
        b.run(0, x, 0.125, stream=c)
        torch.cuda.synchronize()
        out.append(x)
    assert torch.equal(*out)


def test_refusals():
    from paper_2606_06309_gb300.block import ActiveBlock, BlockWeights

    def weights(ffn):
        return BlockWeights(*[(torch.zeros(*shape, dtype=H16), None) for shape in
                              ((192, 64), (64, 64), (64, 64), (128, 32), (64, 64), (ffn, 64), (64, ffn))])

    core = SimpleNamespace(F=2, N=6, H=1, d=64, Kc=None)
    # no axis rotates: nothing of this needs a GPU
    first = ActiveBlock(core, 2, 3, weights(256), (0, 0, 0), 1, own_cache=True)
    bare = ActiveBlock(core, 2, 3, weights(256), (0, 0, 0), 1)
    for kw in (dict(buffers=first), dict(buffers=bare, own_cache=True)):
        with pytest.raises(ValueError, match="without a cache"):
            ActiveBlock(core, 2, 3, weights(256), (0, 0, 0), 1, **kw)
    with pytest.raises(ValueError, match="ffn"):
        ActiveBlock(core, 2, 3, weights(128), (0, 0, 0), 1, own_cache=True, buffers=first)
    second = ActiveBlock(core, 2, 3, weights(256), (0, 0, 0), 1, own_cache=True, buffers=first)
    assert second.qkv is first.qkv and second.rows is first.rows and second.ffn is first.ffn
    assert second.cache[0] is not first.cache[0]
