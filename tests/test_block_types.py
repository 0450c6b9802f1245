"""ActiveBlock takes weights of the step core's type only: its attention reads bf16 whatever it is given."""
from types import SimpleNamespace

import pytest
import torch


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_block_refuses_other_types(dtype):
    from paper_2606_06309_gb300.block import ActiveBlock, BlockWeights
    w = BlockWeights(*[(torch.zeros(*shape, dtype=dtype), None) for shape in
                       ((192, 64), (64, 64), (64, 64), (128, 32), (64, 64), (256, 64), (64, 256))])
    core = SimpleNamespace(F=2, N=6, H=1, d=64, Kc=None)
    with pytest.raises(ValueError, match="bfloat16"):
        ActiveBlock(core, 2, 3, w, (24, 20, 20), 1)
