"""rf_linear's loading warps on tiles of few boxes.

A tile across frames is loaded in boxes dealt to several warps, which all go round the ring of
stages.  Nothing holds the ring for a warp that has no box in it, so each that goes round has to have
one (the dealing is checked on the CPU); on the GPU, tiles of two to nine boxes over many more
stages than the ring has, exact in whole numbers.
"""
import os
import shutil
import subprocess

import pytest
import torch

from ops_check import DEV, SENTINEL, lists, row_mask

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_loading_warp_has_a_box(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "deal_check"
    r = subprocess.run([gxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I",
                        os.path.join(ROOT, "paper_2606_06309_gb300", "csrc"),
                        os.path.join(ROOT, "tests", "c_abi", "deal_check.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [
    (5, 3, (0, 2, 4), 4096, 130),              # three boxes of three tokens
    (9, 1, (0, 3, 5, 8), 8192, 64),            # four of one token
    (9, 5, (1, 2, 3, 5, 8), 4160, 300),        # five of five
    (9, 7, (0, 1, 3, 4, 6, 8), 4096, 128),     # six of seven
    (12, 2, (0, 1, 3, 4, 6, 7, 9, 10, 11), 4096, 96),  # nine of two
    (3, 40, (0, 2), 4096, 256),                # two of 32 rows and two of 8
    (8, 32, (0, 3, 5), 4096, 128),             # three of 32 rows
    (30, 96, tuple(range(0, 30, 2)), 2048, 2560),  # pairs: tiles of a few boxes of 32 rows
    (30, 104, tuple(range(1, 30, 2)), 2048, 2560),  # the same, some of one large and one small box
])
def test_tiles_of_few_boxes(cuda_lib, shape):
    F, N, frames, K, O = shape
    g = torch.Generator().manual_seed(N)
    X = torch.randint(-4, 5, (F * N, K), generator=g)
    W = torch.randint(-4, 5, (O, K), generator=g)
    want = torch.full((F * N, O), SENTINEL, dtype=torch.float64)
    rows = row_mask(frames, F, N)
    want[rows] = X[rows].double() @ W.T.double()
    act, cnt = lists(frames, F, N)
    h = torch.bfloat16
    x, w = X.to(DEV).to(h), W.to(DEV).to(h)
    Y = torch.full((F * N, O), SENTINEL, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(20):
        Y.fill_(SENTINEL)
        cuda_lib.rf_linear(Y, x, w, F, N, active=act, counts=cnt, status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
        assert torch.equal(Y.cpu().double(), want)
