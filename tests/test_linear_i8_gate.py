"""The row of a per-frame gate that rf_linear_i8's pairs read for rows behind the last token: one of a frame that
there is, whatever the number of tokens.  The rows' arithmetic is checked on the CPU; on the GPU, results without a
list where the last tile's second half has no token, and NaN behind the gate's last row."""
import math
import os
import shutil
import subprocess

import pytest
import torch

from ops_check import DEV
from oracle import ops_oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_gate_row_is_of_a_frame(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "gate_check"
    r = subprocess.run([gxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I",
                        os.path.join(ROOT, "paper_2606_06309_gb300", "csrc"),
                        os.path.join(ROOT, "tests", "c_abi", "gate_check.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("F,N,O", [(3, 1111, 1536),   # 3333 tokens: the last half begins behind them
                                   (1, 1027, 1920),   # one frame
                                   (7, 333, 1344),    # halves of two frames, 2331 tokens
                                   (5, 1030, 960)])   # 5150: the padding ends inside the last half
def test_gate_without_a_list(cuda_lib, F, N, O):
    """Whole numbers throughout, so every result is exact: sums below 2^24, times a gate below 2^4, fp32 below 2^24
    by the digits' and K's choice (72 * 20^2 * 15 = 432,000)."""
    rf = cuda_lib
    T, K = F * N, 72
    g = torch.Generator().manual_seed(N)
    X = torch.randint(-20, 21, (T, 80), generator=g).to(torch.int8)
    W = torch.randint(-20, 21, (O, 80), generator=g).to(torch.int8)
    G = torch.full((F + 2, O), math.nan)
    G[:F] = torch.randint(-15, 16, (F, O), generator=g).float()
    gate, one = G.to(DEV)[:F], torch.ones(max(T, O), device=DEV)
    Y = torch.full((T, O), math.nan, device=DEV)
    rf.rf_linear_i8(Y, X.to(DEV)[:, :K], one[:T], W.to(DEV)[:, :K], one[:O], F, N, gate=gate)
    torch.cuda.synchronize()
    want, _, _ = ops_oracle.linear_i8(X[:, :K], torch.ones(T), W[:, :K], torch.ones(O), range(F), N, gate=G[:F])
    assert torch.equal(Y.cpu().double(), want)
