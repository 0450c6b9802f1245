"""Shared pieces of the tests of rf_rope, rf_linear and rf_cross_attn."""
import torch

DEV = "cuda"
SENTINEL = 7.0  # rows the kernels must not write keep this value
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# Half the spacing of a type's values at |y|, relative to |y| at most (8, 11 and 24 significant
# bits), and half the spacing of its smallest values.
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def rounding(y, dtype):
    """Largest error of rounding the 64-bit values y to dtype."""
    return ROUND[dtype] * y.abs() + TINY[dtype]


def lists(frames, F, N):
    """Active list and counts on the device (unused entries hold frame 0)."""
    act = torch.tensor(list(frames) + [0] * (F - len(frames)), dtype=torch.int32, device=DEV)
    cnt = torch.tensor([len(frames), len(frames) * N], dtype=torch.int32, device=DEV)
    return act, cnt


def row_mask(frames, F, N):
    m = torch.zeros(F * N, dtype=torch.bool)
    for f in frames:
        m[f * N:(f + 1) * N] = True
    return m


def check(got, want, bound, rows, label=""):
    """|got - want| <= bound on the given rows (want 64-bit), SENTINEL on the others."""
    got = got.detach().cpu().double()
    assert (got[~rows] == SENTINEL).all(), f"{label}: a row of a skipped frame was written"
    g, w, b = got[rows], want[rows], bound[rows]
    assert torch.isfinite(g).all(), f"{label}: non-finite result"
    ratio = ((g - w).abs() / b).max().item() if g.numel() else 0.0
    print(f"{label}: worst error {ratio:.3f} of its bound")
    assert ratio <= 1.0, f"{label}: {ratio} of the bound"
