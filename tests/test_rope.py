"""rf_rope and rf_rope_table: rotary positions over time, height and width.

Bound per element, derived: the table's cos and sin are rounded once (2^-25 each), the products and
the sum of a pair in fp32 (2^-24 of each product and of the result), so a result before its
rounding is off by less than 2^-22 (|x0| + |x1|); then it is rounded to the stored type.
"""
import math

import numpy as np
import pytest
import torch

from ops_check import DEV, DTYPES, SENTINEL, check, lists, rounding, row_mask
from oracle import ops_oracle

# F, gh, gw, frames, Hq, Hk, d, dims
SHAPES = [
    (4, 8, 8, (0, 3), 2, 2, 64, (24, 20, 20)),       # the smallest video, keyframes only
    (7, 17, 59, (0, 2, 3, 5, 6), 5, 1, 128, (16, 40, 40)),  # odd grid, part of the head rotated
    (3, 5, 7, (1,), 3, 0, 128, (44, 42, 42)),        # queries only, odd pairs per axis
    (1, 1, 1, (0,), 1, 1, 8, (8, 0, 0)),             # one token, one axis
    (2, 3, 1, (), 2, 2, 64, (0, 64, 0)),             # nothing active
    (3, 2, 9, (0, 1, 2), 9, 2, 256, (100, 2, 50)),   # the widest head, R/2 off the vectors
    (5, 4, 3, (4,), 1, 4, 72, (0, 0, 24)),           # one short axis, the rest passes through
    (2, 1, 300, (0, 1), 4, 4, 64, (0, 0, 0)),        # nothing rotates
]


def _tables(rf, pos, dims, base=10000.0):
    return [torch.from_numpy(rf.rf_rope_table(p, dim, base)).to(DEV) if dim else None
            for p, dim in zip(pos, dims)]


def _bound(X, Y, dims, pairing, dtype):
    """Per element of the rotated part; the rest is exact."""
    x = X.detach().cpu().double().abs()
    R = sum(dims)
    b = torch.full(Y.shape, 1e-300, dtype=torch.float64)
    if pairing == "interleaved":
        s = (x[..., 0:R:2] + x[..., 1:R:2]).repeat_interleave(2, dim=-1)
    else:
        s = (x[..., :R // 2] + x[..., R // 2:R]).repeat(1, 1, 2)
    b[..., :R] = 2.0 ** -22 * s * 1.01 + rounding(Y[..., :R], dtype)
    return b


@pytest.mark.gpu
@pytest.mark.parametrize("pairing", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rope_matches_oracle(cuda_lib, shape, dtype, pairing):
    rf = cuda_lib
    F, gh, gw, frames, Hq, Hk, d, dims = SHAPES[shape]
    dt, N = DTYPES[dtype], gh * gw
    g = torch.Generator().manual_seed(100 + shape)
    pos = [np.arange(F) * 1.5 + 0.25, np.arange(gh), np.arange(gw) - 2.0]  # any positions
    # a row holds more than the heads: queries and keys are slices of a fused buffer
    fused = torch.randn(F * N, Hq + Hk + 2, d, generator=g).to(dt).to(DEV)
    Xq, Xk = fused[:, :Hq], fused[:, Hq:Hq + Hk] if Hk else None
    act, cnt = lists(frames, F, N)
    tables = _tables(rf, pos, dims)
    rows = row_mask(frames, F, N)
    for inverse in (False, True):
        Yq = torch.full((F * N, Hq, d), SENTINEL, dtype=dt, device=DEV)
        Yk = torch.full((F * N, Hk, d), SENTINEL, dtype=dt, device=DEV) if Hk else None
        rf.rf_rope(Yq, Xq, Yk, Xk, F, gh, gw, dims, tables, pairing=pairing, inverse=inverse,
                   active=act, counts=cnt)
        torch.cuda.synchronize()
        for X, Y in ((Xq, Yq), (Xk, Yk)):
            if X is None:
                continue
            want = ops_oracle.rope(X, frames, pos, dims, pairing=pairing, inverse=inverse)
            check(Y, want, _bound(X, want, dims, pairing, dt), rows, f"rope {shape} {dtype}")
            # what passes through keeps its bits
            assert torch.equal(Y[rows.to(DEV)][..., sum(dims):], X[rows.to(DEV)][..., sum(dims):])


@pytest.mark.gpu
def test_rope_in_place_without_a_list_and_back(cuda_lib):
    """All frames (no list), in place; the inverse takes it back: each way is within the bound, so the
    way back is within twice 2^-22 (|x0| + |x1|), a rotation leaving |x0| + |x1| within sqrt 2."""
    rf = cuda_lib
    F, gh, gw, H, d, dims = 3, 6, 11, 4, 128, (44, 42, 42)
    X = torch.randn(F * gh * gw, H, d, generator=torch.Generator().manual_seed(3)).to(DEV)
    pos = [np.arange(n) for n in (F, gh, gw)]
    tables = _tables(rf, pos, dims)
    Y, K = X.clone(), X.clone()
    rf.rf_rope(Y, Y, K, K, F, gh, gw, dims, tables)
    assert torch.equal(Y, K)
    assert (Y - X).abs().max() > 1.0
    rf.rf_rope(Y, Y, None, None, F, gh, gw, dims, tables, inverse=True)
    s = (X[..., 0::2].abs() + X[..., 1::2].abs()).repeat_interleave(2, dim=-1)
    assert ((Y - X).abs() <= 2.0 ** -22 * (1 + math.sqrt(2.0)) * s + 2.0 ** -24 * X.abs()).all()


@pytest.mark.gpu
def test_rope_gradient_is_the_inverse(cuda_lib):
    """d<G, rope(X)>/dX by central differences (the map is linear: exact up to the rounding of
    <G, .> in 64 bits of fp32 outputs, 2^-22 (|x0| + |x1|) |g| over the step) against the inverse."""
    rf = cuda_lib
    F, gh, gw, H, d, dims = 2, 2, 3, 1, 16, (4, 6, 4)
    g = torch.Generator().manual_seed(5)
    X, G = (torch.randn(F * gh * gw, H, d, generator=g) for _ in range(2))
    tables = _tables(rf, [np.arange(n) for n in (F, gh, gw)], dims)

    def f(x, inverse=False):
        y = torch.empty_like(x, device=DEV)
        rf.rf_rope(y, x.to(DEV), None, None, F, gh, gw, dims, tables, pairing="half",
                   inverse=inverse)
        return y.cpu().double()

    grad = f(G, inverse=True)
    h = 0.5
    worst = 0.0
    for i in range(0, X.numel(), 5):
        e = torch.zeros(X.numel())
        e[i] = h
        e = e.view_as(X)
        diff = ((f(X + e) - f(X - e)) * G.double()).sum().item() / (2 * h)
        # two outputs of two evaluations differ, each off by 2^-22 (|x0| + |x1|) <= 2^-22 * 12
        worst = max(worst, abs(diff - grad.flatten()[i].item()))
    assert worst <= 4 * 2.0 ** -22 * 12 * G.abs().max().item() / (2 * h)


@pytest.mark.gpu
def test_rope_commutes_with_the_projection_of_cached_keys(cuda_lib):
    """Eq. 3 of rotated keys is the rotation of Eq. 3: why keys are cached rotated.  In fp32, both
    orders are within a few roundings (2^-22 each) of |alpha k1| + |beta k0| of the pair."""
    rf = cuda_lib
    F, gh, gw, H, d, dims = 2, 3, 4, 2, 64, (24, 20, 20)
    g = torch.Generator().manual_seed(6)
    K0, K1 = (torch.randn(F * gh * gw, H, d, generator=g).to(DEV) for _ in range(2))
    tables = _tables(rf, [np.arange(n) for n in (F, gh, gw)], dims)
    a = 0.375
    mixed, r0, r1, rm = (torch.empty_like(K0) for _ in range(4))
    torch.add(a * K1, K0, alpha=1 - a, out=mixed)
    for x, y in ((K0, r0), (K1, r1), (mixed, rm)):
        rf.rf_rope(y, x, None, None, F, gh, gw, dims, tables)
    s = (K0.abs() + K1.abs())
    s = (s[..., 0::2] + s[..., 1::2]).repeat_interleave(2, dim=-1)
    assert ((a * r1 + (1 - a) * r0 - rm).abs() <= 4 * 2.0 ** -22 * s).all()


@pytest.mark.gpu
def test_rope_keeps_infinities_and_nan_in_their_pairs(cuda_lib):
    rf = cuda_lib
    d, dims = 64, (16, 16, 16)
    X = torch.randn(12, 2, d, generator=torch.Generator().manual_seed(8))
    X[3, 1, 4], X[5, 0, 60] = math.nan, math.inf
    tables = _tables(rf, [np.arange(n) for n in (2, 2, 3)], dims)
    Y = torch.empty_like(X, device=DEV)
    rf.rf_rope(Y, X.to(DEV), None, None, 2, 2, 3, dims, tables)
    bad = torch.zeros(X.shape, dtype=torch.bool)
    bad[3, 1, 4:6] = True
    assert torch.equal(torch.isnan(Y.cpu()), bad)
    assert Y[5, 0, 60].item() == math.inf  # past R: passes through


def test_table_is_64_bit_and_rounded_once():
    import paper_2606_06309_gb300 as rf
    pos = [0.0, 1.0, 17.25, -3.0, 118799.0]
    t = rf.rf_rope_table(pos, 44, 10000.0)
    assert t.shape == (5, 22, 2) and t.dtype == np.float32
    for i, p in enumerate(pos):
        for j in range(22):
            a = p * 10000.0 ** (-2.0 * j / 44)
            # the angle itself is rounded in 64 bits: 2^-52 of it at most, twice
            tol = 2.0 ** -25 + abs(a) * 2.0 ** -51
            assert abs(t[i, j, 0] - math.cos(a)) <= tol and abs(t[i, j, 1] - math.sin(a)) <= tol


def test_rope_refuses_bad_arguments():
    import paper_2606_06309_gb300 as rf
    lib = rf.load()
    P = 256
    ok = [P, P, 256, 256, 2, P, P, 256, 256, 2, 0, 4, 8, 8, 128, 44, 42, 42, P, P, P, 0, 0, P, P,
          None]
    cases = [(0, None, 1), (1, None, 1), (2, 255, 1), (3, 260, 3), (4, 0, 1), (5, None, 1),
             (6, P + 8, 3), (9, 0, 1), (10, 7, 2), (11, 0, 1), (12, 0, 1), (13, 1 << 30, 1),
             (14, 12, 2), (14, 264, 2), (15, 45, 1), (15, 46, 1), (16, -2, 1), (18, None, 1),
             (19, P + 4, 3), (21, 2, 1), (23, None, 1), (24, None, 1)]
    for i, v, want in cases:
        args = list(ok)
        args[i] = v
        assert lib.rf_rope(*args) == want, (i, v)
    args = list(ok)
    args[0], args[2] = P, 512  # in place with two strides
    assert lib.rf_rope(*args) == 1
    for bad in (([1.0], 3, 10000.0), ([1.0], 0, 10000.0), ([], 4, 10000.0), ([1.0], 4, 0.0),
                ([math.nan], 4, 10000.0), ([1.0], 4, math.inf)):
        with pytest.raises(rf.RFError):
            rf.rf_rope_table(*bad)
    x = torch.zeros(6, 2, 64)
    for y, k, t in ((torch.zeros(6, 2, 32), None, [None] * 3),
                    (torch.zeros(6, 2, 64, dtype=torch.float16), None, [None] * 3),
                    (torch.zeros(6, 64, 2).transpose(1, 2), None, [None] * 3),
                    (x, torch.zeros(5, 1, 64), [None] * 3),
                    (x, None, [torch.zeros(1, 7, 2), None, None])):
        with pytest.raises(ValueError):
            rf.rf_rope(y, x, k, k, 1, 2, 3, (16, 0, 0), t, stream=0)
