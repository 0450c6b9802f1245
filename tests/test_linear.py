"""rf_linear: matrix product with bias, activation, gate and residual.

Bound per element, derived.  z = sum + bias: each of the K + 1 additions in fp32 loses at most one
unit 2^-23 of a partial sum, which is at most S = sum |x w| + |bias|: |dz| <= (K + 1) 2^-23 S.  The
activations change by at most 1.2 |dz| (the largest slope of gelu is 1.13, of silu 1.10) and are
themselves evaluated to within 2^-16 of their value (the argument of the exponential is rounded:
|s| 2^-22 of the result, |s| < 64; beyond, the value is below e^-60 |z|) plus 2^-20 |z|.  Gate and
residual round once each (2^-23 of their results), then the result is rounded to its type.
"""
import math

import pytest
import torch

from ops_check import DEV, DTYPES, SENTINEL, check, lists, rounding, row_mask
from oracle import ops_oracle

# F, N, frames, K, O
SHAPES = [
    (1, 1, (0,), 64, 128),               # one row
    (1, 1, (0,), 1000, 777),             # one row, odd sizes, K split over a cluster
    (1, 16, (0,), 8, 8),                 # the smallest product
    (1, 1, (0,), 1, 1),
    (5, 3, (0, 2, 4), 256, 130),         # frames of three tokens: gathered row by row
    (33, 1, tuple(range(0, 33, 2)), 512, 96),
    (1, 333, (0,), 1000, 777),
    (4, 64, (0, 3), 128, 256),
    (7, 100, (1, 2, 6), 320, 200),       # tiles across frames that are padded to 8 rows
    (3, 700, (0, 2), 192, 1536),         # more rows than a tile
    (6, 1003, (0, 1, 2, 4, 5), 77, 3000),  # many tiles: pairs of CTAs, K within one block
    (3, 1560, (0, 2), 200, 2500),
    (4, 1100, (0, 1, 3), 72, 2501),      # many tiles, rows of results off every vector's boundary
    (2, 40, (), 64, 64),                 # nothing active
    (300, 2, tuple(range(0, 300, 3)), 64, 1600),
    (300, 5, tuple(range(1, 300, 2)), 72, 3000),  # pairs of CTAs on frames of five tokens
    (40, 7, tuple(range(40)), 520, 300),          # tiles of whole frames of seven tokens
]
OPTIONS = [  # bias, act, gate, residual, out32
    (False, None, None, False, False),
    (True, "gelu_tanh", None, False, False),
    (True, "gelu", "frame", True, True),
    (True, "silu", "shared", True, False),
    (False, None, "frame", True, False),
]


def _pad(n):
    return (n + 7) // 8 * 8


def _inputs(F, N, K, O, dt, out, seed, bias, gate, residual, pad=8):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(F * N, _pad(K), generator=g).to(dt).to(DEV)[:, :K]
    W = (torch.randn(O, _pad(K) + 8, generator=g) / math.sqrt(K)).to(dt).to(DEV)[:, :K]
    b = torch.randn(O, generator=g).to(dt).to(DEV) if bias else None
    ga = None
    if gate == "shared":
        ga = torch.randn(O, generator=g).to(DEV)
    elif gate == "frame":
        ga = torch.randn(F, O + 4, generator=g).to(DEV)[:, :O]
    R = torch.randn(F * N, O + pad, generator=g).to(out).to(DEV)[:, :O] if residual else None
    return X, W, b, ga, R


def _bound(want, S, X, W, K, act, gate, residual, frames, N, out):
    lin, _ = ops_oracle.linear(X, W, frames, N)  # without the epilogue, for |z|
    dz = (K + 1) * 2.0 ** -23 * S
    if act is not None:
        z = S  # |z| <= S
        dz = 1.2 * dz + 2.0 ** -16 * z + 2.0 ** -20 * z
    a = want.clone()
    rows = row_mask(frames, lin.shape[0] // N, N)
    if residual is not None:
        a = want - residual.cpu().double()
    b = dz
    if gate is not None:
        g = gate.cpu().double()
        g = g.expand(lin.shape) if g.dim() == 1 else g.repeat_interleave(N, dim=0)
        b = b * g.abs() + 2.0 ** -23 * a.abs()
    b = b + 2.0 ** -23 * (a.abs() + want.abs())
    b = b * 1.01 + rounding(want, out)
    b[~rows] = 1.0
    return b


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("option", range(len(OPTIONS)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_linear_matches_oracle(cuda_lib, shape, option, dtype):
    rf = cuda_lib
    F, N, frames, K, O = SHAPES[shape]
    bias, act, gate, residual, out32 = OPTIONS[option]
    dt = DTYPES[dtype]
    out = torch.float32 if out32 else dt
    # option 3: rows of the residual off the 16-byte boundaries
    X, W, b, ga, R = _inputs(F, N, K, O, dt, out, 7 + shape, bias, gate, residual,
                             pad=3 if option == 3 else 8)
    act_l, cnt = lists(frames, F, N)
    # options 1 and 4: result rows off the 16-byte boundaries (1: of an odd number of elements)
    ld = {1: O | 1, 4: O + 2 + O % 2}.get(option, _pad(O))
    Y = torch.full((F * N, ld), SENTINEL, dtype=out, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    rf.rf_linear(Y[:, :O], X, W, F, N, bias=b, act=act, gate=ga, residual=R, active=act_l,
                 counts=cnt, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    assert (Y[:, O:].float() == SENTINEL).all(), "columns past the row were written"
    if not frames:
        assert (Y.float() == SENTINEL).all()
        return
    want, S = ops_oracle.linear(X, W, frames, N, b, act, ga, R)
    check(Y[:, :O], want, _bound(want, S, X, W, K, act, ga, R, frames, N, out),
          row_mask(frames, F, N), f"linear {SHAPES[shape]} {option} {dtype}")


@pytest.mark.gpu
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_linear_exact_on_whole_numbers(cuda_lib, shape):
    """Small whole numbers: every product and sum is exact, so is the result, bit for bit, and a
    lost or doubled element shows.  No list: every frame is computed."""
    rf = cuda_lib
    F, N, _, K, O = SHAPES[shape]
    g = torch.Generator().manual_seed(shape)
    X = torch.randint(-8, 9, (F * N, _pad(K)), generator=g)[:, :K]
    W = torch.randint(-8, 9, (O, _pad(K)), generator=g)[:, :K]
    R = torch.randint(-999, 1000, (F * N, O), generator=g)
    b = torch.randint(-99, 100, (O,), generator=g)
    gate = torch.randint(-3, 4, (F, O), generator=g)
    want = (X @ W.T + b) * gate.repeat_interleave(N, dim=0) + R

    def dev(t, dt):  # rows of K elements on 16-byte boundaries
        buf = torch.zeros(t.shape[0], _pad(t.shape[1]), dtype=dt, device=DEV)
        buf[:, :t.shape[1]] = t.to(DEV)
        return buf[:, :t.shape[1]]

    Y = R.float().to(DEV)
    rf.rf_linear(Y, dev(X, torch.bfloat16), dev(W, torch.bfloat16), F, N,
                 bias=b.to(DEV).to(torch.bfloat16), gate=gate.float().to(DEV), residual=Y)
    torch.cuda.synchronize()
    assert torch.equal(Y.cpu().double(), want.double())


@pytest.mark.gpu
def test_linear_rows_do_not_mix(cuda_lib):
    """NaN and infinities of skipped frames, of the padding behind a row, and of one active row do not
    reach other rows."""
    rf = cuda_lib
    F, N, K, O = 5, 100, 72, 160
    g = torch.Generator().manual_seed(2)
    buf = torch.randn(F * N, 96, generator=g).to(torch.bfloat16)
    clean = buf.clone()
    frames = (1, 3)
    skipped = ~row_mask(frames, F, N)
    buf[skipped] = math.nan
    buf[:, K:] = math.inf
    buf[N + 7, 3] = math.nan
    W = torch.randn(O, K, generator=g).to(torch.bfloat16).to(DEV)
    act, cnt = lists(frames, F, N)
    out = []
    for x in (buf, clean):
        Y = torch.full((F * N, O), SENTINEL, device=DEV)
        rf.rf_linear(Y, x.to(DEV)[:, :K], W, F, N, active=act, counts=cnt)
        out.append(Y.cpu())
    bad, good = out
    assert torch.isnan(bad[N + 7]).all()
    bad[N + 7] = good[N + 7]
    assert torch.equal(bad, good)


@pytest.mark.gpu
def test_linear_on_another_stream_and_in_a_graph(cuda_lib):
    rf = cuda_lib
    F, N, K, O = 2, 300, 128, 512
    X, W, b, _, R = _inputs(F, N, K, O, torch.bfloat16, torch.bfloat16, 4, True, None, True)
    Y0, Y1 = (torch.zeros(F * N, O, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rf.rf_linear(Y0, X, W, F, N, bias=b, act="silu", residual=R)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        rf.rf_linear(Y1, X, W, F, N, bias=b, act="silu", residual=R)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y0, Y1)
    Y1.zero_()
    torch.cuda.synchronize()
    rf.rf_linear(Y1, X, W, F, N, bias=b, act="silu", residual=R, stream=s)
    s.synchronize()
    assert torch.equal(Y0, Y1)


def test_linear_refuses_bad_arguments():
    import paper_2606_06309_gb300 as rf
    lib = rf.load()
    P = 256
    ok = [P, 256, 0, P, 128, P, 128, 0, 4, 64, 128, 256, P, 0, P, 256, P, 256, P, P, None, None]
    cases = [(0, None, 1), (3, None, 1), (5, None, 1), (7, 2, 2), (7, 9, 2), (2, 1, 2), (8, 0, 1),
             (9, 0, 1), (10, 0, 1), (11, 0, 1), (13, 4, 1), (13, -1, 1), (1, 255, 1), (4, 120, 1),
             (4, 129, 3), (6, 130, 3), (6, 64, 1), (15, 8, 1), (17, 8, 1), (3, P + 2, 3),
             (5, P + 8, 3), (0, P + 1, 3), (12, P + 1, 3), (14, P + 2, 3), (16, P + 1, 3),
             (18, None, 1), (19, None, 1), (9, 1 << 30, 1), (11, 0x7FFFFFFF, 1)]
    for i, v, want in cases:
        args = list(ok)
        args[i] = v
        assert lib.rf_linear(*args) == want, (i, v)
    z = torch.zeros
    h = torch.bfloat16
    X, W, Y = z(6, 16, dtype=h), z(24, 16, dtype=h), z(6, 24, dtype=h)
    for kw, y in ((dict(), z(6, 25, dtype=h)), (dict(bias=z(24)), Y), (dict(bias=z(23, dtype=h)), Y),
                  (dict(gate=z(24, dtype=h)), Y), (dict(gate=z(5, 24)), Y),
                  (dict(residual=z(6, 24)), Y), (dict(residual=z(5, 24, dtype=h)), Y),
                  (dict(), z(24, 6, dtype=h).T)):
        with pytest.raises(ValueError):
            rf.rf_linear(y, X, W, 2, 3, stream=0, **kw)
    with pytest.raises(KeyError):
        rf.rf_linear(Y, X, W, 2, 3, act="relu6", stream=0)
