"""rf_cross_attn: the active frames' tokens over an encoder's states of another length.

Bounds, derived.  A score is off by ds = (d + 1) 2^-23 scale sum |q k| (each fp32 addition loses at
most one unit of a partial sum) + 2^-22 |s| (its scaling and the subtraction of the maximum), which
changes a probability by ds of itself, as does its exponential (2^-21).  Probabilities are rounded
to 16 bits for the product with V: u of each (u half the type's spacing; in fp16 also 2^-25, the
spacing of its smallest values, of a row whose largest probability is at least 1 before the division).
Sums over the keys lose (L + 1) 2^-23.  With P|V| = sum_j p_j |v_j|:
    |dO|   <= (u + 2 ds + 2^-19 + 2 (L + 1) 2^-23) P|V| [+ 2^-25 sum |v| in fp16], then one rounding
    |dLSE| <= ds + (L + 1) 2^-23 + 2^-19 + 2^-22 |LSE|
"""
import math

import pytest
import torch

from ops_check import DEV, DTYPES, ROUND, SENTINEL, check, lists, rounding, row_mask
from oracle import ops_oracle

# F, N, frames, H, Hkv, d, L
SHAPES = [
    (4, 64, (0, 3), 2, 2, 64, 77),
    (3, 200, (0, 2), 3, 3, 128, 512),          # query tiles across frames, whole key tiles
    (1, 1, (0,), 1, 1, 64, 1),                 # one token, one state
    (5, 1, (0, 1, 4), 12, 12, 128, 1000),      # single tokens
    (6, 1, (0, 2, 3, 5), 8, 2, 128, 300),      # single tokens, four heads on a key head
    (2, 1, (0, 1), 24, 1, 64, 129),
    (7, 5, (1, 2, 6), 6, 2, 64, 40),           # frames of five tokens, three heads per key head
    (3, 100, (0, 1, 2), 2, 1, 128, 260),       # two heads x 100 tokens: more than a tile
    (4, 30, (0, 1, 3), 4, 1, 128, 500),        # four heads x 30 tokens: packed, one frame per tile
    (5, 130, (0, 4), 20, 20, 64, 128),         # many items, one key tile
    (9, 333, (0, 1, 3, 4, 8), 10, 5, 128, 257),  # more items than SMs
    (3, 9, (0, 2), 40, 1, 64, 64),             # forty heads on a key head, frames off 8 rows
    (2, 6, (0, 1), 32, 1, 64, 200),            # rows gathered one by one
    (2, 17, (1,), 2, 2, 128, 4000),            # long states, few rows: dealt to a cluster
    (3, 100, (0, 1, 2), 160, 160, 64, 200),    # several items per SM, every second without a tile B
    (3, 16, (), 2, 2, 64, 64),                 # nothing active
]


def _ranges(kind, F, L):
    if kind == "lengths":   # packed, ragged, the second one empty
        w = [0 if f == 1 else 1 + f % 3 for f in range(F)]
        edge = [L * sum(w[:f]) // max(1, sum(w)) for f in range(F + 1)]
        return [(edge[f], edge[f + 1]) for f in range(F)]
    if kind == "windows":   # overlapping, off the tiles, past both ends
        return [(f * L // F - 3, f * L // F + L // 2 + 1) for f in range(F)]
    return None


def _mask(kind, L, g):
    if kind is None:
        return None
    if kind == "none_left":
        return torch.zeros(L, dtype=torch.uint8)
    if kind == "tail":
        return (torch.arange(L) < max(1, 2 * L // 3)).to(torch.uint8)
    return (torch.rand(L, generator=g) < 0.5).to(torch.uint8) * 255


def _run(rf, Q, K, V, F, N, frames, scale, ranges, keep, **kw):
    act, cnt = lists(frames, F, N)
    H, T = Q.shape[1], F * N
    O = torch.full((T, H, Q.shape[2]), SENTINEL, dtype=Q.dtype, device=DEV)
    lse = torch.full((H, T), SENTINEL, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = None if ranges is None else torch.tensor(ranges, dtype=torch.int32, device=DEV)
    m = None if keep is None else keep.to(DEV)
    rf.rf_cross_attn(O, lse, Q, K, V, F, N, scale, kv_range=r, key_mask=m, active=act, counts=cnt,
                     status=st, **kw)
    torch.cuda.synchronize()
    assert st.item() == 0
    return O, lse


def _compare(O, lse, Q, K, V, F, N, frames, scale, ranges, keep, label):
    want, wlse = ops_oracle.cross_attention(Q, K, V, frames, N, scale, ranges, keep)
    rows = row_mask(frames, F, N)
    L, d, dt = K.shape[0], Q.shape[2], Q.dtype
    # P|V|: the same attention over |v|
    pv, _ = ops_oracle.cross_attention(Q, K, V.abs(), frames, N, scale, ranges, keep)
    q, k = Q.cpu().double().abs(), K.cpu().double().abs()
    big = torch.zeros(q.shape[:2], dtype=torch.float64)
    if L:
        for h in range(q.shape[1]):
            big[:, h] = (q[:, h] @ k[:, h // (q.shape[1] // k.shape[1])].T).amax(dim=1)
    ds = scale * big * ((d + 1) * 2.0 ** -23 + 2.0 ** -22)
    sums = (L + 1) * 2.0 ** -23
    b = (ROUND[dt] + 2 * ds + 2.0 ** -19 + 2 * sums)[..., None] * pv
    if dt == torch.float16 and L:
        b = b + 2.0 ** -25 * V.cpu().double().abs().sum(dim=0).amax()
    b = b * 1.05 + rounding(want, dt) + 1e-300
    check(O, want, b, rows, label)
    lw, lg = wlse.T[rows], lse.cpu().double().T[rows]
    assert (lse.cpu().T[~rows] == SENTINEL).all()
    none = lw == -math.inf
    assert torch.equal(lg == -math.inf, none)
    lb = (ds.expand(wlse.T.shape)[rows] + sums + 2.0 ** -19 + 2.0 ** -22 * lw.abs()) * 1.05
    assert (((lg - lw).abs() <= lb) | none).all(), label


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("keys", [(None, None), ("lengths", None), ("windows", "holes"),
                                  (None, "tail"), (None, "none_left"), ("lengths", "holes")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_cross_matches_oracle(cuda_lib, shape, keys, dtype):
    rf = cuda_lib
    F, N, frames, H, Hkv, d, L = SHAPES[shape]
    g = torch.Generator().manual_seed(31 * shape + d)
    dt = DTYPES[dtype]
    Q = torch.randn(F * N, H + 1, d, generator=g).to(dt).to(DEV)[:, :H]
    KV = torch.randn(L, 2, Hkv, d, generator=g).to(dt)
    ranges, keep = _ranges(keys[0], F, L), _mask(keys[1], L, g)
    scale = d ** -0.5
    if keep is not None:  # masked states hold anything
        bad = KV.clone()
        bad[keep == 0] = math.nan
        if L > 2:
            bad[1::2][keep[1::2] == 0] = math.inf
        dev = bad.to(DEV)
    else:
        dev = KV.to(DEV)
    O, lse = _run(rf, Q, dev[:, 0], dev[:, 1], F, N, frames, scale, ranges, keep)
    if keep is not None:  # 64-bit statement over the kept ones: any finite value in their place
        KV[keep == 0] = 0
    _compare(O, lse, Q, KV[:, 0], KV[:, 1], F, N, frames, scale, ranges, keep,
             f"cross {SHAPES[shape]} {keys} {dtype}")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_cross_states_of_other_ranges_do_not_matter(cuda_lib, d):
    """NaN in every state outside the active frames' ranges, up to the range's own last tile."""
    rf = cuda_lib
    F, N, H, L = 3, 40, 2, 300
    g = torch.Generator().manual_seed(4)
    Q = torch.randn(F * N, H, d, generator=g).to(torch.bfloat16).to(DEV)
    K, V = (torch.randn(L, H, d, generator=g).to(torch.bfloat16) for _ in range(2))
    ranges, frames = [(5, 150), (150, 151), (160, 297)], (0, 2)
    good = _run(rf, Q, K.to(DEV), V.to(DEV), F, N, frames, d ** -0.5, ranges, None)
    K2, V2 = K.clone(), V.clone()
    for x in (K2, V2):
        x[:5], x[150:160], x[297:] = math.nan, math.inf, math.nan
    bad = _run(rf, Q, K2.to(DEV), V2.to(DEV), F, N, frames, d ** -0.5, ranges, None)
    assert torch.equal(good[0], bad[0]) and torch.equal(good[1], bad[1])


@pytest.mark.gpu
@pytest.mark.parametrize("L", [0, 1, 127, 128, 129, 512])
def test_cross_without_a_list_and_lengths(cuda_lib, L):
    """Every frame (no list); no state at all gives zeros and -inf."""
    rf = cuda_lib
    F, N, H, d = 2, 150, 3, 64
    g = torch.Generator().manual_seed(L)
    Q = torch.randn(F * N, H, d, generator=g).to(torch.bfloat16).to(DEV)
    K, V = (torch.randn(L, H, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    O = torch.full((F * N, H, d), SENTINEL, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((H, F * N), SENTINEL, device=DEV)
    rf.rf_cross_attn(O, lse, Q, K, V, F, N, d ** -0.5)
    torch.cuda.synchronize()
    _compare(O, lse, Q, K, V, F, N, (0, 1), d ** -0.5, None, None, f"cross L {L}")


@pytest.mark.gpu
def test_cross_extreme_scores(cuda_lib):
    """A maximum that moves from tile to tile, up and down, equal scores, and near-argmax rows."""
    rf = cuda_lib
    F, N, H, d, L = 1, 140, 2, 128, 700
    g = torch.Generator().manual_seed(9)
    Q = torch.randn(N, H, d, generator=g)
    K, V = (torch.randn(L, H, d, generator=g) for _ in range(2))
    ramp = torch.linspace(0.1, 6.0, L)[:, None, None]
    for q, k in ((Q, K * ramp), (Q, K * ramp.flip(0)), (Q * 0, K), (Q * 12, K)):
        q, k, v = (x.to(torch.bfloat16).to(DEV) for x in (q, k, V))
        O, lse = _run(rf, q, k, v, F, N, (0,), d ** -0.5, None, None)
        _compare(O, lse, q, k, v, F, N, (0,), d ** -0.5, None, None, "cross extreme")


@pytest.mark.gpu
def test_cross_equals_the_step_cores_attention(cuda_lib):
    """Over the keys of the sequence itself rf_cross_attn computes what rf_attn does: both round
    P and O once, so they differ by at most twice the bound's dominant terms."""
    rf = cuda_lib
    F, N, H, d = 3, 200, 2, 128
    g = torch.Generator().manual_seed(11)
    Q, K, V = (torch.randn(F * N, H, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(3))
    frames = (0, 2)
    act, cnt = lists(frames, F, N)
    A = torch.zeros_like(Q)
    la = torch.zeros(H, F * N, device=DEV)
    rf.rf_attn(A, la, Q, K, V, Q.stride(0), A.stride(0), F, N, H, d, act, cnt, d ** -0.5)
    O, lse = _run(rf, Q, K, V, F, N, frames, d ** -0.5, None, None)
    rows = row_mask(frames, F, N).to(DEV)
    assert (O[rows].float() - A[rows].float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -9)
    assert (lse[:, rows] - la[:, rows]).abs().max() <= 1e-4


def test_cross_refuses_bad_arguments():
    import paper_2606_06309_gb300 as rf
    lib = rf.load()
    P = 256
    ok = [P, None, P, P, P, 512, 512, 256, 256, 0, 4, 64, 4, 2, 128, 77, P, P, P, P, 0.1, None, None]
    cases = [(0, None, 1), (2, None, 1), (3, None, 1), (4, None, 1), (5, 511, 1), (6, 516, 3),
             (7, 255, 1), (8, 260, 3), (9, 2, 2), (10, 0, 1), (11, 0, 1), (12, 3, 1), (13, 0, 1),
             (14, 96, 2), (15, -1, 1), (16, P + 4, 3), (18, None, 1), (19, None, 1), (20, 0.0, 1),
             (20, math.nan, 1), (20, math.inf, 1), (0, P + 2, 3), (3, P + 8, 3), (1, P + 2, 3),
             (11, 1 << 30, 1), (15, 0x7FFFFFFF, 1)]
    for i, v, want in cases:
        args = list(ok)
        args[i] = v
        assert lib.rf_cross_attn(*args) == want, (i, v)
    z, h = torch.zeros, torch.bfloat16
    Q, K = z(6, 4, 64, dtype=h), z(9, 2, 64, dtype=h)
    O = torch.zeros_like(Q)
    for o, k, v, kw in ((O, K, K[:8], {}), (O.float(), K, K, {}), (O[:5], K, K, {}),
                        (O, K, K, dict(kv_range=z(2, 2))), (O, K, K, dict(key_mask=z(9))),
                        (O, K, K, dict(key_mask=z(8, dtype=torch.uint8))),
                        (O, K.transpose(1, 2).contiguous().transpose(1, 2), K, {})):
        with pytest.raises(ValueError):
            rf.rf_cross_attn(o, None, Q, k, v, 2, 3, 0.1, stream=0, **kw)
    with pytest.raises(ValueError):
        rf.rf_cross_attn(O, z(4, 5), Q, K, K, 2, 3, 0.1, stream=0)
