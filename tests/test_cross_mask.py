"""rf_cross_attn under masks of many forms: what is not seen is not visited, or not brought at all.

The bounds are those of test_cross_attn.py.
"""
import pytest
import torch

from ops_check import DEV, DTYPES
from test_cross_attn import _compare, _ranges, _run

# F, N, frames, H, Hkv, d, L
SHAPES = [
    (3, 200, (0, 2), 3, 3, 128, 1500),
    (5, 1, (0, 1, 4), 12, 12, 128, 1000),         # single tokens
    (6, 1, (0, 2, 3, 5), 8, 2, 64, 3001),         # four heads on a key head
    (4, 30, (0, 1, 3), 4, 1, 128, 2050),          # packed rows
    (2, 17, (1,), 2, 2, 128, 9000),               # dealt to a cluster
    (1, 3, (0,), 1, 1, 64, 20011),
    (9, 333, (0, 1, 3, 4, 8), 20, 10, 64, 1111),  # several items per SM
    (3, 100, (0, 1, 2), 160, 160, 128, 700),      # every second item without a tile B
    (4, 300, (0, 1, 2, 3), 160, 160, 64, 500),    # five items per SM of one tile of keys or a few
    (4, 300, (0, 1, 2, 3), 100, 100, 128, 500),
]


def _keep(kind, L, g):
    keep = torch.zeros(L, dtype=torch.uint8)
    if kind == "one":
        keep[(5 * L) // 7] = 1
    elif kind == "ends":
        keep[0] = keep[L - 1] = 1
    elif kind == "tiles":  # 256 of them: two whole tiles
        keep[torch.randperm(L, generator=g)[:256]] = 1
    elif kind == "middle":
        keep[L // 3 + 1:L - L // 4] = 1
    elif kind == "first_quarter":  # all that is seen falls to the first CTAs of a cluster
        keep[torch.randperm(L // 4, generator=g)[:L // 12]] = 3
    else:
        keep[torch.rand(L, generator=g) < kind] = 128
    return keep


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["one", "ends", "tiles", "middle", "first_quarter", 0.02, 0.2, 0.55,
                                  0.7, 0.95])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_cross_masks_match_oracle(cuda_lib, shape, kind):
    F, N, frames, H, Hkv, d, L = SHAPES[shape]
    dt = DTYPES["bf16" if shape % 2 else "fp16"]
    g = torch.Generator().manual_seed(1000 + shape)
    Q = torch.randn(F * N, H, d, generator=g).to(dt).to(DEV)
    K, V = (torch.randn(L, Hkv, d, generator=g).to(dt).to(DEV) for _ in range(2))
    keep = _keep(kind, L, g)
    # what is not seen must not matter, whatever it holds
    K[keep.to(DEV) == 0] = float("nan")
    V[keep.to(DEV) == 0] = float("inf")
    O, lse = _run(cuda_lib, Q, K, V, F, N, frames, d ** -0.5, None, keep)
    K[keep.to(DEV) == 0] = 0
    V[keep.to(DEV) == 0] = 0
    _compare(O, lse, Q, K, V, F, N, frames, d ** -0.5, None, keep, f"{SHAPES[shape]} {kind}")


@pytest.mark.gpu
@pytest.mark.parametrize("ranges", ["lengths", "windows"])
@pytest.mark.parametrize("kind", ["middle", "ends", 0.2])
def test_cross_masks_within_ranges(cuda_lib, kind, ranges):
    F, N, frames, H, Hkv, d, L = 16, 130, tuple(range(0, 16, 2)), 24, 24, 64, 2600
    g = torch.Generator().manual_seed(7)
    Q = torch.randn(F * N, H, d, generator=g).to(torch.bfloat16).to(DEV)
    K, V = (torch.randn(L, Hkv, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    keep, r = _keep(kind, L, g), _ranges(ranges, F, L)
    O, lse = _run(cuda_lib, Q, K, V, F, N, frames, d ** -0.5, r, keep)
    _compare(O, lse, Q, K, V, F, N, frames, d ** -0.5, r, keep, f"{ranges} {kind}")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["middle", 0.2, 0.9])
def test_cross_mask_off_word_boundaries_strides_streams_and_graphs(cuda_lib, kind):
    """The mask one byte off a word, keys and values in one buffer, on another stream, captured."""
    N, H, d, L = 150, 4, 128, 1003
    g = torch.Generator().manual_seed(9)
    Q = torch.randn(N, H, d, generator=g).to(torch.bfloat16).to(DEV)
    KV = torch.randn(L, 2, H, d, generator=g).to(torch.bfloat16).to(DEV)
    keep = _keep(kind, L, g)
    buf = torch.full((L + 9,), 7, dtype=torch.uint8, device=DEV)  # what lies beside it is not read
    want = torch.zeros_like(Q)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    buf[4:4 + L] = keep.to(DEV)
    lse = torch.zeros(H, N, device=DEV)
    cuda_lib.rf_cross_attn(want, lse, Q, KV[:, 0], KV[:, 1], 1, N, d ** -0.5,
                           key_mask=buf[4:4 + L], status=status)
    _compare(want, lse, Q, KV[:, 0], KV[:, 1], 1, N, (0,), d ** -0.5, None, keep, str(kind))
    buf.fill_(7)
    buf[5:5 + L] = keep.to(DEV)
    got = torch.zeros_like(Q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cuda_lib.rf_cross_attn(got, None, Q, KV[:, 0], KV[:, 1], 1, N, d ** -0.5,
                               key_mask=buf[5:5 + L], status=status, stream=side)
    graph.replay()
    torch.cuda.synchronize()
    assert status.item() == 0
    assert torch.equal(got, want)
    buf[5:5 + L] = 0  # another mask in the same place: nothing seen
    graph.replay()
    torch.cuda.synchronize()
    assert (got == 0).all()
