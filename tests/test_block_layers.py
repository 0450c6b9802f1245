"""Several ActiveBlocks over one StepCore, compacted once per step, as a model's layers.

Each block has its own cache.  Against the 64-bit statement of each block, fed with what the block before
it stored (bound as in test_block.py), and, bit for bit, against a step core per block.
"""
import math

import pytest
import torch

import oracle
from ops_check import DEV
from test_block import PlainBlock

H16 = torch.bfloat16
F, GH, GW, H, D_HEAD, HKV, DE, DF, L, S = 4, 6, 7, 4, 64, 2, 96, 512, 40, 4
N, D, DIMS = GH * GW, H * D_HEAD, (24, 20, 20)
IS_KEY, STRIDE = [1, 0, 0, 1], [2] * S


def _norm(h):
    h = h.double()
    return (h - h.mean(-1, keepdim=True)) / h.std(-1, unbiased=False, keepdim=True)


def _weights(g):
    from paper_2606_06309_gb300.block import BlockWeights

    def lin(o, i):
        return ((torch.randn(o, i, generator=g) / math.sqrt(i)).to(H16).to(DEV),
                (0.1 * torch.randn(o, generator=g)).to(H16).to(DEV))

    return BlockWeights(lin(3 * D, D), lin(D, D), lin(D, D), lin(2 * HKV * D_HEAD, DE), lin(D, D),
                        lin(DF, D), lin(D, DF))


def _core(kv_cache=True):
    from paper_2606_06309_gb300.stepcore import StepCore, upload_plan
    return StepCore(F, N, N * 16, H, D_HEAD, upload_plan(F, S, IS_KEY, STRIDE, 0, DEV), DEV,
                    kv_cache=kv_cache)


def _case(n):
    g = torch.Generator().manual_seed(23)
    weights = [_weights(g) for _ in range(n)]
    kv = [[torch.randn(F * N, H, D_HEAD, generator=g).to(H16) for _ in range(2)] for _ in range(n)]
    enc = torch.randn(L, DE, generator=g).to(H16)
    gates = [torch.randn(F, D, generator=g), torch.randn(D, generator=g)]
    return weights, kv, enc, gates, torch.randn(F * N, D, generator=g).to(H16)


def _norms():
    return [lambda h: _norm(h).to(H16)] * 3


@pytest.mark.gpu
@pytest.mark.parametrize("core_cache", [False, True])
def test_layers_share_a_core(cuda_lib, core_cache):
    from paper_2606_06309_gb300.block import ActiveBlock
    weights, kv, enc, gates, x0 = _case(3)
    mask = (torch.arange(L) < 33).to(torch.uint8)
    dev_gates = [t.to(DEV) for t in gates]
    scale = D_HEAD ** -0.5
    core = _core(core_cache)
    # with the core's cache: one of the blocks may have that one
    blocks = [ActiveBlock(core, GH, GW, w, DIMS, HKV, own_cache=i > 0 or not core_cache)
              for i, w in enumerate(weights)]
    plain = [PlainBlock(w, F, GH, GW, H, D_HEAD, DIMS, HKV, *c) for w, c in zip(weights, kv)]
    for b, (K0, V0) in zip(blocks, kv):
        b.set_kv_cache(K0.to(DEV), V0.to(DEV))
        b.encode(enc.to(DEV), mask.to(DEV))
    host = oracle.schedule(F, S, IS_KEY, STRIDE, 0)
    x = x0.to(DEV)
    for s in range(S):  # every frame, the keyframes, every frame, the keyframes
        core.compact(s)
        for i, b in enumerate(blocks):
            before = x.clone()
            b.run(s, x, scale, norms=_norms(), gates=dev_gates)
            torch.cuda.synchronize()
            assert core.status.item() == 0
            ref, rows = plain[i].run(s, before.cpu().double(), host, scale, _norm, gates, enc, mask)
            got = x.cpu().double()
            err = (got[rows] - ref[rows]).norm() / ref[rows].norm()
            print(f"step {s}, block {i}: relative error {err:.4f}")
            assert err <= 10 * 2.0 ** -9
            assert torch.equal(x[~rows.to(DEV)], before[~rows.to(DEV)])


def _trajectory(blocks, cores, kv, enc, x0):
    for b, (K0, V0) in zip(blocks, kv):
        b.set_kv_cache(K0.to(DEV), V0.to(DEV))
        b.encode(enc.to(DEV))
    x = x0.to(DEV)
    for s in range(S):
        for c in cores:
            c.compact(s)
        for b in blocks:
            b.run(s, x, D_HEAD ** -0.5, norms=_norms())
    torch.cuda.synchronize()
    return x


@pytest.mark.gpu
def test_one_core_or_one_per_block(cuda_lib):
    from paper_2606_06309_gb300.block import ActiveBlock
    weights, kv, enc, _, x0 = _case(3)
    one = _core(kv_cache=False)
    got = _trajectory([ActiveBlock(one, GH, GW, w, DIMS, HKV, own_cache=True) for w in weights], [one],
                      kv, enc, x0)
    cores = [_core() for _ in weights]
    want = _trajectory([ActiveBlock(c, GH, GW, w, DIMS, HKV) for c, w in zip(cores, weights)], cores,
                       kv, enc, x0)
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_one_cache_for_two_layers_is_refused(cuda_lib):
    """Where it would give wrong keys: not for a block in another's place, and not where the caller changes
    the caches between the blocks."""
    from paper_2606_06309_gb300.block import ActiveBlock
    weights, kv, enc, _, x0 = _case(2)
    core = _core()
    a, b = (ActiveBlock(core, GH, GW, w, DIMS, HKV) for w in weights)
    x, scale = x0.to(DEV), D_HEAD ** -0.5
    core.compact(0)
    a.run(0, x, scale)
    b.run(0, x, scale)
    core.compact(1)
    before = x.clone()
    with pytest.raises(ValueError, match="own_cache"):
        a.run(1, x, scale)
    torch.cuda.synchronize()
    assert torch.equal(x, before)
    b.run(1, x, scale)      # the last one's keys are there
    core.compact(2)
    a.run(2, x, scale)      # every frame is active: no key is wanted back
    core.compact(3)
    b.run(3, x, scale)      # one block in the other's place
    # the caller's own caches, changed between the blocks
    caches = [[t.clone() for t in (core.Kc, core.Vc)] for _ in range(2)]
    x = x0.to(DEV)
    for s in range(S):
        core.compact(s)
        for block, cache in zip((a, b), caches):
            core.Kc, core.Vc = cache
            block.run(s, x, scale)
    torch.cuda.synchronize()
    assert core.status.item() == 0
