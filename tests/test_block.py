"""ActiveBlock: the step core's attention and the operators around it, two steps of a small video.

Against the same block from the 64-bit statements of its parts, with every stored tensor rounded to
bf16 where the block stores one.  A value on the edge between two bf16 values can be rounded either
way, and carries on: every stored tensor is off by at most the rounding error it has itself (2^-9 of
its norm, as the error of a rounding is evenly spread over +-2^-9 relative).  Ten tensors are stored
one after the other on the longest path, so the results' norms differ by less than 10 * 2^-9 = 2%.
"""
import math

import pytest
import torch

import oracle
from oracle import ops_oracle
from ops_check import DEV, row_mask

H16 = torch.bfloat16


def r16(x):
    return x.to(H16).double()


class PlainBlock:
    def __init__(self, w, F, gh, gw, H, d, dims, Hkv, K0, V0):
        self.w, self.F, self.gh, self.gw, self.N = w, F, gh, gw, gh * gw
        self.H, self.d, self.dims, self.Hkv = H, d, dims, Hkv
        D = H * d
        self.cache = [torch.stack([r16(x).reshape(F, self.N, D)] * 2).numpy() for x in (K0, V0)]

    def lin(self, x, name, frames, **kw):
        W, b = getattr(self.w, name)
        y, _ = ops_oracle.linear(x, W, frames, self.N, bias=b, **kw)
        return r16(y)

    def run(self, s, x, plan, scale, norm, gates, enc, mask):
        F, N, H, d, D = self.F, self.N, self.H, self.d, self.H * self.d
        frames = [f for f in range(F) if plan["mask"][s][f]]
        rows = row_mask(frames, F, N)
        x = x.clone()
        qkv = self.lin(r16(norm(x)), "qkv", frames).view(F * N, 3, H, d)
        pos = [list(range(n)) for n in (F, self.gh, self.gw)]
        q, k = (r16(ops_oracle.rope(qkv[:, i], frames, pos, self.dims)) for i in (0, 1))
        kv = []
        for j, t in enumerate((k, qkv[:, 2])):
            t = torch.nan_to_num(t).reshape(F, N, D).numpy()
            out, self.cache[j] = oracle.project_kv_cache(t, self.cache[j], plan["cur_slot"][s],
                                                         plan["alpha"][s], plan["mask"][s])
            kv.append(r16(torch.from_numpy(out)).reshape(F * N, H, d))
        o, _ = ops_oracle.cross_attention(q, kv[0], kv[1], frames, N, scale)
        y = self.lin(r16(o).reshape(F * N, D), "out", frames, gate=gates[0], residual=x)
        x[rows] = y[rows]
        qc = self.lin(r16(norm(x)), "cross_q", frames).view(F * N, H, d)
        L = enc.shape[0]
        W, b = self.w.cross_kv
        e = r16(ops_oracle.linear(enc, W, [0], L, bias=b)[0]).view(L, 2, self.Hkv, d)
        o, _ = ops_oracle.cross_attention(qc, e[:, 0], e[:, 1], frames, N, scale, None, mask)
        y = self.lin(r16(o).reshape(F * N, D), "cross_out", frames, residual=x)
        x[rows] = y[rows]
        u = self.lin(r16(norm(x)), "up", frames, act="gelu_tanh")
        y = self.lin(u, "down", frames, gate=gates[1], residual=x)
        x[rows] = y[rows]
        return x, rows


@pytest.mark.gpu
def test_block_two_steps(cuda_lib):
    from paper_2606_06309_gb300.block import ActiveBlock, BlockWeights
    from paper_2606_06309_gb300.stepcore import StepCore, upload_plan
    F, gh, gw, H, d, Hkv, De, Df, L, S = 4, 6, 7, 4, 64, 2, 96, 512, 40, 4
    N, D, dims = gh * gw, H * d, (24, 20, 20)
    g = torch.Generator().manual_seed(17)

    def lin(o, i):
        return ((torch.randn(o, i, generator=g) / math.sqrt(i)).to(H16).to(DEV),
                (0.1 * torch.randn(o, generator=g)).to(H16).to(DEV))

    w = BlockWeights(lin(3 * D, D), lin(D, D), lin(D, D), lin(2 * Hkv * d, De), lin(D, D), lin(Df, D),
                     lin(D, Df))
    is_key, stride = [1, 0, 0, 1], [2] * S
    plan = upload_plan(F, S, is_key, stride, 0, DEV)
    core = StepCore(F, N, N * 16, H, d, plan, DEV)
    K0, V0 = (torch.randn(F * N, H, d, generator=g).to(H16) for _ in range(2))
    core.set_kv_cache(K0.to(DEV), V0.to(DEV))
    block = ActiveBlock(core, gh, gw, w, dims, Hkv)
    enc = torch.randn(L, De, generator=g).to(H16)
    mask = (torch.arange(L) < 33).to(torch.uint8)
    block.encode(enc.to(DEV), mask.to(DEV))
    gates = [torch.randn(F, D, generator=g), torch.randn(D, generator=g)]
    x0 = torch.randn(F * N, D, generator=g).to(H16)

    def norm(h):
        h = h.double()
        return (h - h.mean(-1, keepdim=True)) / h.std(-1, unbiased=False, keepdim=True)

    plain = PlainBlock(w, F, gh, gw, H, d, dims, Hkv, K0, V0)
    host = oracle.schedule(F, S, is_key, stride, 0)
    x, ref = x0.to(DEV), x0.double()
    scale = d ** -0.5
    for s in (0, 1):  # every frame, then the keyframes over projected keys and values
        before = x.clone()
        core.compact(s)
        block.run(s, x, scale, norms=[lambda h: norm(h).to(H16)] * 3, gates=[t.to(DEV) for t in gates])
        torch.cuda.synchronize()
        assert core.status.item() == 0
        ref, rows = plain.run(s, ref, host, scale, norm, gates, enc, mask)
        got = x.cpu().double()
        err = (got[rows] - ref[rows]).norm() / ref[rows].norm()
        print(f"step {s}: {int(rows.sum())} rows, relative error {err:.4f}")
        assert err <= 10 * 2.0 ** -9
        assert torch.equal(x[~rows.to(DEV)], before[~rows.to(DEV)])
        ref = got.clone()  # the next step from the same hidden states


def test_block_checks_its_grid():
    from types import SimpleNamespace

    from paper_2606_06309_gb300.block import ActiveBlock
    with pytest.raises(ValueError):
        ActiveBlock(SimpleNamespace(N=64), 8, 9, None, (16, 0, 0), 1)
