"""A process' first calls of the operators, made by several threads at once, each on a stream of its own:
the bits that one thread gets afterwards."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import math, threading
import torch
import paper_2606_06309_gb300 as rf

H, d, L, h, dev = 4, 64, 200, torch.bfloat16, "cuda"
D = H * d
g = torch.Generator().manual_seed(1)
def rnd(*shape): return torch.randn(shape, generator=g).to(h).to(dev)
W, Wide, K, V = rnd(D, D) / 16, rnd(5120, D) / 16, rnd(L, H, d), rnd(L, H, d)
X = [rnd(600 + i, D) for i in range(8)]
tables = [torch.from_numpy(rf.rf_rope_table(range(n), 32, 1e4)).to(dev) for n in (1, 700)]
status = torch.zeros(8, 1, dtype=torch.int32, device=dev)

def work(i, stream):
    x, T, out = X[i], X[i].shape[0], []
    with torch.cuda.stream(stream):
        y, w = torch.empty_like(x), torch.empty(T, 5120, dtype=h, device=dev)
        o = torch.empty(T, H, d, dtype=h, device=dev)
        lo = torch.empty(100, D, dtype=h, device=dev)
        w_table = tables[1][:T]
        for _ in range(5):
            rf.rf_linear(y, x, W, 1, T, act="silu", status=status[i])
            q = y.view(T, H, d)
            rf.rf_rope(q, q, None, None, 1, 1, T, (32, 0, 32), (tables[0], None, w_table))
            rf.rf_cross_attn(o, None, q, K, V, 1, T, 0.125, status=status[i])
            rf.rf_linear(w, o.view(T, D), Wide, 1, T, status=status[i])
            rf.rf_linear(lo, x[:100], W, 1, 100, status=status[i])
        return y, o, w, lo

torch.cuda.synchronize()
streams = [torch.cuda.Stream() for _ in X]
got, ready = [None] * 8, threading.Barrier(8)
def thread(i):
    torch.cuda.set_device(0)
    ready.wait()
    got[i] = work(i, streams[i])
threads = [threading.Thread(target=thread, args=(i,)) for i in range(8)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert not status.any(), status
for i in range(8):
    want = work(i, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert got[i] is not None and all(torch.equal(a, b) for a, b in zip(got[i], want)), i
assert not status.any()
print("same")
"""


@pytest.mark.gpu
def test_first_calls_of_several_threads(cuda_lib):
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.strip() == "same"
