"""rf_linear's activations by themselves, over their tails.

One column of K, inputs of 8 or 11 bits and weights that are powers of two: the sum is the product,
exactly, and the result is the activation of a known number, in 32 bits.  Relative bounds, derived:
  gelu       z^2 / 2 in the exponent is off by less than 2.5 2^-24 of itself, which is within (z^2 + |z|) 2^-23
             of the value; the rest is an exponential (2^-22), a quotient (2^-22) and some twelve
             products and sums (2^-24 each) or a function evaluated as well as that: 2^-20 in all
  silu       with |s| the exponent (log2 e |s| is rounded to 32 bits, which costs |s| 2^-23 of e^s), s = z: an
             exponential in two factors of 2^-22 each, a quotient (2^-22) and three products (2^-24
             each): |z| 2^-23 + 2^-20
  gelu_tanh  s = 2 sqrt(2/pi) (z + 0.044715 z^3) itself from four operations and three constants, each
             off by at most 2^-24, so |s| (2^-23 + 7 2^-24) + 2^-20 <= |s| 2^-21 + 2^-20
and 2^-126 absolute: numbers below the smallest normal one may be lost.
"""
import math

import pytest
import torch

from ops_check import DEV, DTYPES


def _act(z, act):
    """In 64 bits, without cancellation in the tails; and the relative bound."""
    if act == "silu":
        return z * torch.sigmoid(z), z.abs() * 2.0 ** -23 + 2.0 ** -20
    if act == "gelu_tanh":  # (1 + tanh u) / 2 is the sigmoid of 2 u
        s = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        return z * torch.sigmoid(s), s.abs() * 2.0 ** -21 + 2.0 ** -20
    return (0.5 * z * torch.erfc(-z / math.sqrt(2.0)),
            (z * z + z.abs()) * 2.0 ** -23 + 2.0 ** -20)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,d_out", [(1, 777), (200, 128), (600, 5120), (600, 5123)])
def test_activation(cuda_lib, rows, d_out, dtype, act):
    dt = DTYPES[dtype]
    top = 100.0 if act == "silu" else 12.0
    g = torch.Generator().manual_seed(rows)
    x = ((torch.rand(rows, 1, generator=g) * 2 - 1) * top).to(dt)
    w = (2.0 ** -torch.randint(0, 6, (d_out, 1), generator=g).float()).to(dt)
    w[::7] *= -1
    X, W = (torch.zeros(t.shape[0], 8, dtype=dt, device=DEV) for t in (x, w))
    X[:, :1], W[:, :1] = x.to(DEV), w.to(DEV)
    Y = torch.empty(rows, d_out, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    cuda_lib.rf_linear(Y, X[:, :1], W[:, :1], 1, rows, act=act, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    z = x.double() * w.double().T
    want, rel = _act(z, act)
    ratio = (Y.cpu().double() - want).abs() / (rel * want.abs() + 2.0 ** -126)
    i = int(ratio.argmax())
    print(f"{act} {dtype} {rows} x {d_out}: {ratio.max():.3f} of the bound, at z = {z.flatten()[i]:.4f}")
    assert ratio.max() <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activation_of_infinities(cuda_lib, act):
    """+inf stays, -inf times a weight of 0 within the activation is NaN as the formula has it, NaN stays; and
    the largest finite numbers give themselves or zero."""
    x = torch.tensor([[math.inf], [math.nan], [3e38], [-3e38]], dtype=torch.bfloat16)
    X = torch.zeros(4, 8, dtype=torch.bfloat16, device=DEV)
    W = torch.zeros(1, 8, dtype=torch.bfloat16, device=DEV)
    X[:, :1], W[:, :1] = x.to(DEV), 1.0
    Y = torch.empty(4, 1, device=DEV)
    cuda_lib.rf_linear(Y, X[:, :1], W[:, :1], 1, 4, act=act)
    y = Y.cpu()[:, 0]
    assert y[0] == math.inf and torch.isnan(y[1])
    assert y[2] == x[2, 0].float() and y[3] == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activation_of_tiny_numbers(cuda_lib, act):
    """Next to 0 each is z / 2, to 2^-20 of it, down to the smallest normal results."""
    e = torch.arange(-124, -20)
    z = torch.cat([(1 + 37 / 128) * 2.0 ** e, -(1 + 91 / 128) * 2.0 ** e])[:, None].to(torch.bfloat16)
    for rows in (z, z.repeat(3, 1)):  # both kernels
        n = rows.shape[0]
        d_out = 8 if n <= 256 else 5120
        X = torch.zeros(n, 8, dtype=torch.bfloat16, device=DEV)
        W = torch.zeros(d_out, 8, dtype=torch.bfloat16, device=DEV)
        X[:, :1], W[:, :1] = rows.to(DEV), 1.0
        Y = torch.empty(n, d_out, device=DEV)
        cuda_lib.rf_linear(Y, X[:, :1], W[:, :1], 1, n, act=act)
        y, x = Y.cpu().double(), rows.double()
        want, _ = _act(x, act)
        assert ((y - want).abs() <= 2.0 ** -20 * want.abs()).all()
