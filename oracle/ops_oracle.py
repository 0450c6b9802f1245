"""Plain 64-bit statements of the operators around the attention: rotary positions over three axes,
attention to an encoder's states, and the linear layer with its epilogue.

Row by row and pair by pair from the definitions, on the CPU, with nothing shared with the library.
Inputs are tensors of any type; results are float64 tensors in which rows of frames that are not
active are left at NaN (nothing may be compared there).
"""
import math

import torch

__all__ = ["rope", "cross_attention", "linear"]


def _rows(frames, N):
    return torch.tensor([f * N + p for f in frames for p in range(N)], dtype=torch.long)


def rope(X, frames, pos, dims, base=10000.0, pairing="interleaved", inverse=False):
    """X [F*gh*gw, H, d]; pos: the positions of the three axes' (F, gh, gw) places."""
    F, gh, gw = (len(p) for p in pos)
    x = X.detach().cpu().double()
    out = torch.full(x.shape, math.nan, dtype=torch.float64)
    rows = _rows(frames, gh * gw)
    place = (rows // (gh * gw), rows // gw % gh, rows % gw)
    xr = x[rows]
    y = xr.clone()
    R, i = sum(dims), 0  # i: pair over all axes
    for axis, dim in enumerate(dims):
        at = torch.tensor([float(p) for p in pos[axis]], dtype=torch.float64)[place[axis]]
        for j in range(dim // 2):
            a = at * base ** (-2.0 * j / dim)
            c, s = a.cos()[:, None], (-a if inverse else a).sin()[:, None]
            i0, i1 = (2 * i, 2 * i + 1) if pairing == "interleaved" else (i, i + R // 2)
            y[:, :, i0] = xr[:, :, i0] * c - xr[:, :, i1] * s
            y[:, :, i1] = xr[:, :, i0] * s + xr[:, :, i1] * c
            i += 1
    out[rows] = y
    return out


def cross_attention(Q, K, V, frames, N, scale, ranges=None, keep=None):
    """Q [F*N, H, d] over K, V [L, Hkv, d] -> O [F*N, H, d], lse [H, F*N].

    ranges: (begin, end) of every frame's keys, or None: all; keep [L]: nonzero = may be seen."""
    q, k, v = (x.detach().cpu().double() for x in (Q, K, V))
    H, Hkv, L = q.shape[1], k.shape[1], k.shape[0]
    O = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full((H, q.shape[0]), math.nan, dtype=torch.float64)
    for f in frames:
        b, e = (0, L) if ranges is None else ranges[f]
        keys = [j for j in range(max(b, 0), min(e, L)) if keep is None or int(keep[j]) != 0]
        rows = slice(f * N, f * N + N)
        for h in range(H):
            if not keys:
                O[rows, h] = 0.0
                lse[h, rows] = -math.inf
                continue
            s = scale * q[rows, h] @ k[keys, h // (H // Hkv)].T
            m = s.max(dim=1, keepdim=True).values
            p = (s - m).exp()
            l = p.sum(dim=1, keepdim=True)
            O[rows, h] = p @ v[keys, h // (H // Hkv)] / l
            lse[h, rows] = (m + l.log())[:, 0]
    return O, lse


def activation(z, act):
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def linear(X, W, frames, N, bias=None, act=None, gate=None, residual=None):
    """-> (Y, S): the result and, of every element, sum_k |x w| + |bias|."""
    x, w = X.detach().cpu().double(), W.detach().cpu().double()
    Y = torch.full((x.shape[0], w.shape[0]), math.nan, dtype=torch.float64)
    S = Y.clone()
    rows = _rows(frames, N)
    z, s = x[rows] @ w.T, x[rows].abs() @ w.abs().T
    if bias is not None:
        b = bias.detach().cpu().double()
        z, s = z + b, s + b.abs()
    z = activation(z, act)
    if gate is not None:
        g = gate.detach().cpu().double()
        z = z * (g if g.dim() == 1 else g[rows // N])
    if residual is not None:
        z = z + residual.detach().cpu().double()[rows]
    Y[rows], S[rows] = z, s
    return Y, S
