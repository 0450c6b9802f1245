"""Python binding of librf.so, the RhymeFlow asynchronous step core for GB300.

Argument marshalling only: each function takes torch tensors (or host numpy
arrays for the planner), passes their raw pointers and sizes to the C ABI
declared in ``include/rf.h`` and raises ``RFError`` on a non-OK status.  Every
step of the computation runs in the library's CUDA kernels; there is no CPU or
PyTorch fallback, and a missing library is an error.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

__all__ = ["load", "lib_path", "RFError", "rf_plan_build", "rf_schedule_compact",
           "rf_project", "rf_project_kv", "rf_attn", "rf_attn_block_masked",
           "rf_attn_workspace_bytes", "rf_attn_noalloc", "rf_step", "rf_step_core", "rf_frame_gram",
           "rf_keyframe_select", "rf_rope_table", "rf_rope",
           "rf_cross_attn", "rf_linear", "rf_selftest_bounded_wait", "rf_pipeline_create",
           "rf_pipeline_step", "rf_pipeline_sync", "rf_pipeline_bytes", "rf_pipeline_destroy",
           "rf_status_str", "rf_version", "EXPORTS"]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB: Optional[ctypes.CDLL] = None

# Every symbol include/rf.h declares.
EXPORTS = ("rf_status_str", "rf_version", "rf_last_error", "rf_plan_build",
           "rf_schedule_compact", "rf_project", "rf_project_kv", "rf_attn",
           "rf_attn_block_masked", "rf_attn_workspace_bytes",
           "rf_attn_noalloc", "rf_step", "rf_step_core", "rf_frame_gram", "rf_keyframe_select",
           "rf_rope_table", "rf_rope", "rf_cross_attn", "rf_linear",
           "rf_pipeline_create", "rf_pipeline_step", "rf_pipeline_sync", "rf_pipeline_bytes",
           "rf_pipeline_destroy", "rf_selftest_bounded_wait")

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
_SIG = {
    "rf_status_str": ([_i32], ctypes.c_char_p),
    "rf_version": ([], _i32),
    "rf_last_error": ([], ctypes.c_char_p),
    "rf_plan_build": ([_i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp], _i32),
    "rf_schedule_compact": ([_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp], _i32),
    "rf_project": ([_vp, _vp, _vp, _vp, _vp, _i32, _i64, _vp], _i32),
    "rf_project_kv": ([_vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                       _vp], _i32),
    "rf_attn": ([_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _f32,
                 _vp, _i64, _vp, _vp], _i32),
    "rf_attn_workspace_bytes": ([_i32], _i64),
    "rf_attn_block_masked": ([_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _vp,
                              _vp, _f32, _vp, _vp, _i64, _vp, _vp], _i32),
    "rf_selftest_bounded_wait": ([_vp, _i32, _vp], _i32),
    "rf_frame_gram": ([_vp, _i32, _i64, _i64, _vp, _vp], _i32),
    "rf_keyframe_select": ([_vp, _i32, _i32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                            ctypes.c_double, _vp, _vp], _i32),
    "rf_attn_noalloc": ([_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _vp, _vp,
                         _f32, _vp, _vp], _i32),
    "rf_step": ([_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i64, _vp], _i32),
    "rf_step_core": ([_vp] * 5 + [_i32, _i32, _i64, _i32, _i32] + [_vp] * 14 +
                     [_i64, _i64, _i64, _f32, _vp, _i64, _vp, _vp], _i32),
    "rf_rope_table": ([_vp, _i32, _i32, ctypes.c_double, _vp], _i32),
    "rf_rope": ([_vp, _vp, _i64, _i64, _i32, _vp, _vp, _i64, _i64] + [_i32] * 9 + [_vp, _vp, _vp] +
                [_i32, _i32, _vp, _vp, _vp], _i32),
    "rf_cross_attn": ([_vp] * 5 + [_i64] * 4 + [_i32] * 7 + [_vp] * 4 + [_f32, _vp, _vp], _i32),
    "rf_linear": ([_vp, _i64, _i32, _vp, _i64, _vp, _i64] + [_i32] * 5 +
                  [_vp, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp], _i32),
    "rf_pipeline_create": ([_i32, _i32, _i32, _i32, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                            _vp, _vp, _i32, _vp, _vp, _vp, ctypes.POINTER(_vp)], _i32),
    "rf_pipeline_step": ([_vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _f32], _i32),
    "rf_pipeline_sync": ([_vp, _vp], _i32),
    "rf_pipeline_bytes": ([_vp, _vp, _vp, _vp], _i32),
    "rf_pipeline_destroy": ([_vp], None),
}


class RFError(RuntimeError):
    def __init__(self, fn: str, status: int):
        detail = load().rf_last_error().decode()
        super().__init__(f"{fn} failed: {rf_status_str(status)} ({status}): {detail}")
        self.status = status


def lib_path() -> str:
    return os.path.join(_HERE, "librf.so")


def load() -> ctypes.CDLL:
    """Load librf.so (built by ``build.build()``); raises if it is missing."""
    global _LIB
    if _LIB is None:
        p = lib_path()
        if not os.path.exists(p):
            raise RuntimeError(f"{p} is missing: build it with __graft_entry__.build() "
                               "(there is no fallback implementation)")
        lib = ctypes.CDLL(p)
        for name, (args, res) in _SIG.items():
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = res
        _LIB = lib
    return _LIB


def _check(fn: str, st: int):
    if st != 0:
        raise RFError(fn, st)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    address = getattr(t, "data_ptr", None)  # most are tensors
    if address is not None:
        return address()
    if isinstance(t, int):
        return t
    return t.ctypes.data


_CURRENT = None  # () -> handle of the current stream


def _current_stream():
    """That function; torch is imported with the first call that needs it."""
    global _CURRENT
    import torch
    raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream",
                                                        "_cuda_getDevice"))
    if raw is None or device is None:
        _CURRENT = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    else:  # the same handle without a Stream object: 0.2 us of host time instead of 2.9
        _CURRENT = lambda: raw(device())  # noqa: E731
    return _CURRENT


def _stream(stream) -> Optional[int]:
    if stream is None:
        return (_CURRENT or _current_stream())()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def rf_status_str(status: int) -> str:
    return load().rf_status_str(int(status)).decode()


def rf_version() -> int:
    return load().rf_version()


def rf_plan_build(F: int, S: int, is_key, stride, T_w: int, sigma=None):
    """Host planner.  Returns numpy arrays mask, alpha, beta, dt, cur_slot ([S, F])."""
    is_key = np.ascontiguousarray(np.asarray(is_key, dtype=np.uint8))
    stride = np.ascontiguousarray(np.asarray(stride, dtype=np.int32))
    sig = None if sigma is None else np.ascontiguousarray(np.asarray(sigma, dtype=np.float64))
    mask = np.zeros((S, F), np.uint8)
    alpha = np.zeros((S, F), np.float32)
    beta = np.zeros((S, F), np.float32)
    dt = np.zeros((S, F), np.float32)
    slot = np.zeros((S, F), np.uint8)
    _check("rf_plan_build", load().rf_plan_build(
        F, S, _ptr(is_key), _ptr(stride), T_w, _ptr(sig), _ptr(mask), _ptr(alpha), _ptr(beta),
        _ptr(dt), _ptr(slot)))
    return {"mask": mask, "alpha": alpha, "beta": beta, "dt": dt, "cur_slot": slot}


def rf_schedule_compact(mask, F: int, N: int, active, skipped, token_idx, counts, stream=None):
    _check("rf_schedule_compact", load().rf_schedule_compact(
        _ptr(mask), F, N, _ptr(active), _ptr(skipped), _ptr(token_idx), _ptr(counts),
        _stream(stream)))


def rf_project(ctx, z2, cur_slot, alpha, beta, F: int, E: int, stream=None):
    _check("rf_project", load().rf_project(
        _ptr(ctx), _ptr(z2), _ptr(cur_slot), _ptr(alpha), _ptr(beta), F, E, _stream(stream)))


def rf_project_kv(K, V, kv_row_stride: int, Kc, Vc, cur_slot, alpha, beta, active, skipped,
                  counts, F: int, N: int, D: int, stream=None):
    _check("rf_project_kv", load().rf_project_kv(
        _ptr(K), _ptr(V), kv_row_stride, _ptr(Kc), _ptr(Vc), _ptr(cur_slot), _ptr(alpha),
        _ptr(beta), _ptr(active), _ptr(skipped), _ptr(counts), F, N, D, _stream(stream)))


def rf_attn(O, lse, Q, K, V, qkv_row_stride: int, o_row_stride: int, F: int, N: int, H: int,
            d: int, active, counts, softmax_scale: float, workspace=None, status=None,
            stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rf_attn", load().rf_attn(
        _ptr(O), _ptr(lse), _ptr(Q), _ptr(K), _ptr(V), qkv_row_stride, o_row_stride, F, N, H, d,
        _ptr(active), _ptr(counts), float(softmax_scale), _ptr(workspace), ws_bytes,
        _ptr(status), _stream(stream)))


def rf_attn_block_masked(O, lse, Q, K, V, qkv_row_stride: int, o_row_stride: int, F: int,
                         N: int, H: int, d: int, active, counts, softmax_scale: float, block_mask,
                         workspace=None, status=None, stream=None):
    """rf_attn under the frame mask x token block mask (block_mask uint8 [H, nb, nb])."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rf_attn_block_masked", load().rf_attn_block_masked(
        _ptr(O), _ptr(lse), _ptr(Q), _ptr(K), _ptr(V), qkv_row_stride, o_row_stride, F, N, H, d,
        _ptr(active), _ptr(counts), float(softmax_scale), _ptr(block_mask), _ptr(workspace),
        ws_bytes, _ptr(status), _stream(stream)))


def rf_attn_noalloc(O, lse, Q, K, V, qkv_row_stride: int, o_row_stride: int, F: int, N: int,
                    H: int, d: int, active, counts, softmax_scale: float, status=None,
                    stream=None):
    """rf_attn for callers that cannot allocate: the library's own static scratch."""
    _check("rf_attn_noalloc", load().rf_attn_noalloc(
        _ptr(O), _ptr(lse), _ptr(Q), _ptr(K), _ptr(V), qkv_row_stride, o_row_stride, F, N, H, d,
        _ptr(active), _ptr(counts), float(softmax_scale), _ptr(status), _stream(stream)))


def rf_selftest_bounded_wait(status, limit_us: int, stream=None):
    """Run the device bounded-wait self-test; *status receives RF_ERR_DEVICE_TIMEOUT."""
    _check("rf_selftest_bounded_wait", load().rf_selftest_bounded_wait(
        _ptr(status), int(limit_us), _stream(stream)))


def rf_frame_gram(P, G, stream=None):
    """G[i][j] = <P_i, P_j> for fp32 proxies P [F, E] (row stride P.stride(0)) into fp64 G."""
    F, E = P.shape
    _check("rf_frame_gram", load().rf_frame_gram(_ptr(P), F, E, P.stride(0), _ptr(G),
                                                 _stream(stream)))


def rf_keyframe_select(G, M: int, tau: float, dtau: float, delta_up: float, delta_down: float):
    """Algorithm 1 over a host fp64 Gram matrix; returns the keyframe mask (uint8 [F])."""
    G = np.ascontiguousarray(np.asarray(G, dtype=np.float64))
    F = G.shape[0]
    is_key = np.zeros(F, np.uint8)
    n = np.zeros(1, np.int32)
    _check("rf_keyframe_select", load().rf_keyframe_select(
        _ptr(G), F, M, tau, dtau, delta_up, delta_down, _ptr(is_key), _ptr(n)))
    return is_key


def rf_attn_workspace_bytes(d: int) -> int:
    n = load().rf_attn_workspace_bytes(d)
    if n < 0:
        raise RFError("rf_attn_workspace_bytes", 1)
    return n


def rf_step(z2, cur_slot, v, dt, active, counts, F: int, E: int, stream=None):
    _check("rf_step", load().rf_step(
        _ptr(z2), _ptr(cur_slot), _ptr(v), _ptr(dt), _ptr(active), _ptr(counts), F, E,
        _stream(stream)))


def rf_step_core(mask, cur_slot, alpha, beta, dt, F: int, N: int, E: int, H: int, d: int, active,
                 skipped, token_idx, counts, ctx, z2, v, Kc, Vc, O, lse, Q, K, V,
                 qkv_row_stride: int, kv_row_stride: int, o_row_stride: int,
                 softmax_scale: float, workspace=None, status=None, stream=None):
    """A whole step in two launches; Kc and Vc None: without the rolling cache."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rf_step_core", load().rf_step_core(
        _ptr(mask), _ptr(cur_slot), _ptr(alpha), _ptr(beta), _ptr(dt), F, N, E, H, d,
        _ptr(active), _ptr(skipped), _ptr(token_idx), _ptr(counts), _ptr(ctx), _ptr(z2), _ptr(v),
        _ptr(Kc), _ptr(Vc), _ptr(O), _ptr(lse), _ptr(Q), _ptr(K), _ptr(V), qkv_row_stride,
        kv_row_stride, o_row_stride, float(softmax_scale), _ptr(workspace), ws_bytes,
        _ptr(status), _stream(stream)))


_DTYPES: dict = {}  # torch types -> rf_dtype (torch is imported with the first tensor's call)
_PAIRINGS = {"interleaved": 0, "half": 1}
_ACTS = {None: 0, "none": 0, "gelu": 1, "gelu_tanh": 2, "silu": 3}
_F32 = 2


def _dtype(fn: str, t, *same) -> int:
    """rf_dtype of t; the tensors `same` (None is skipped) have to share it."""
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: _F32})
    kind = t.dtype
    for o in same:
        if o is not None and o.dtype is not kind:
            raise ValueError(f"{fn}: tensors of one type wanted, got {kind} and {o.dtype}")
    if kind not in _DTYPES:
        raise ValueError(f"{fn}: bf16, fp16 or fp32 wanted, got {kind}")
    return _DTYPES[kind]


def _rows(fn: str, name: str, t, shape) -> int:
    """Row stride of t [rows, n] or [rows, heads, d], whose rows have to be contiguous."""
    if t.shape != shape:
        raise ValueError(f"{fn}: {name} has shape {tuple(t.shape)}, not {shape}")
    n = shape[-1]
    if shape[0] > 1 and t.is_contiguous():  # (a single row counts as contiguous at any stride)
        return n * shape[1] if len(shape) == 3 else n
    st = t.stride()
    ok = st[-1] == 1 or n <= 1
    if len(shape) == 3:
        ok = ok and (st[1] == n or shape[1] <= 1)
        n *= shape[1]
    if not ok:
        raise ValueError(f"{fn}: a row of {name} is not contiguous (strides {st})")
    # one row: its stride is free, and torch may report any
    return st[0] if shape[0] > 1 or st[0] > n else n


def _row(fn: str, name: str, t, n: int) -> int:
    """Address of a row [n] or [1, n]."""
    if t.dim() != 1:
        _rows(fn, name, t, (1, n))
    elif t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{fn}: {name} is not a contiguous row of {n} ({tuple(t.shape)}, "
                         f"strides {t.stride()})")
    return t.data_ptr()


_NAMES: dict = {}  # torch types -> their names: str() of one takes as long as the whole check


def _whole(fn: str, name: str, t, shape, kinds) -> Optional[int]:
    """Address of an optional contiguous tensor of a given shape and type."""
    if t is None:
        return None
    kind = t.dtype
    if kind not in _NAMES:
        _NAMES[kind] = str(kind)
    if t.shape != shape or _NAMES[kind] not in kinds or not t.is_contiguous():
        raise ValueError(f"{fn}: {name} is not a contiguous {shape} of {' or '.join(kinds)}")
    return t.data_ptr()


def rf_rope_table(pos, dim: int, base: float = 10000.0):
    """(cos, sin) table of one axis, a host array fp32 [n, dim/2, 2], for any positions `pos`."""
    pos = np.ascontiguousarray(np.asarray(pos, dtype=np.float64))
    out = np.zeros((pos.size, max(dim, 0) // 2, 2), np.float32)
    _check("rf_rope_table", load().rf_rope_table(_ptr(pos), pos.size, dim, float(base), _ptr(out)))
    return out


def rf_rope(Yq, Xq, Yk, Xk, F: int, gh: int, gw: int, dims, tables, pairing: str = "interleaved",
            inverse: bool = False, active=None, counts=None, stream=None):
    """Rotary positions of queries Xq [F*gh*gw, Hq, d] and keys Xk (or None) into Yq and Yk, which
    may be the inputs themselves.  dims: rotated elements (time, height, width); tables: the three
    axes' device tables of rf_rope_table, None where dims is 0."""
    fn = "rf_rope"
    shape = (F * gh * gw, *Xq.shape[1:])
    dim_t, dim_h, dim_w = dims
    t, h, w = tables
    yq = _rows(fn, "Yq", Yq, shape)
    xq = yq if Xq is Yq else _rows(fn, "Xq", Xq, shape)
    kp = (None, None, 0, 0, 0)
    if Xk is not None:
        ks = (shape[0], Xk.shape[1], shape[2])
        yk = _rows(fn, "Yk", Yk, ks)
        kp = (Yk.data_ptr(), Xk.data_ptr(), yk, yk if Xk is Yk else _rows(fn, "Xk", Xk, ks), ks[1])
    elif Yk is not None:
        raise ValueError(f"{fn}: Yk without Xk")
    dt = _dtype(fn, Xq, Yq, Xk, Yk)
    f32 = ("torch.float32",)
    st = (_LIB or load()).rf_rope(
        Yq.data_ptr(), Xq.data_ptr(), yq, xq, shape[1], *kp, dt, F, gh, gw, shape[2], dim_t, dim_h,
        dim_w, _whole(fn, "time's table", t, (F, dim_t // 2, 2), f32),
        _whole(fn, "height's table", h, (gh, dim_h // 2, 2), f32),
        _whole(fn, "width's table", w, (gw, dim_w // 2, 2), f32), _PAIRINGS[pairing], inverse,
        _ptr(active), _ptr(counts), _stream(stream))
    if st:
        raise RFError(fn, st)


def rf_cross_attn(O, lse, Q, K, V, F: int, N: int, softmax_scale: float, kv_range=None,
                  key_mask=None, active=None, counts=None, status=None, stream=None):
    """Attention of Q [F*N, H, d] to an encoder's states K, V [L, Hkv, d], bf16 or fp16.

    kv_range int32 [F, 2]: the states [begin, end) each frame sees; key_mask uint8 or bool [L],
    zero = not seen; lse fp32 [H, F*N] or None."""
    fn = "rf_cross_attn"
    H, d = Q.shape[1:]
    kv = tuple(K.shape)
    L, Hkv, _ = kv
    rows = (F * N, H, d)
    if kv[2] != d:
        raise ValueError(f"{fn}: head dim {d} of Q, {kv[2]} of K")
    st = (_LIB or load()).rf_cross_attn(
        O.data_ptr(), _whole(fn, "lse", lse, (H, F * N), ("torch.float32",)), Q.data_ptr(),
        K.data_ptr(), V.data_ptr(), _rows(fn, "O", O, rows), _rows(fn, "Q", Q, rows),
        _rows(fn, "K", K, kv), _rows(fn, "V", V, kv), _dtype(fn, Q, O, K, V), F, N, H, Hkv, d, L,
        _whole(fn, "kv_range", kv_range, (F, 2), ("torch.int32",)),
        _whole(fn, "key_mask", key_mask, (L,), ("torch.uint8", "torch.bool")), _ptr(active),
        _ptr(counts), softmax_scale, _ptr(status), _stream(stream))
    if st:
        raise RFError(fn, st)


def rf_linear(Y, X, W, F: int, N: int, bias=None, act=None, gate=None, residual=None, active=None,
              counts=None, status=None, stream=None):
    """Y = residual + gate * act(X W^T + bias) for the active frames' rows.

    X [F*N, d_in], W [d_out, d_in] and bias [d_out] in bf16 or fp16; Y and residual [F*N, d_out]
    in that type or fp32; gate fp32 [d_out], or [F, d_out] for one per frame; act None, "gelu",
    "gelu_tanh" or "silu".  residual may be Y."""
    fn = "rf_linear"
    T = F * N
    d_out, d_in = W.shape
    dt, out = _dtype(fn, X, W, bias), _dtype(fn, Y, residual)
    b = g = r = None
    gate_stride = r_stride = 0
    if bias is not None:
        b = _row(fn, "bias", bias, d_out)
    if gate is not None:
        if _dtype(fn, gate) != _F32:
            raise ValueError(f"{fn}: gate is not fp32")
        if gate.dim() == 1:
            g = _row(fn, "gate", gate, d_out)
        else:
            gate_stride, g = _rows(fn, "gate", gate, (F, d_out)), gate.data_ptr()
    if residual is not None:
        r, r_stride = residual.data_ptr(), _rows(fn, "residual", residual, (T, d_out))
    st = (_LIB or load()).rf_linear(
        Y.data_ptr(), _rows(fn, "Y", Y, (T, d_out)), out, X.data_ptr(), _rows(fn, "X", X, (T, d_in)),
        W.data_ptr(), _rows(fn, "W", W, (d_out, d_in)), dt, F, N, d_in, d_out, b, _ACTS[act], g,
        gate_stride, r, r_stride, _ptr(active), _ptr(counts), _ptr(status), _stream(stream))
    if st:
        raise RFError(fn, st)


def rf_pipeline_create(F: int, N: int, H: int, d: int, E: int, plan: dict, z2, K0, V0,
                       depth: int, compute, h2d, d2h) -> int:
    """Host-fed step pipeline over the host plan (rf_plan_build's arrays), an initial fp32
    [2, F, E] latent store (host array or tensor) and the initial keys and values K0, V0 (bf16
    [F*N, H, d] contiguous host tensors) that both slots of the rolling cache start with;
    returns an opaque handle."""
    # every array is bound to a name, so that none is freed before the call reads it
    mask = np.ascontiguousarray(plan["mask"], dtype=np.uint8)
    alpha = np.ascontiguousarray(plan["alpha"], dtype=np.float32)
    beta = np.ascontiguousarray(plan["beta"], dtype=np.float32)
    dt = np.ascontiguousarray(plan["dt"], dtype=np.float32)
    slot = np.ascontiguousarray(plan["cur_slot"], dtype=np.uint8)
    z = np.ascontiguousarray(np.asarray(z2.cpu() if hasattr(z2, "cpu") else z2), dtype=np.float32)
    k0, v0 = (x.cpu().contiguous() if hasattr(x, "cpu") else np.ascontiguousarray(x)
              for x in (K0, V0))
    S = mask.shape[0]
    out = _vp()
    _check("rf_pipeline_create", load().rf_pipeline_create(
        F, N, H, d, E, S, _ptr(mask), _ptr(alpha), _ptr(beta), _ptr(dt), _ptr(slot), _ptr(z),
        _ptr(k0), _ptr(v0), depth, _stream(compute), _stream(h2d), _stream(d2h),
        ctypes.byref(out)))
    return out.value


def rf_pipeline_step(handle: int, s: int, hQ, hK, hV, hv, hO, hz2, hctx,
                     softmax_scale: float):
    _check("rf_pipeline_step", load().rf_pipeline_step(
        handle, s, _ptr(hQ), _ptr(hK), _ptr(hV), _ptr(hv), _ptr(hO), _ptr(hz2), _ptr(hctx),
        float(softmax_scale)))


def rf_pipeline_sync(handle: int) -> int:
    """Wait for every enqueued step; returns the device status word."""
    st = np.zeros(1, np.int32)
    _check("rf_pipeline_sync", load().rf_pipeline_sync(handle, _ptr(st)))
    return int(st[0])


def rf_pipeline_bytes(handle: int):
    """(steps, host->device bytes, device->host bytes) enqueued so far."""
    v = np.zeros(3, np.int64)
    _check("rf_pipeline_bytes", load().rf_pipeline_bytes(
        handle, v.ctypes.data, v.ctypes.data + 8, v.ctypes.data + 16))
    return int(v[0]), int(v[1]), int(v[2])


def rf_pipeline_destroy(handle: int):
    if handle:
        load().rf_pipeline_destroy(handle)
