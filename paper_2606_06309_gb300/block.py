"""A transformer block of a video diffusion model, run for the active frames of a step.

The step core's attention with the operators around it, on one stream with no host synchronisation:

  1. rf_linear   queries, keys and values of the active frames' tokens, one product
  2. rf_rope     rotary positions over time, height and width, in place
  3. rf_project_kv, rf_attn   (StepCore) skipped frames' keys and values from the layer's rolling cache,
                 which holds rotated keys; active queries over the whole sequence
  4. rf_linear   output projection, gated, onto the stream of hidden states
  5. rf_linear, rf_cross_attn, rf_linear   attention to the encoder's states, onto the stream
  6. rf_linear   feed-forward pair: activation in the first, gate and stream in the second

The hidden states are [F*N, D] for all frames; only the active frames' rows are read and written.
Normalisations stay the model's: each of the three is a callable on the hidden states.

A model's blocks run over one StepCore (plan, lists, workspace), each with a cache of its own:

    blocks = []
    for w in layers:
        blocks.append(ActiveBlock(core, gh, gw, w, dims, heads_kv, own_cache=True,
                                  buffers=blocks[0] if blocks else None))
    core.compact(s)                     # once per step
    for block in blocks: block.run(s, x, scale, ...)
"""
from __future__ import annotations

from contextlib import nullcontext
from dataclasses import dataclass
from typing import Callable, Optional, Tuple

import numpy as np
import torch

from . import _stream, rf_cross_attn, rf_linear, rf_rope, rf_rope_table
from .stepcore import StepCore

Linear = Tuple[torch.Tensor, Optional[torch.Tensor]]  # weight [out, in], bias [out] or None


@dataclass
class BlockWeights:
    qkv: Linear      # [3 H d, D]: queries, keys, values
    out: Linear      # [D, H d]
    cross_q: Linear  # [H d, D]
    cross_kv: Linear  # [2 Hkv d, De]: keys, values of the encoder's states
    cross_out: Linear  # [D, H d]
    up: Linear       # [Df, D]
    down: Linear     # [D, Df]


def _on(stream):
    """What torch allocates and runs inside (the norms, too) is ordered on `stream`."""
    if stream is None:
        return nullcontext()
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)


class _Enqueued:
    """The work on the current stream so far, for other streams to wait for.  Work recorded in a graph
    has no place among theirs, and a stream being captured cannot wait for what is outside: there
    the order is the caller's."""

    def __init__(self):
        self.stream, self.event = _stream(None), None
        if not torch.cuda.is_current_stream_capturing():
            self.event = torch.cuda.Event()
            self.event.record()

    def wait(self, at: int):
        """at: the current stream's handle."""
        if at != self.stream and self.event is not None and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().wait_event(self.event)


def _one_layer(core: StepCore, block, s: int):
    """Refuse core's cache where it lost this block's keys: this block and then another one stored theirs
    of the step before, and this one now wants them back for frames that are skipped."""
    Kc = core.Kc
    if Kc.is_inference():  # counts no versions
        return
    cache = (Kc.data_ptr(), Kc._version)  # replaced or written by the caller: another layer's now
    last_cache, last_s, writers = getattr(core, "_cache_writers", (None, None, []))
    if cache == last_cache and s == last_s:
        core._cache_writers = (cache, s, [w for w in writers if w != id(block)] + [id(block)])
        return
    if cache == last_cache and id(block) in writers[:-1] and not core.plan.host["mask"][s].all():
        raise ValueError("ActiveBlock: another block has stored its keys in the step core's cache: "
                         "blocks that share a step core each need own_cache=True")
    core._cache_writers = (cache, s, [id(block)])


class ActiveBlock:
    """Buffers and tables of one block over `core`'s frames, whose N tokens are a grid gh x gw.

    dims: rotated elements of a head per axis (time, height, width).  positions: the axes' positions,
    0, 1, 2, ... where None.  Weights are bf16, the step core's type.

    own_cache: a rolling key/value cache of this block's own, zeros at first (set_kv_cache), so that
    several blocks can share core, which may then have none.  Otherwise core's cache is this
    layer's, and no other's.

    buffers: another block whose buffers (not its cache) this one uses too, as it runs before or after
    that one on the same stream: 75,600 tokens, D = 5120, feed-forward 13,824 take 5.2 GB.  Without a
    cache, its own or core's, a block's buffers hold its skipped frames' keys and cannot be shared.

    encode and run may be given different streams: run waits for the encoder's states and for the
    block's making, and states are kept until the runs that read them are done.  What else a call
    reads is the caller's to order, and a block is kept while runs on other streams than it was
    made on are under way."""

    def __init__(self, core: StepCore, gh: int, gw: int, weights: BlockWeights, dims, heads_kv: int,
                 positions=None, base: float = 10000.0, pairing: str = "interleaved",
                 act: str = "gelu_tanh", own_cache: bool = False,
                 buffers: Optional["ActiveBlock"] = None):
        if gh * gw != core.N:
            raise ValueError(f"a grid of {gh} x {gw} is not {core.N} tokens")
        if weights.qkv[0].dtype is not torch.bfloat16:  # the step core reads queries, keys, values so
            raise ValueError(f"weights of {weights.qkv[0].dtype}: the step core's attention is of "
                             "torch.bfloat16")
        self.core, self.gh, self.gw, self.w = core, gh, gw, weights
        self.dims, self.heads_kv, self.pairing, self.act = tuple(dims), heads_kv, pairing, act
        T, H, d = core.F * core.N, core.H, core.d
        wt = weights.qkv[0]
        pos = positions or [np.arange(n) for n in (core.F, gh, gw)]
        self.tables = [torch.from_numpy(rf_rope_table(p, dim, base)).to(wt.device) if dim else None
                       for p, dim in zip(pos, self.dims)]

        def zeros(name, *shape):
            if buffers is None:
                return torch.zeros(shape, dtype=wt.dtype, device=wt.device)
            t = getattr(buffers, name)
            if t.shape != shape or t.device != wt.device:
                raise ValueError(f"{name} is {tuple(t.shape)} on {t.device} in the block whose buffers are "
                                 f"to be shared, not {shape} on {wt.device}")
            return t

        if buffers is not None:
            if (not own_cache and core.Kc is None) or (buffers.cache is None and buffers.core.Kc is None):
                raise ValueError("a block without a cache has its skipped frames' keys in its buffers")
            if buffers._made is not None:
                buffers._made.wait(_stream(None))
        self.qkv = zeros("qkv", T, 3, H, d)
        self.rows = zeros("rows", T, H, d)  # attention's results
        self.ffn = zeros("ffn", T, weights.up[0].shape[0])
        self.cache = None      # own keys and values, [2, F, N, H d] each
        if own_cache:
            self.cache = tuple(torch.zeros(2, core.F, core.N, H * d, dtype=wt.dtype, device=wt.device)
                               for _ in range(2))
        self.enc = None        # [L, 2, Hkv, d]
        self.enc_mask = self.enc_range = None
        self._made, self._encoded = _Enqueued() if wt.is_cuda else None, None
        self._enc_homes = ()   # streams that the states and what is kept with them were allocated on
        self._enc_read = {}    # stream -> event behind its last run that read them
        self._enc_old = []     # earlier states still being read, with such events

    def set_kv_cache(self, K0: torch.Tensor, V0: torch.Tensor):
        """StepCore.set_kv_cache for this layer's cache."""
        self.core.set_kv_cache(K0, V0, self.cache)

    def encode(self, states: torch.Tensor, mask=None, ranges=None, stream=None):
        """Keys and values of an encoder's states [L, De], kept until the next call: once per prompt.
        mask [L]: zero = padding; ranges int32 [F, 2]: the states each frame sees."""
        L = states.shape[0]
        w, b = self.w.cross_kv
        capturing = torch.cuda.is_current_stream_capturing
        homes = () if mask is None and ranges is None else (_stream(None),)
        quiet = capturing()  # nothing may be asked of events outside a capture
        with _on(stream):
            enc = torch.empty(L, 2, self.heads_kv, self.core.d, dtype=w.dtype, device=w.device)
            rf_linear(enc.view(L, -1), states, w, 1, L, bias=b, status=self.core.status)
            encoded, quiet = _Enqueued(), quiet or capturing()
        if not quiet:
            self._enc_old = [o for o in self._enc_old if not all(e.query() for e in o[-1])]
        if self._enc_read:
            self._enc_old.append((self.enc, self.enc_mask, self.enc_range, list(self._enc_read.values())))
        self.enc, self.enc_mask, self.enc_range = enc, mask, ranges
        self._encoded, self._enc_homes, self._enc_read = encoded, (encoded.stream, *homes), {}

    def run(self, s: int, x: torch.Tensor, scale: float, norms=(None, None, None), gates=(None, None),
            stream=None):
        """Step s: x [F*N, D], rows of the active frames updated in place.  norms: callables in front
        of the attention, the attention to the encoder and the feed-forward pair (None: none);
        gates: fp32 [D] or [F, D] of the attention and of the feed-forward pair (None: 1).

        core.compact(s) has been called for the step (once, for all blocks)."""
        with _on(stream):
            at = _stream(None)
            for before in (self._made, self._encoded):
                if before is not None:
                    before.wait(at)
            try:
                self._run(s, x, scale, norms, gates)
            finally:
                if any(h != at for h in self._enc_homes) and not torch.cuda.is_current_stream_capturing():
                    if at not in self._enc_read:
                        self._enc_read[at] = torch.cuda.Event()
                    self._enc_read[at].record()

    def _run(self, s, x, scale, norms, gates):
        c, w = self.core, self.w
        T, F, N, H, d = c.F * c.N, c.F, c.N, c.H, c.d
        on = dict(active=c.active, counts=c.counts)
        lin = dict(on, status=c.status)
        n1, n2, n3 = (n or (lambda h: h) for n in norms)
        q, k, v = self.qkv.unbind(1)
        if self.cache is None and c.Kc is not None:
            _one_layer(c, self, s)

        rf_linear(self.qkv.view(T, -1), n1(x), w.qkv[0], F, N, bias=w.qkv[1], **lin)
        rf_rope(q, q, k, k, F, self.gh, self.gw, self.dims, self.tables, pairing=self.pairing, **on)
        if self.cache is not None:
            c.project_kv(s, k, v, cache=self.cache)
        elif c.Kc is not None:
            c.project_kv(s, k, v)
        c.attn(self.rows, q, k, v, scale)
        rf_linear(x, self.rows.view(T, H * d), w.out[0], F, N, bias=w.out[1], gate=gates[0],
                  residual=x, **lin)

        if self.enc is not None:
            qc = self.qkv[:, 0]
            rf_linear(qc.view(T, H * d), n2(x), w.cross_q[0], F, N, bias=w.cross_q[1], **lin)
            rf_cross_attn(self.rows, None, qc, self.enc[:, 0], self.enc[:, 1], F, N, scale,
                          kv_range=self.enc_range, key_mask=self.enc_mask, **lin)
            rf_linear(x, self.rows.view(T, H * d), w.cross_out[0], F, N, bias=w.cross_out[1],
                      residual=x, **lin)

        rf_linear(self.ffn, n3(x), w.up[0], F, N, bias=w.up[1], act=self.act, **lin)
        rf_linear(x, self.ffn, w.down[0], F, N, bias=w.down[1], gate=gates[1], residual=x, **lin)
