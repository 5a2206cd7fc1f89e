"""Convenience layer over the binding: upload weights, allocate the workspace
and outputs with PyTorch, run ``octree_nca_infer``; state caches, parameter lists,
training and cell layers.  Allocation and marshalling only; the computation is the library's.
"""
from __future__ import annotations

import contextlib
import warnings
from typing import List, Optional, Sequence

import numpy as np
import torch

from . import (Model, MX4Buffers, OctreeNCAError, StateCacheBuffers, _stream, _cache_call,
               check_train_weights, lib, mx4_shapes, octree_nca_adamw, octree_nca_clip_grads,
               octree_nca_dropout, octree_nca_grad_norm, octree_nca_infer,
               octree_nca_mx4_backward, octree_nca_mx4_backward_workspace_bytes,
               octree_nca_mx4_dequantise, octree_nca_mx4_linear, octree_nca_mx4_product,
               octree_nca_mx4_quantise, octree_nca_param_table, octree_nca_param_table_bytes,
               octree_nca_train_kept_workspace_bytes, octree_nca_train_step,
               octree_nca_train_step_kept, octree_nca_train_workspace_bytes,
               octree_nca_workspace_bytes, param_structs, state_cache_refs)

WEIGHT_FIELDS = ("conv_w", "conv_b", "w1", "b1", "w2")


def upload_weights(levels, device="cuda") -> List[dict]:
    """Per-level weights (objects or dicts holding fp32 numpy arrays in the
    canonical layout) -> list of dicts of contiguous fp32 device tensors."""
    out = []
    for w in levels:
        get = (lambda k: w[k]) if isinstance(w, dict) else (lambda k: getattr(w, k))
        out.append({k: torch.from_numpy(np.ascontiguousarray(get(k), dtype=np.float32))
                    .to(device) for k in WEIGHT_FIELDS})
    return out


def to_device_image(image: np.ndarray, model: Model, device="cuda") -> torch.Tensor:
    """[D][H][W][n_in] numpy image -> contiguous device tensor of the model's storage type."""
    assert image.ndim == 4 and image.shape[-1] == model.n_in
    with warnings.catch_warnings():
        # a read-only (memory-mapped) array is only read by the copy below
        warnings.filterwarnings("ignore", message="The given NumPy array is not writable")
        t = torch.from_numpy(np.ascontiguousarray(image))
    return t.to(device=device, dtype=model.torch_dtype)


class Inference:
    """Buffers for repeated inference of one model on one finest extent."""

    def __init__(self, model: Model, finest: Sequence[int], factors, device="cuda",
                 want_state=True, want_seg=True):
        self.model = model
        self.finest = tuple(int(v) for v in finest)
        self.factors = [tuple(int(v) for v in f) for f in factors]
        ws = octree_nca_workspace_bytes(model, self.finest, self.factors, want_state)
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=device)
        d, h, w = self.finest
        self.state = (torch.empty((d, h, w, model.channels), dtype=model.torch_dtype,
                                  device=device) if want_state else None)
        self.seg = torch.empty((d, h, w), dtype=torch.uint8, device=device) if want_seg else None

    def __call__(self, image: torch.Tensor, weights, steps, fire_rate: float, seed: int,
                 level_events=None, stream=None):
        octree_nca_infer(self.model, image, self.factors, weights, steps, fire_rate, seed,
                         self.workspace, self.state, self.seg, level_events, stream)
        return self.state, self.seg


def infer(model: Model, image: torch.Tensor, factors, weights, steps, fire_rate: float,
          seed: int, stream=None):
    """One-shot inference; returns (final state, seg) as device tensors."""
    run = Inference(model, image.shape[:3], factors, device=image.device)
    return run(image, weights, steps, fire_rate, seed, stream=stream)


def _torch_stream(stream):
    """torch's stream of a stream or a handle (0: the default stream)."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream)) if stream else torch.cuda.default_stream()


def _on(stream):
    """Context in which torch allocates and fills on ``stream`` (None: as it is)."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(_torch_stream(stream))


class _Buffers:
    """An object's own buffers, filled on the stream that is current here.  The
    first use on another stream waits for the fills, and torch does not hand the
    memory out again before that stream's work so far is done (a stream given as
    a handle may be gone by then, so there the object has to outlive the work)."""

    def __init__(self, *tensors):
        self.tensors = tensors
        self.streams = {_stream(None)}     # that torch keeps the memory for
        self.waited = set(self.streams)    # that come after the fills
        # within a capture the graph has its own order
        self.filled = None if torch.cuda.is_current_stream_capturing() else torch.cuda.Event()
        if self.filled is not None:
            self.filled.record()

    def use(self, stream) -> int:
        """Handle of the stream of a call."""
        handle = _stream(stream)
        if handle not in (self.waited if type(stream) is int else self.streams):
            self._first_use(stream, handle)
        return handle

    def _first_use(self, stream, handle):
        # a captured stream cannot wait for work outside; torch starts a capture
        # with the device idle
        if self.filled is None or torch.cuda.is_current_stream_capturing():
            return
        if stream is None:
            stream = torch.cuda.current_stream()
        if handle not in self.waited:
            _torch_stream(stream).wait_event(self.filled)
            self.waited.add(handle)
        if isinstance(stream, torch.cuda.Stream):
            for t in self.tensors:
                t.record_stream(stream)
            self.streams.add(handle)


class StateCache:
    """States of one model and extent held in 8 bits (octnca_state_cache):
    ``slots`` of them, each channel of ``block`` consecutive cells with one
    scale.  ``codes`` / ``scales``: device memory to use instead of new.  Calls
    on any stream come after the fill of new memory; among each other they are
    ordered by the caller, as is what else made the tensors they are given."""

    def __init__(self, model: Model, extent: Sequence[int], slots: int, code="i8", block=64,
                 codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                 device="cuda"):
        self.model = model
        self.extent = tuple(int(v) for v in extent)
        d, h, w = self.extent
        cells, c = d * h * w, model.channels
        own = []
        if codes is None:
            codes = torch.zeros((slots, cells, c), dtype=torch.int8, device=device)
            own.append(codes)
        if scales is None:
            scales = torch.zeros((slots, -(-cells // block), c), device=device)
            own.append(scales)
        self.buffers = StateCacheBuffers(codes, scales, cells, code, block)
        self.refs = state_cache_refs(model, self.buffers)
        self._own = _Buffers(*own)

    def write(self, states: torch.Tensor, slots: Optional[torch.Tensor] = None, first=0,
              from_cell=0, stream=None) -> None:
        """states [n][...][C]: whole states, or their cells from ``from_cell`` on.
        ``slots``: device int64 [n], entries outside the cache are left out; or
        None for slots first, first + 1, ..."""
        _cache_call(lib().octree_nca_state_cache_write, self.model, self.refs, states, from_cell,
                    slots, first, self._own.use(stream))

    def read(self, out: torch.Tensor, slots: Optional[torch.Tensor] = None, first=0, from_cell=0,
             stream=None) -> torch.Tensor:
        """Fills and returns ``out`` [n][...][C]; slots outside the cache read as zeros."""
        _cache_call(lib().octree_nca_state_cache_read, self.model, self.refs, out, from_cell, slots,
                    first, self._own.use(stream))
        return out


class Parameters:
    """Many tensors with their gradients, listed once: global norm, clipping and
    the clipped AdamW update, a few launches whatever their number.

    ``grads`` are fp32, fp16 or bf16; ``clipped`` (fp32, fp16 or bf16; may be
    ``grads``) receives the clipped gradients; ``params``, ``m``, ``v`` and
    ``ema`` are fp32.  The tensors are read and written where they are: the list
    keeps them alive, and they must not be replaced by others.  ``step`` is the
    number of updates made so far (device int64 [1]).  Calls of one list must
    not overlap (it holds their scratch memory).  ``stream`` is the one that the
    list is made on; calls on any stream come after that."""

    def __init__(self, grads, params=None, m=None, v=None, ema=None, clipped=None,
                 step: Optional[torch.Tensor] = None, stream=None):
        self.tensors = [list(x) if x is not None else None
                        for x in (grads, params, m, v, ema, clipped)]
        device = self.tensors[0][0].device if self.tensors[0] else torch.device("cuda")
        structs = param_structs(*self.tensors)
        n = len(self.tensors[0])
        size = octree_nca_param_table_bytes(structs, n)
        with _on(stream):
            self.table = torch.empty(size, dtype=torch.uint8, device=device)
            self.list = octree_nca_param_table(structs, n, self.table)
            self.norm = torch.zeros((), device=device)
            own = [self.table, self.norm]
            if step is None:
                step = torch.zeros(1, dtype=torch.int64, device=device)
                own.append(step)
            self.step = step
            self._own = _Buffers(*own)

    def grad_norm(self, scale=1.0, stream=None) -> torch.Tensor:
        """scale * (2-norm of all gradients), a device scalar that the next call overwrites."""
        octree_nca_grad_norm(self.list, self.norm, scale, self._own.use(stream))
        return self.norm

    def clip(self, max_norm: float, scale=1.0, stream=None) -> torch.Tensor:
        """clipped = scale * gradients, shortened to ``max_norm`` if their norm
        is larger; returns the norm (as grad_norm)."""
        octree_nca_clip_grads(self.list, max_norm, scale, self.norm, self._own.use(stream))
        return self.norm

    def adamw(self, lr: float, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0,
              max_norm=float("inf"), scale=1.0, ema_decay=0.99, stream=None) -> torch.Tensor:
        """One update with the clipped gradients; left out if their norm is not
        finite.  Returns the norm before clipping (as grad_norm)."""
        octree_nca_adamw(self.list, self.step, lr, betas, eps, weight_decay, max_norm, scale,
                         ema_decay, self.norm, self._own.use(stream))
        return self.norm


class Trainer:
    """Training of one model on images of one extent: gradients of a training
    step, then the clipped AdamW update of all weights with a running average.

    ``weights``: per level a dict of device fp32 tensors (upload_weights),
    updated in place; ``ema`` their running averages.  ``keep``: None keeps every
    state in fp32 (octree_nca_train_step), "i8" or "f8" in 8 bits
    (octree_nca_train_step_kept), in about half the memory at 20 steps a level
    and less with more steps.  Steps on any stream come after what the
    constructor enqueued; steps on several streams are ordered by the caller."""

    def __init__(self, model: Model, finest: Sequence[int], factors, steps, weights,
                 keep: Optional[str] = None, block=64, lr=1.6e-3, betas=(0.9, 0.99), eps=1e-8,
                 weight_decay=0.0, max_norm=float("inf"), ema_decay=0.99):
        self.model, self.weights, self.keep, self.block = model, weights, keep, block
        self.finest = tuple(int(v) for v in finest)
        self.factors = [tuple(int(v) for v in f) for f in factors]
        self.steps = [int(v) for v in steps]
        check_train_weights(model, len(self.steps), weights)
        device = weights[0]["w1"].device
        if keep is None:
            size = octree_nca_train_workspace_bytes(model, self.finest, self.factors, self.steps)
        else:
            size = octree_nca_train_kept_workspace_bytes(model, self.finest, self.factors,
                                                         self.steps, keep, block)
        if size == 0:
            raise OctreeNCAError("Trainer: invalid model, extent, factors or steps")
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)
        like = lambda f: [{k: f(w[k]) for k in WEIGHT_FIELDS} for w in weights]
        self.grads, self.ema = like(torch.zeros_like), like(torch.clone)
        m, v = like(torch.zeros_like), like(torch.zeros_like)
        flat = lambda sets: [s[k] for s in sets for k in WEIGHT_FIELDS]
        self.loss = torch.zeros(1, dtype=torch.float64, device=device)
        self._own = _Buffers(self.workspace, self.loss,
                             *(t for sets in (self.grads, self.ema, m, v) for t in flat(sets)))
        self.parameters = Parameters(flat(self.grads), flat(weights), flat(m), flat(v),
                                     ema=flat(self.ema))
        self.settings = dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay,
                             max_norm=max_norm, ema_decay=ema_decay)

    def gradients(self, image: torch.Tensor, target: torch.Tensor, fire_rate: float, seed: int,
                  final_state=None, stream=None) -> torch.Tensor:
        """Fills ``grads``; returns the loss (device fp64 [1], overwritten by the next call)."""
        want = self.finest + (self.model.n_in,)
        if tuple(image.shape) != want:
            raise OctreeNCAError(f"image: expected {want}, got {tuple(image.shape)}")
        stream = self._own.use(stream)
        if self.keep is None:
            octree_nca_train_step(self.model, image, self.factors, self.weights, self.steps,
                                  fire_rate, seed, target, self.workspace, self.grads, self.loss,
                                  final_state, stream)
        else:
            octree_nca_train_step_kept(self.model, image, self.factors, self.weights, self.steps,
                                       fire_rate, seed, target, self.workspace, self.grads,
                                       self.loss, final_state, self.keep, self.block, stream)
        return self.loss

    def step(self, image: torch.Tensor, target: torch.Tensor, fire_rate: float, seed: int,
             stream=None, **settings):
        """One training step with an update; ``settings`` override the
        constructor's for this step (lr, ...).  Returns the loss and the
        gradients' norm before clipping, both on the device."""
        loss = self.gradients(image, target, fire_rate, seed, stream=stream)
        norm = self.parameters.adamw(stream=stream, **{**self.settings, **settings})
        return loss, norm


class MX4Matrix:
    """Rows of values in microscaled 4 bits (octnca_mx4), 17 bytes for 32 columns:
    ``rows`` of them at most, ``used`` by the last quantise.  ``codes`` /
    ``scales``: device memory of mx4_shapes to use instead of new."""

    def __init__(self, rows: int, cols: int, codes: Optional[torch.Tensor] = None,
                 scales: Optional[torch.Tensor] = None, device="cuda"):
        self.rows, self.cols = int(rows), int(cols)
        shapes = mx4_shapes(self.rows, self.cols)
        own = []
        if codes is None:
            codes = torch.zeros(shapes[0], dtype=torch.uint8, device=device)
            own.append(codes)
        if scales is None:
            scales = torch.zeros(shapes[1], dtype=torch.uint8, device=device)
            own.append(scales)
        self.buffers = MX4Buffers(self.rows, self.cols, codes, scales)
        self.struct = self.buffers.struct()
        self._own = _Buffers(*own)

    @property
    def used(self) -> int:
        return self.struct.rows

    @used.setter
    def used(self, n: int):
        if not 0 <= n <= self.rows:
            raise OctreeNCAError(f"{n} rows, the matrix has room for {self.rows}")
        self.struct.rows = n

    def quantise(self, x: torch.Tensor, stream=None) -> "MX4Matrix":
        """Takes x [...][cols], of fp32, fp16 or bf16."""
        before, self.used = self.used, x.numel() // self.cols
        try:
            octree_nca_mx4_quantise(x, self.struct, self._own.use(stream))
        except Exception:      # refused: nothing has been written
            self.used = before
            raise
        return self

    def dequantise(self, out: torch.Tensor, stream=None) -> torch.Tensor:
        """Fills and returns ``out`` [...][cols] with the rows in use."""
        octree_nca_mx4_dequantise(self.struct, out, self._own.use(stream))
        return out


class CellLayer:
    """A linear layer on every cell, out = x weight^T + bias, with weights and
    inputs in microscaled 4 bits.

    ``weight`` [outs][cols] and ``bias`` (fp32 [outs] or None) stay the caller's;
    ``refresh`` takes the weights over after they change.  ``rows``: the most cells
    of a call.  ``train``: with memory for the gradients ``grad_weight`` and
    ``grad_bias`` (fp32).  Calls of one layer must not overlap: it holds the kept
    inputs and the gradients.  Calls on any stream come after what the constructor
    enqueued, and are ordered among each other by the caller."""

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, rows=1,
                 train=False):
        if weight.dim() != 2:
            raise OctreeNCAError(f"weight: expected [outs][cols], got {tuple(weight.shape)}")
        self.weight, self.bias = weight, bias
        self.outs, self.cols = weight.shape
        self.w = MX4Matrix(self.outs, self.cols, device=weight.device)
        self.kept = MX4Matrix(rows, self.cols, device=weight.device)
        self.last = self.kept      # what the last forward has multiplied
        self.grad_weight = self.grad_bias = self.workspace = None
        own = [self.w.buffers.codes, self.w.buffers.scales, self.kept.buffers.codes,
               self.kept.buffers.scales]
        if train:
            size = octree_nca_mx4_backward_workspace_bytes(rows, self.cols, self.outs)
            if size == 0:
                raise OctreeNCAError("CellLayer: invalid rows or weights")
            device = weight.device
            self.workspace = torch.empty(size, dtype=torch.uint8, device=device)
            self.grad_weight = torch.zeros((self.outs, self.cols), device=device)
            self.grad_bias = torch.zeros(self.outs, device=device) if bias is not None else None
            own += [t for t in (self.workspace, self.grad_weight, self.grad_bias) if t is not None]
        self.refresh()
        self._own = _Buffers(*own)

    def refresh(self, stream=None) -> None:
        """Takes ``weight`` over."""
        self.w.quantise(self.weight, stream)

    def forward(self, x, out: torch.Tensor, relu=False, stream=None) -> torch.Tensor:
        """Fills and returns ``out`` [...][outs].  x: [...][cols], left in 4 bits in
        ``kept``; or an MX4Matrix of such rows."""
        handle = self._own.use(stream)
        if isinstance(x, MX4Matrix):
            x._own.use(stream)
            octree_nca_mx4_product(x.struct, self.w.struct, out, self.bias, relu, handle)
            self.last = x
        else:
            kept = self.kept
            before, kept.used = kept.used, x.numel() // self.cols
            try:
                octree_nca_mx4_linear(x, kept.struct, self.w.struct, out, self.bias, relu, handle)
            except Exception:      # refused: nothing has been written
                kept.used = before
                raise
            self.last = kept
        return out

    def backward(self, grad_out: torch.Tensor, grad_in: Optional[torch.Tensor] = None,
                 kept: Optional[MX4Matrix] = None, stream=None) -> None:
        """Fills ``grad_weight`` and ``grad_bias``, and grad_in [...][cols] (of
        grad_out's type) if given, for the gradient of the last forward's out
        (without its relu), or of the product of the rows ``kept``."""
        if self.workspace is None:
            raise OctreeNCAError("CellLayer: made without train=True")
        handle = self._own.use(stream)
        rows = self.last if kept is None else kept
        rows._own.use(stream)
        octree_nca_mx4_backward(grad_out, rows.struct, self.w.struct, grad_in, self.grad_weight,
                                self.grad_bias, self.workspace, handle)


class Dropout:
    """Dropout with a mask that is drawn anew in every call (octnca_dropout).

    A mask is that of ``seed`` and index + step: each layer takes a seed of its own (of
    one seed, index 1 drops at a step what index 0 drops at the next).
    ``step``: device int64 [1] that counts training steps, read by the kernel and
    added to ``index``, so that a captured graph draws a new mask each time it is
    replayed; the gradient has to see the same value as the forward."""

    def __init__(self, rate: float, seed: int, step: Optional[torch.Tensor] = None):
        self.rate, self.seed, self.step = float(rate), int(seed), step

    def __call__(self, x: torch.Tensor, out: torch.Tensor, gate: Optional[torch.Tensor] = None,
                 add: Optional[torch.Tensor] = None, index=0, stream=None) -> torch.Tensor:
        """Fills and returns ``out`` (which may be x, gate or add): x where it is
        kept and gate > 0, scaled, plus ``add``.  ReLU and dropout: gate = x; their
        gradient: x the gradient, the same gate and index."""
        octree_nca_dropout(x, out, self.rate, self.seed, index, self.step, gate, add, stream)
        return out
