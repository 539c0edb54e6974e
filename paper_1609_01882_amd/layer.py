"""What a layer needs around its attention memory: rotary positions and norms around a block -- argument marshalling for the
`psc_rotary_*` and `psc_residual_norm_*` calls (see `include/psc.h`).

    rope = psc.Rotary(128)                                  # or frequencies=psc.rotary_frequencies(128, stretch=8.0, ...)
    q = rope(q, positions)                                  # [rows, heads, head_dim], differentiable
    q = cache.append(k, v, table, lengths, first=seen, rotary=rope, q=q)      # keys turned on their way into the memory
    x, z = psc.residual_norm(x, y, after=w1, gate=g, activation="sigmoid", before=w2)       # differentiable
"""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch

from .binding import PscError, _check, _load, _workspace
from .kv import _DTYPES, _array, _dtype, _duals, _no_tangents, _stream_address


class _Rotary(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("dims", C.c_int), ("interleaved", C.c_int), ("factor", C.c_float)]


class _Norm(C.Structure):
    _fields_ = [("rows", C.c_int), ("width", C.c_int), ("stream_dtype", C.c_int), ("block_dtype", C.c_int), ("weight_dtype", C.c_int),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("y", C.c_void_p), ("y_stride", C.c_int64), ("gate", C.c_void_p),
                ("gate_stride", C.c_int64), ("gate_rows", C.c_int), ("activation", C.c_int), ("after", C.c_void_p), ("before", C.c_void_p),
                ("residual_scale", C.c_float), ("block_scale", C.c_float), ("eps", C.c_float)]


_pack = struct.Struct("@5iPqPqPq2i2P3f0P").pack     # the same fields, packed at once: a call of a few microseconds notices
assert struct.calcsize("@5iPqPqPq2i2P3f0P") == C.sizeof(_Norm)


_MOST_FLOAT32 = float.fromhex("0x1.fffffep127")


def _current(index, what):
    if torch.cuda.current_device() != index:
        raise PscError(f"{what} is on cuda:{index}, the current device is cuda:{torch.cuda.current_device()}")
    return _stream_address(index)


def _once(backward):
    """A backward pass that cannot be differentiated again.  (The wrapper that says so to autograd costs a tenth of a small step, and is
    needed only where a graph of the gradients is asked for.)"""
    guarded = torch.autograd.function.once_differentiable(backward)
    return staticmethod(lambda ctx, *grads: (guarded if torch.is_grad_enabled() else backward)(ctx, *grads))


# ------------------------------------------------------------------------------------------- rotary positions
def rotary_frequencies(dims: int, base: float = 10000.0, *, stretch: float = 1.0, trained: int | None = None, low: float = 1.0,
                       high: float = 4.0, blend: str = "turns"):
    """Radians that a position adds to each of the dims / 2 pairs: base ** (-2 i / dims), as a list of float64.

    `stretch` s > 1 makes them fit s times longer contexts.  Without `trained` all are divided by s (positions interpolated).
    With it -- the length that the model was trained for -- pairs that turn more than `high` times within it stay as they
    are, those that turn fewer than `low` times are divided by s, and those between get a share of both: linear in their
    turns (blend="turns"), or in their number i between the two borders, rounded outwards (blend="pairs")."""
    if dims < 2 or dims % 2:
        raise PscError(f"dims: expected an even number from 2 on, got {dims}")
    if not base > 1.0 or not stretch > 0.0 or not math.isfinite(base) or not math.isfinite(stretch):
        raise PscError(f"base ({base}) must be above 1, stretch ({stretch}) above 0")
    f = [base ** (-2.0 * i / dims) for i in range(dims // 2)]
    if trained is None:
        return [x / stretch for x in f]
    if not 0.0 < low < high or trained < 1 or blend not in ("turns", "pairs"):
        raise PscError(f"trained ({trained}) must be positive, low ({low}) positive and below high ({high}), blend \"turns\" or \"pairs\"")
    if blend == "turns":
        keep = [(trained * x / (2.0 * math.pi) - low) / (high - low) for x in f]
    else:
        border = lambda turns: dims * math.log(trained / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))  # noqa: E731
        first, last = max(math.floor(border(high)), 0), min(math.ceil(border(low)), dims - 1)
        keep = [1.0 - (i - first) / max(last - first, 1e-3) for i in range(dims // 2)]
    keep = [min(max(k, 0.0), 1.0) for k in keep]
    return [x * k + x / stretch * (1.0 - k) for x, k in zip(f, keep)]


class Rotary:
    """Turns the first `dims` coordinates of heads by their row's position.  `frequencies` (dims / 2 radians to a position;
    None: `rotary_frequencies(dims, base)`), `interleaved`: pairs of neighbours, not half of `dims` apart; `factor`
    scales what is turned."""

    def __init__(self, dims: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0, frequencies=None, device="cuda"):
        frequencies = rotary_frequencies(dims, base) if frequencies is None else [float(f) for f in frequencies]
        if dims < 2 or dims % 2 or len(frequencies) != dims // 2:
            raise PscError(f"dims ({dims}) must be even, with a frequency for each pair, got {len(frequencies)}")
        if not abs(factor) <= _MOST_FLOAT32:
            raise PscError("factor must be finite in 32 bits")
        turns = (C.c_uint64 * (dims // 2))()
        _check(_load().psc_rotary_turns((C.c_double * (dims // 2))(*frequencies), dims // 2, turns))
        self.dims, self.interleaved, self.factor, self.frequencies = dims, bool(interleaved), float(factor), frequencies
        signed = [t - (1 << 64) if t >> 63 else t for t in turns]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.device, self._index = self.turns.device, self.turns.get_device()
        self._struct = bytes(_Rotary(self.turns.data_ptr(), dims, self.interleaved, self.factor))

    def __call__(self, x, positions=None, first=None, offsets=None, out=None):
        """x [rows, heads, head_dim] (or [rows, head_dim]) turned: row r at positions[r] (int32), or at first[b] + its place in
        its sequence b, [batch] (int32; `offsets` [batch + 1]: where sequences begin, None: equal parts), or at r.
        Rows that no sequence has are copied.  Differentiable in x, backwards (an x that carries a tangent is refused); `out` (which may be x):
        written, and no gradient."""
        if _duals._current_level >= 0:
            _no_tangents(x, out)
        if out is None and x.requires_grad and torch.is_grad_enabled():
            return _Turned.apply(x, self, positions, first, offsets)
        if out is not None and torch.is_grad_enabled() and (x.requires_grad or out.requires_grad):
            raise PscError("out: has no gradient; detach x, or call under torch.no_grad()")
        return self._turn(x, positions, first, offsets, out, False)

    def inverse(self, x, positions=None, first=None, offsets=None, out=None):
        """The transposed: turned back, times the factor (with factor 1 the inverse).  Nothing flows back."""
        if _duals._current_level >= 0:
            _no_tangents(x, out)
        if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
            raise PscError("x: the transposed has no gradient; detach x, or call under torch.no_grad()")
        return self._turn(x, positions, first, offsets, out, True)

    def _turn(self, x, positions, first, offsets, out, transposed):
        stream, index = _current(self._index, "the rotary"), self._index
        code, shape = _dtype(x, "x"), x.shape
        if len(shape) == 3:
            rows, heads, dim = shape
            row_stride, head_stride, last = x.stride()
        elif len(shape) == 2:
            (rows, dim), heads, (row_stride, last), head_stride = shape, 1, x.stride(), 0
        else:
            rows, heads, dim, last = 0, 0, 0, 0
        if x.get_device() != index or dim < self.dims or last != 1:
            raise PscError(f"x: expected [rows, heads, head_dim >= {self.dims}] on {self.device} with contiguous coordinates, got {list(shape)} "
                           f"with strides {list(x.stride())} on {x.device}")
        batch = 1
        if positions is not None and (first is not None or offsets is not None):
            raise PscError("positions: of rows, or first and offsets of sequences")
        if first is not None:
            batch = first.shape[0] if first.dim() == 1 else 0
        elif offsets is not None:
            batch = offsets.shape[0] - 1 if offsets.dim() == 1 else 0
        if batch < 1:
            raise PscError("first, offsets: expected [batch] and [batch + 1]")
        if (rows | heads | dim | batch) >> 31:
            raise PscError(f"x, first, offsets: {rows} rows of {heads} heads of {dim} and {batch} sequences do not fit 32 bits")
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            to = heads * dim, dim
        else:
            if out.shape != shape or out.dtype is not x.dtype or out.get_device() != index or out.stride(-1) != 1:
                raise PscError(f"out: expected {x.dtype} {list(shape)} on {self.device} with contiguous coordinates")
            to = out.stride(0), out.stride(1) if heads > 1 else 0
        _check(_load().psc_rotary_rows(self._struct, transposed, code, x.data_ptr(), row_stride, head_stride, rows, heads, dim,
                                       _array(positions, torch.int32, (rows,), "positions", index), batch,
                                       _array(offsets, torch.int32, (batch + 1,), "offsets", index),
                                       _array(first, torch.int32, (batch,), "first", index), out.data_ptr(), *to, stream))
        return out


class _Turned(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, rotary, positions, first, offsets):
        ctx.rotary = rotary
        ctx.save_for_backward(positions, first, offsets)
        return rotary._turn(x, positions, first, offsets, None, False)

    @_once
    def backward(ctx, dy):
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        return ctx.rotary._turn(dy, *ctx.saved_tensors, None, True), None, None, None, None


# ------------------------------------------------------------------------------------------- norms around a block
_ACTIVATIONS = {"none": 0, None: 0, "sigmoid": 1, "silu": 2}


def _struct_of(x, y, gate, after, before, numbers):
    """The call's struct; what it points to has been checked."""
    some = y if x is None else x
    rows, width = some.shape
    weights = after if after is not None else before
    block = some if y is None else y
    x_at, x_stride = (0, 0) if x is None else (x.data_ptr(), x.stride(0))
    y_at, y_stride = (0, 0) if y is None else (y.data_ptr(), y.stride(0))
    gate_at, gate_stride, gate_rows = (0, 0, 0) if gate is None else (gate.data_ptr(), gate.stride(0), gate.shape[0])
    activation, *scales = numbers
    try:
        return _pack(rows, width, _DTYPES[some.dtype], _DTYPES[block.dtype], _DTYPES[torch.float32 if weights is None else weights.dtype],
                     x_at, x_stride, y_at, y_stride, gate_at, gate_stride, gate_rows, activation, 0 if after is None else after.data_ptr(),
                     0 if before is None else before.data_ptr(), *scales)
    except (struct.error, OverflowError) as e:
        raise PscError(f"x [{rows}, {width}], scales {scales}: {e}") from None


def _forward(x, y, gate, after, before, numbers, want_h, want_stat):
    some = y if x is None else x
    norm = _struct_of(x, y, gate, after, before, numbers)
    h = torch.empty_like(some, memory_format=torch.contiguous_format) if want_h else None
    z = stat = None
    if before is not None:
        z = torch.empty_like(some if y is None else y, memory_format=torch.contiguous_format)
    if want_stat:
        stat = torch.empty((some.shape[0], 2), dtype=torch.float32, device=some.device)
    _check(_load().psc_residual_norm_forward(norm, h.data_ptr() if want_h else None, None if z is None else z.data_ptr(),
                                             stat.data_ptr() if want_stat else None, _current(some.get_device(), "x")))
    return h, z, stat


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, gate, after, before, numbers, want_h):
        h, z, stat = _forward(x, y, gate, after, before, numbers, want_h, True)
        ctx.numbers = numbers
        ctx.save_for_backward(x, y, gate, after, before, stat)
        ctx.set_materialize_grads(False)
        return h, z

    @_once
    def backward(ctx, dh, dz):
        *given, stat = ctx.saved_tensors
        wanted = ctx.needs_input_grad
        if stat.shape[0] == 0:
            return (*(torch.zeros_like(t) if w else None for t, w in zip(given, wanted)), None, None)
        norm, lib = _struct_of(*given, ctx.numbers), _load()
        if dh is not None and not dh.is_contiguous():
            dh = dh.contiguous()
        if dz is not None and not dz.is_contiguous():
            dz = dz.contiguous()
        grads = [torch.empty_like(t, memory_format=torch.contiguous_format) if w else None for t, w in zip(given, wanted)]
        need = lib.psc_residual_norm_workspace_bytes(norm)
        space = _workspace(need, stat.device)
        _check(lib.psc_residual_norm_backward(norm, stat.data_ptr(), *(None if t is None else t.data_ptr() for t in (dh, dz, *grads)), space.data_ptr(),
                                              need, _current(stat.get_device(), "x")))
        return (*grads, None, None)


def _rows_of(t, width, dtype, name, device):
    """t as [rows, width] with contiguous coordinates, one stride apart."""
    if t.dtype is not dtype or t.get_device() != device or t.dim() < 1 or t.shape[-1] != width:
        raise PscError(f"{name}: expected {dtype} [..., {width}] on cuda:{device}, got {t.dtype} {list(t.shape)} on {t.device}")
    if t.dim() != 2:
        try:
            t = t.view(-1, width)
        except RuntimeError:
            raise PscError(f"{name}: rows must lie at one stride, got strides {list(t.stride())}") from None
    if width > 1 and t.stride(1) != 1:
        raise PscError(f"{name}: expected contiguous coordinates, got strides {list(t.stride())}")
    return t


def residual_norm(x, y=None, *, gate=None, activation="none", after=None, before=None, residual_scale=1.0, block_scale=1.0, eps=1e-6):
    """Norms before and after a block with its gate and residual scale, in one pass: (h, z) of a residual stream x and a
    block's output y, both [..., width],
        u = rms(y) * after * act(gate)        rms(t) = t / sqrt(mean t^2 + eps)
        h = residual_scale * x + block_scale * u        z = rms(h) * before
    `after`, `before` [width] (None: no such norm; without `before` z is None), `gate` (None: none) of y's rows, or with
    fewer rows [rows', width] of which each serves rows / rows' consecutive ones, through `activation` ("none", "sigmoid",
    "silu").  x or y may be None.  h has x's type (float32, or y's), z and the gate y's (without y: x's).  Without y and with residual_scale 1 h is x.
    Differentiable in all tensors, backwards and once (tensors that carry a tangent are refused)."""
    if _duals._current_level >= 0:
        _no_tangents(x, y, gate, after, before)
    some = y if x is None else x
    if some is None:
        raise PscError("x and y are None")
    code, device = _ACTIVATIONS.get(activation), some.get_device()
    if code is None:
        raise PscError(f"activation: expected \"none\", \"sigmoid\" or \"silu\", got {activation!r}")
    if device < 0 or some.dim() < 1:
        raise PscError(f"x: expected CUDA tensors [..., width], got {list(some.shape)} on {some.device}")
    _dtype(some, "x")
    shape, width = some.shape, some.shape[-1]
    kind = some.dtype
    plain = y is None and residual_scale == 1.0
    if x is not None:
        x2 = _rows_of(x, width, kind, "x", device)
    else:
        x2 = None
    if y is None:
        if gate is not None or after is not None:
            raise PscError("gate, after: without y")
        y2 = None
    else:
        if y.shape != shape:
            raise PscError(f"y: expected {list(shape)}, got {list(y.shape)}")
        if kind is not torch.float32 and y.dtype is not kind:
            raise PscError(f"x: expected float32 or y's {y.dtype}, got {kind}")
        kind = y.dtype
        _dtype(y, "y")
        y2 = _rows_of(y, width, kind, "y", device)
    if gate is not None:
        gate = _rows_of(gate, width, kind, "gate", device)
        rows, gates = y2.shape[0], gate.shape[0]
        if rows and (gates == 0 or rows % gates):
            raise PscError(f"gate: {rows} rows are no multiple of {gates}")
    weights = after if after is not None else before
    if weights is not None:
        if weights.dtype is not torch.float32 and weights.dtype is not kind:
            raise PscError(f"after, before: expected float32 or {kind}, got {weights.dtype}")
        _array(after, weights.dtype, (width,), "after", device)
        _array(before, weights.dtype, (width,), "before", device)
    if plain and before is None:
        return x, None
    numbers = (code, residual_scale, block_scale, eps)
    if torch.is_grad_enabled() and any([t is not None and t.requires_grad for t in (x2, y2, gate, after, before)]):
        h, z = _ResidualNorm.apply(x2, y2, gate, after, before, numbers, not plain)
    else:
        h, z, _ = _forward(x2, y2, gate, after, before, numbers, not plain, False)
    if len(shape) != 2:
        h, z = None if h is None else h.view(shape), None if z is None else z.view(shape)
    return x if plain else h, z
