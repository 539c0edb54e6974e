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

import torch

from .binding import PscError, _check, _load, _workspace
from .kv import _DTYPES, PSC_F32, _array, _dtype, _ints, _stream_address


class _Rotary(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("dims", C.c_int), ("interleaved", C.c_int), ("factor", C.c_float)]


class _Norm(C.Structure):
    _fields_ = [("rows", C.c_int), ("width", C.c_int), ("stream_dtype", C.c_int), ("block_dtype", C.c_int), ("weight_dtype", C.c_int),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("y", C.c_void_p), ("y_stride", C.c_int64), ("gate", C.c_void_p),
                ("gate_stride", C.c_int64), ("gate_rows", C.c_int), ("activation", C.c_int), ("after", C.c_void_p), ("before", C.c_void_p),
                ("residual_scale", C.c_float), ("block_scale", C.c_float), ("eps", C.c_float)]


def _current(index, what):
    if torch.cuda.current_device() != index:
        raise PscError(f"{what} is on cuda:{index}, the current device is cuda:{torch.cuda.current_device()}")
    return _stream_address(index)


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
        if not math.isfinite(factor):
            raise PscError("factor must be finite")
        turns = (C.c_uint64 * (dims // 2))()
        _check(_load().psc_rotary_turns((C.c_double * (dims // 2))(*frequencies), dims // 2, turns))
        self.dims, self.interleaved, self.factor, self.frequencies = dims, bool(interleaved), float(factor), frequencies
        signed = [t - (1 << 64) if t >> 63 else t for t in turns]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.device, self._index = self.turns.device, self.turns.get_device()
        self._struct = _Rotary(self.turns.data_ptr(), dims, self.interleaved, self.factor)

    def __call__(self, x, positions=None, first=None, offsets=None, out=None):
        """x [rows, heads, head_dim] (or [rows, head_dim]) turned: row r at positions[r] (int32), or at first[b] + its place in
        its sequence b, [batch] (int32; `offsets` [batch + 1]: where sequences begin, None: equal parts), or at r.
        Rows that no sequence has are copied.  Differentiable in x; `out` (which may be x): written, and no gradient."""
        if out is None and x.requires_grad and torch.is_grad_enabled():
            return _Turned.apply(x, self, positions, first, offsets)
        if out is not None and torch.is_grad_enabled() and (x.requires_grad or out.requires_grad):
            raise PscError("out: has no gradient; detach x, or call under torch.no_grad()")
        return self._turn(x, positions, first, offsets, out, False)

    def inverse(self, x, positions=None, first=None, offsets=None, out=None):
        """The transposed: turned back, times the factor (with factor 1 the inverse).  Nothing flows back."""
        if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
            raise PscError("x: the transposed has no gradient; detach x, or call under torch.no_grad()")
        return self._turn(x, positions, first, offsets, out, True)

    def _turn(self, x, positions, first, offsets, out, transposed):
        stream = _current(self._index, "the rotary")
        code = _dtype(x, "x")
        whole = x.unsqueeze(1) if x.dim() == 2 else x
        if whole.dim() != 3 or x.get_device() != self._index or whole.shape[2] < self.dims or whole.stride(2) != 1:
            raise PscError(f"x: expected [rows, heads, head_dim >= {self.dims}] on {self.device} with contiguous coordinates, got {list(x.shape)} "
                           f"with strides {list(x.stride())} on {x.device}")
        rows, heads, dim = whole.shape
        batch = 1
        if positions is not None and (first is not None or offsets is not None):
            raise PscError("positions: of rows, or first and offsets of sequences")
        if first is not None:
            batch = first.shape[0] if first.dim() == 1 else 0
        elif offsets is not None:
            batch = offsets.shape[0] - 1 if offsets.dim() == 1 else 0
        if batch < 1:
            raise PscError("first, offsets: expected [batch] and [batch + 1]")
        if out is None:
            out = torch.empty((rows, heads, dim) if x.dim() == 3 else (rows, dim), dtype=x.dtype, device=x.device)
        to = out.unsqueeze(1) if out.dim() == 2 and x.dim() == 2 else out
        if to.shape != whole.shape or to.dtype != x.dtype or to.get_device() != self._index or to.stride(2) != 1:
            raise PscError(f"out: expected {x.dtype} {list(x.shape)} on {self.device} with contiguous coordinates")
        _ints(rows=rows, heads=heads, head_dim=dim)
        _check(_load().psc_rotary_rows(C.byref(self._struct), int(transposed), code, whole.data_ptr(), whole.stride(0), whole.stride(1), rows, heads, dim,
                                       _array(positions, torch.int32, (rows,), "positions", self._index), batch,
                                       _array(offsets, torch.int32, (batch + 1,), "offsets", self._index),
                                       _array(first, torch.int32, (batch,), "first", self._index),
                                       to.data_ptr(), to.stride(0), to.stride(1), stream))
        return out


class _Turned(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, rotary, positions, first, offsets):
        ctx.rotary = rotary
        ctx.save_for_backward(positions, first, offsets)
        return rotary._turn(x, positions, first, offsets, None, False)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        return ctx.rotary._turn(dy, *ctx.saved_tensors, None, True), None, None, None, None


# ------------------------------------------------------------------------------------------- norms around a block
_ACTIVATIONS = {"none": 0, None: 0, "sigmoid": 1, "silu": 2}


def _matrix(t, dtype, rows, width, name, device):
    """Address and row stride of [rows, width] with contiguous coordinates."""
    if t is None:
        return None, 0
    if t.dim() != 2 or t.shape[1] != width or (rows is not None and t.shape[0] != rows) or t.dtype != dtype or t.get_device() != device or \
            (width > 1 and t.stride(1) != 1):
        raise PscError(f"{name}: expected {dtype} [{'rows' if rows is None else rows}, {width}] on cuda:{device} with contiguous coordinates, got "
                       f"{t.dtype} {list(t.shape)} with strides {list(t.stride())} on {t.device}")
    return t.data_ptr(), t.stride(0)


def _norm_struct(x, y, gate, after, before, activation, residual_scale, block_scale, eps):
    some = y if x is None else x
    device, (rows, width) = some.get_device(), some.shape
    block = (y if y is not None else x).dtype
    weights = after if after is not None else before
    weight = torch.float32 if weights is None else weights.dtype
    x_at, x_stride = _matrix(x, some.dtype, rows, width, "x", device)
    y_at, y_stride = _matrix(y, block, rows, width, "y", device)
    gate_at, gate_stride = _matrix(gate, block, None, width, "gate", device)
    if gate is not None and (gate.shape[0] == 0 or rows % gate.shape[0]) and rows:
        raise PscError(f"gate: {rows} rows are no multiple of {gate.shape[0]}")
    after_at = _array(after, weight, (width,), "after", device)
    before_at = _array(before, weight, (width,), "before", device)
    _ints(rows=rows, width=width)
    return _Norm(rows, width, _DTYPES[some.dtype], _DTYPES[block], _DTYPES.get(weight, PSC_F32), x_at, x_stride, y_at, y_stride, gate_at, gate_stride,
                 0 if gate is None else gate.shape[0], activation, after_at, before_at, residual_scale, block_scale, eps)


def _forward(x, y, gate, after, before, numbers, want_h, want_stat):
    n = _norm_struct(x, y, gate, after, before, *numbers)
    some = y if x is None else x
    stream = _current(some.get_device(), "x")
    h = torch.empty(some.shape, dtype=some.dtype, device=some.device) if want_h else None
    z = torch.empty(some.shape, dtype=(y if y is not None else x).dtype, device=some.device) if before is not None else None
    stat = torch.empty((n.rows, 2), dtype=torch.float32, device=some.device) if want_stat else None
    _check(_load().psc_residual_norm_forward(C.byref(n), None if h is None else h.data_ptr(), None if z is None else z.data_ptr(),
                                             None if stat is None else stat.data_ptr(), stream))
    return h, z, stat


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, gate, after, before, numbers, want_h):
        h, z, stat = _forward(x, y, gate, after, before, numbers, want_h, True)
        ctx.numbers = numbers
        ctx.save_for_backward(x, y, gate, after, before, stat)
        ctx.set_materialize_grads(False)
        return h, z

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dz):
        x, y, gate, after, before, stat = ctx.saved_tensors
        given = (x, y, gate, after, before)
        n = _norm_struct(*given, *ctx.numbers)
        wanted = ctx.needs_input_grad[:5]
        if n.rows == 0:
            return (*(torch.zeros_like(t) if w else None for t, w in zip(given, wanted)), None, None)
        device = stat.device
        stream = _current(device.index, "x")
        dh, dz = (None if t is None else t.contiguous() for t in (dh, dz))
        grads = [torch.empty(t.shape, dtype=t.dtype, device=device) if w else None for t, w in zip(given, wanted)]
        lib = _load()
        need = lib.psc_residual_norm_workspace_bytes(C.byref(n))
        space = _workspace(need, device)
        at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        _check(lib.psc_residual_norm_backward(C.byref(n), stat.data_ptr(), at(dh), at(dz), *map(at, grads), space.data_ptr(), need, stream))
        return (*grads, None, None)


def residual_norm(x, y=None, *, gate=None, activation="none", after=None, before=None, residual_scale=1.0, block_scale=1.0, eps=1e-6):
    """Norms before and after a block with its gate and residual scale, in one pass: (h, z) of a residual stream x and a
    block's output y, both [..., width],
        u = rms(y) * after * act(gate)        rms(t) = t / sqrt(mean t^2 + eps)
        h = residual_scale * x + block_scale * u        z = rms(h) * before
    `after`, `before` [width] (None: no such norm; without `before` z is None), `gate` (None: none) of y's rows, or with
    fewer rows [rows', width] of which each serves rows / rows' consecutive ones, through `activation` ("none", "sigmoid",
    "silu").  x or y may be None.  h has x's type (float32, or y's), z and the gate y's.  Without y and with residual_scale 1 h is x.
    Differentiable in all tensors."""
    some = y if x is None else x
    if some is None:
        raise PscError("x and y are None")
    if y is None and (gate is not None or after is not None):
        raise PscError("gate, after: without y")
    if activation not in _ACTIVATIONS:
        raise PscError(f"activation: expected \"none\", \"sigmoid\" or \"silu\", got {activation!r}")
    if not some.is_cuda or some.dim() < 1:
        raise PscError(f"x: expected CUDA tensors [..., width], got {list(some.shape)} on {some.device}")
    if x is not None and y is not None and x.shape != y.shape:
        raise PscError(f"y: expected {list(x.shape)}, got {list(y.shape)}")
    for t, name in ((x, "x"), (y, "y")):
        if t is not None:
            _dtype(t, name)
    if x is not None and y is not None and x.dtype not in (torch.float32, y.dtype):
        raise PscError(f"x: expected float32 or y's {y.dtype}, got {x.dtype}")
    for t, name in ((after, "after"), (before, "before")):
        if t is not None and t.dtype not in (torch.float32, (some if y is None else y).dtype):
            raise PscError(f"{name}: expected float32 or the block's type, got {t.dtype}")
    shape, width = some.shape, some.shape[-1]

    def rows_of(t, name):
        if t is None or t.dim() == 2:
            return t
        try:
            return t.view(-1, width)
        except RuntimeError:
            raise PscError(f"{name}: rows must lie at one stride, got strides {list(t.stride())}") from None

    x2, y2, gate2 = rows_of(x, "x"), rows_of(y, "y"), rows_of(gate, "gate")
    numbers = (_ACTIVATIONS[activation], residual_scale, block_scale, eps)
    plain = y is None and residual_scale == 1.0
    if plain and before is None:
        return x, None
    given = (x2, y2, gate2, after, before)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given):
        h, z = _ResidualNorm.apply(*given, numbers, not plain)
    else:
        h, z, _ = _forward(*given, numbers, not plain, False)
    h = x if plain else h.view(shape)
    return h, None if z is None else z.view(shape)
