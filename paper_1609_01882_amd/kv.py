"""Attention memory held in 4 bits: argument marshalling for the `psc_kv_*` calls (see `include/psc.h`).

    cache = psc.KvCache.empty(pages=4096, kv_heads=8, head_dim=128, page=64)
    cache.append(k, v, table, lengths)                      # new tokens, rounded to 4 bits
    lengths += 1
    out, lse = cache.attend(q, table, lengths, weights=w, weights_out=w)
    cache.evict(table, lengths, w, budget=4096, sinks=4, recent=512, ...)

Sequences are rows of `table` [batch, width] (int32, page numbers, negative: none) with `lengths` [batch] (int32)
tokens each.  Rows of several sequences lie one after another, `offsets` [batch + 1] (int32) says where each begins;
without it every sequence has the same number.  Arrays per slot are [batch, kv_heads, width * page].
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct
import types

import torch
from torch.autograd import forward_ad

from .binding import PscError, _check, _load, _workspace

PSC_BF16, PSC_F16, PSC_F32 = 0, 1, 2
_DTYPES = {torch.bfloat16: PSC_BF16, torch.float16: PSC_F16, torch.float32: PSC_F32}


# The address of a device's current stream: 0.1 us where torch has a function that gives it alone, 1.1 through a stream object.
_stream_address = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


# Where torch says whether tensors may carry tangents (a level below 0: none does), so that calls without any ask nothing else.
_duals = forward_ad if hasattr(forward_ad, "_current_level") else types.SimpleNamespace(_current_level=0)


def _no_tangents(*tensors):
    """Refuses tensors that carry a tangent: these calls have no forward-mode derivatives, and would drop it without a word."""
    if any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise PscError("a tensor carries a tangent, and there are no forward-mode derivatives here: take its primal, or differentiate backwards where that is offered")


class _Cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("pages", C.c_int64), ("kv_heads", C.c_int), ("head_dim", C.c_int), ("page", C.c_int), ("table", C.c_void_p),
                ("batch", C.c_int), ("table_width", C.c_int), ("lengths", C.c_void_p)]


_pack = struct.Struct("@4Pq3iP2iP").pack     # the same fields, packed at once: a call of a few microseconds notices
assert struct.calcsize("@4Pq3iP2iP") == C.sizeof(_Cache)


def _array(t, dtype, shape, name, device):
    """Address of a dense tensor of this type and shape on the device (its index); None: a null pointer."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise PscError(f"{name}: expected a contiguous {dtype} tensor of shape {list(shape)} on cuda:{device}, "
                       f"got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _bytes(t, device):
    if t.dtype is not torch.uint8 or t.get_device() != device or not t.is_contiguous():
        raise PscError(f"workspace: expected a contiguous uint8 tensor on cuda:{device}")
    return t.data_ptr(), t.numel()


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise PscError(f"{name}: expected bfloat16, float16 or float32, got {t.dtype}")
    return code


def _ints(**values):
    for name, x in values.items():
        if not -(1 << 31) <= x < 1 << 31:
            raise PscError(f"{name}: {x} does not fit 32 bits")


@functools.lru_cache(maxsize=1024)
def _attention_workspace(call, pages, kv_heads, head_dim, page, batch, width, dtype, rows, max_rows, q_heads, window, sinks, *has):
    sizes = dict(rows=rows, max_rows=max_rows, q_heads=q_heads, window=window, sinks=sinks)
    _ints(batch=batch, width=width, **sizes)
    sizes = dtype, *sizes.values(), *has
    return getattr(_load(), call + "_workspace_bytes")(_pack(0, 0, 0, 0, pages, kv_heads, head_dim, page, 0, batch, width, 0), *sizes)


class KvCache:
    """Keys and values of sequences as 4-bit floats in pages.  Borrows the four buffers (`empty` makes them):
    codes [pages, kv_heads, page, head_dim / 2], scales [pages, kv_heads, page, head_dim / 32], uint8."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        for t, name in ((k_codes, "k_codes"), (k_scales, "k_scales"), (v_codes, "v_codes"), (v_scales, "v_scales")):
            if not (t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous() and t.dim() == 4):
                raise PscError(f"{name}: expected a contiguous CUDA tensor of uint8 with 4 dimensions")
        if k_codes.shape[-1] % 16 or k_codes.shape != v_codes.shape or k_scales.shape != v_scales.shape or \
                k_scales.shape != (*k_codes.shape[:3], k_codes.shape[3] // 16) or \
                len({t.device for t in (k_codes, k_scales, v_codes, v_scales)}) != 1:
            raise PscError("codes [pages, kv_heads, page, head_dim / 2] and scales [pages, kv_heads, page, head_dim / 32] do not match")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.pages, self.kv_heads, self.page, self.head_dim = *k_codes.shape[:3], 2 * k_codes.shape[3]
        self.device, self._index = k_codes.device, k_codes.get_device()

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda"):
        """A cache of its own, all slots zero."""
        make = lambda per: torch.zeros((pages, kv_heads, page, head_dim // per), dtype=torch.uint8, device=device)  # noqa: E731
        return cls(make(2), make(32), make(2), make(32))

    def _args(self, table, lengths, what="lengths"):
        if table.dim() != 2:
            raise PscError(f"table: expected [batch, width], got {list(table.shape)}")
        batch, width = table.shape
        c = _pack(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(), self.v_scales.data_ptr(), self.pages,
                  self.kv_heads, self.head_dim, self.page, _array(table, torch.int32, (batch, width), "table", self._index), batch, width,
                  _array(lengths, torch.int32, (batch,), what, self._index) or 0)
        return c, batch, (batch, self.kv_heads, width * self.page)

    def _rows(self, t, heads, name):
        """Address and strides of rows [n, heads, head_dim]."""
        if t.dim() != 3 or t.shape[1:] != (heads, self.head_dim) or t.get_device() != self._index or t.stride(2) != 1:
            raise PscError(f"{name}: expected [rows, {heads}, {self.head_dim}] on {self.device} with contiguous coordinates, "
                           f"got {list(t.shape)} with strides {list(t.stride())} on {t.device}")
        return t.data_ptr(), t.stride(0), t.stride(1)

    def _stream(self):
        if torch.cuda.current_device() != self._index:
            raise PscError(f"the cache is on {self.device}, the current device is cuda:{torch.cuda.current_device()}")
        return _stream_address(self._index)

    def append(self, k, v, table, lengths, offsets=None, first=None, positions=None, weights=None, rotary=None, q=None, q_out=None):
        """Round the rows k, v [n, kv_heads, head_dim] to 4 bits and write them to slots lengths[b], lengths[b] + 1, ...
        `lengths` stays as it is.  `positions`, per slot (int32), receives first[b], first[b] + 1, ... (`first` None: the
        slots); `weights`, per slot (float32), receives 0.
        `rotary` (a `Rotary`, of a multiple of 16 dimensions): keys are turned first, row r of a sequence by the angles of first[b] + r, and so
        are the queries q [n, q_heads, head_dim] of the same rows, which are returned (in `q_out`, another tensor than q).
        Nothing flows back or forward: tensors that want a gradient or carry a tangent are refused then."""
        c, batch, slots = self._args(table, lengths)
        if k.dim() != 3 or v.dtype != k.dtype or v.shape != k.shape:
            raise PscError(f"k, v: expected [rows, {self.kv_heads}, {self.head_dim}] of one type, got {k.dtype} {list(k.shape)} and {v.dtype} {list(v.shape)}")
        n = k.shape[0]
        if n >> 31:
            _ints(rows=n)
        if rotary is not None:
            return self._append_rotary(c, batch, slots, k, v, offsets, first, positions, weights, rotary, q, q_out)
        if q is not None or q_out is not None:
            raise PscError("q: is turned by a rotary, and there is none")
        _check(_load().psc_kv_append(c, _dtype(k, "k"), *self._rows(k, self.kv_heads, "k"), *self._rows(v, self.kv_heads, "v"), n,
                                     _array(offsets, torch.int32, (batch + 1,), "offsets", self._index),
                                     _array(first, torch.int32, (batch,), "first", self._index),
                                     _array(positions, torch.int32, slots, "positions", self._index),
                                     _array(weights, torch.float32, slots, "weights", self._index), self._stream()))

    def _append_rotary(self, c, batch, slots, k, v, offsets, first, positions, weights, rotary, q, q_out):
        n, heads, device = k.shape[0], 0, self._index
        if rotary._index != device:
            raise PscError(f"rotary: expected on {self.device}, got {rotary.device}")
        if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (k, v, q, q_out)):
            raise PscError("k, v, q: what goes into a memory in 4 bits has no gradient; detach, or call under torch.no_grad()")
        if _duals._current_level >= 0:
            _no_tangents(k, v, q, q_out)
        rows, to = (None, 0, 0), None
        if q is not None:
            heads = q.shape[1] if q.dim() == 3 else 0
            if heads < 1 or q.dtype != k.dtype or q.shape[0] != n:
                raise PscError(f"q: expected {k.dtype} [{n}, q_heads, {self.head_dim}], got {q.dtype} {list(q.shape)}")
            rows = self._rows(q, heads, "q")
            if q_out is None:
                q_out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=self.device)
            to = _array(q_out, q.dtype, (n, heads, self.head_dim), "q_out", device)
        elif q_out is not None:
            raise PscError("q_out: without q")
        _check(_load().psc_kv_append_rotary(c, rotary._struct, _dtype(k, "k"), *self._rows(k, self.kv_heads, "k"),
                                            *self._rows(v, self.kv_heads, "v"), *rows, heads, to, n,
                                            _array(offsets, torch.int32, (batch + 1,), "offsets", device),
                                            _array(first, torch.int32, (batch,), "first", device),
                                            _array(positions, torch.int32, slots, "positions", device),
                                            _array(weights, torch.float32, slots, "weights", device), self._stream()))
        return q_out

    def read(self, table, starts, rows: int, offsets=None, dtype=torch.float32):
        """The held values of the slots starts[b], starts[b] + 1, ... (`rows` of them altogether): k, v [rows, kv_heads,
        head_dim]."""
        c, batch, _ = self._args(table, starts, "starts")
        k = torch.empty((rows, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        _check(_load().psc_kv_read(c, _dtype(k, "dtype"), rows, _array(offsets, torch.int32, (batch + 1,), "offsets", self._index),
                                   k.data_ptr(), v.data_ptr(), self._stream()))
        return k, v

    def attend(self, q, table, lengths, offsets=None, max_rows=None, first=None, positions=None, scale=None, causal=True, window=0,
               sinks=0, weights=None, weights_out=None, out=None, workspace=None):
        """Attention of the rows q [n, q_heads, head_dim]: (out, lse), [n, q_heads, head_dim] and [n, q_heads].
        The rows of a sequence are its last tokens, or stand at first[b], first[b] + 1, ...  `max_rows`: no sequence has
        more rows (with `offsets`; None: n).  `window` > 0: rows see that many positions back from their own, and the
        positions below `sinks`.  `scale` None: 1 / sqrt(head_dim).  `weights_out`, per slot (float32), receives
        `weights` (None: 0) plus the weight that each token was given; they may be the same tensor.  Nothing flows back:
        a `q` that wants a gradient, or carries a tangent, is refused."""
        return self._attend("psc_kv_attention", (self.head_dim, 1), None, q, table, lengths, offsets, max_rows, first, positions, scale, causal,
                            window, sinks, weights, weights_out, out, workspace)

    def attend_difference(self, q, lam, table, lengths, offsets=None, max_rows=None, first=None, positions=None, scale=None, causal=True, window=0,
                          sinks=0, norm=None, eps=1e-6, factor=1.0, weights=None, weights_out=None, out=None, workspace=None):
        """Differential attention of the rows q [n, q_heads, head_dim]: (out, lse), [n, q_heads / 2, 2 head_dim] and [n, q_heads].
        kv heads 2j and 2j + 1 are a pair: a map of each one's keys, both over the two heads' values side by side.  With g
        query heads to a kv head, output head j * g + i is softmax(q1 K1) V - lam softmax(q2 K2) V of the query heads
        2j * g + i and (2j + 1) * g + i, with `norm` [2 head_dim] (float32) divided by the root of its mean square plus
        `eps` and multiplied by `norm`; then by `factor`.  `lam` (float32): [q_heads / 2], or [n, q_heads / 2] for each row.
        `positions` of a pair's heads are alike (the even one's are read); both receive both maps' weights.  head_dim is
        64 or 128, kv_heads even.  16-bit rows' probabilities are rounded to 11 bits in both maps, however little the difference leaves of
        them (float32 rows: 22).  All else as for `attend`; nothing flows back.  Single tokens over long memories are faster in a call of their own than
        beside a sequence of hundreds of rows."""
        heads = q.shape[1] if q.dim() == 3 else 0
        if self.kv_heads % 2 or self.head_dim > 128 or heads < 1 or heads % self.kv_heads:
            raise PscError(f"differential attention takes pairs of kv heads of 64 or 128 and a multiple of {self.kv_heads} query heads, got {heads} over "
                           f"{self.kv_heads} x {self.head_dim}")
        n = q.shape[0]
        if lam.dim() == 1:
            row = 0
            at = _array(lam, torch.float32, (heads // 2,), "lam", self._index)
        else:
            row = lam.stride(0) if lam.dim() else 0
            if lam.shape != (n, heads // 2) or lam.dtype != torch.float32 or lam.get_device() != self._index or (heads > 2 and lam.stride(1) != 1):
                raise PscError(f"lam: expected float32 [{heads // 2}] or [{n}, {heads // 2}] on {self.device} with contiguous heads, got {lam.dtype} "
                               f"{list(lam.shape)} with strides {list(lam.stride())} on {lam.device}")
            at = lam.data_ptr()
        if torch.is_grad_enabled() and (lam.requires_grad or (norm is not None and norm.requires_grad)):
            raise PscError("lam, norm: attention over a memory in 4 bits has no gradient; detach them, or call under torch.no_grad()")
        if _duals._current_level >= 0:
            _no_tangents(lam, norm)
        more = at, row, _array(norm, torch.float32, (2 * self.head_dim,), "norm", self._index), eps, factor
        return self._attend("psc_kv_difference", (2 * self.head_dim, 2), more, q, table, lengths, offsets, max_rows, first, positions, scale, causal,
                            window, sinks, weights, weights_out, out, workspace)

    def _attend(self, call, shape, more, q, table, lengths, offsets, max_rows, first, positions, scale, causal, window, sinks, weights, weights_out,
                out, workspace):
        """`shape`: width of an output head, and how many query heads it takes; `more`: what the call takes behind the sinks."""
        c, batch, slots = self._args(table, lengths)
        n, heads = (q.shape[0], q.shape[1]) if q.dim() == 3 else (0, 0)
        code, device = _dtype(q, "q"), self._index
        rows = self._rows(q, heads, "q")
        if offsets is None:
            max_rows = n // max(batch, 1)
        elif max_rows is None:
            max_rows = n
        if (n | max_rows | window | sinks) >> 31:   # (negative ones too: the call says what is wrong with them)
            _ints(rows=n, max_rows=max_rows, window=window, sinks=sinks)
        if q.requires_grad and torch.is_grad_enabled():
            raise PscError("q: attention over a memory in 4 bits has no gradient; detach q, or call under torch.no_grad()")
        if _duals._current_level >= 0:
            _no_tangents(q)
        outs = (n, heads // shape[1], shape[0])
        if out is None:
            out = (torch.empty(outs, dtype=q.dtype, device=self.device),
                   torch.empty((n, heads), dtype=torch.float32, device=self.device))
        space = None, 0
        if workspace is not None:
            space = _bytes(workspace, device)
        else:
            need = _attention_workspace(call, self.pages, self.kv_heads, self.head_dim, self.page, batch, table.shape[1], code, n, max_rows, heads,
                                        window, sinks, positions is not None, weights_out is not None)
            if need:
                workspace = _workspace(need, self.device)
                space = workspace.data_ptr(), need
        _check(getattr(_load(), call)(c, code, *rows, n, max_rows, heads,
                                      _array(offsets, torch.int32, (batch + 1,), "offsets", device),
                                      _array(first, torch.int32, (batch,), "first", device),
                                      _array(positions, torch.int32, slots, "positions", device),
                                      1.0 / math.sqrt(self.head_dim) if scale is None else scale, int(causal), window, sinks,
                                      *(more or ()),
                                      _array(out[0], q.dtype, outs, "out", device),
                                      _array(out[1], torch.float32, (n, heads), "lse", device),
                                      _array(weights, torch.float32, slots, "weights", device),
                                      _array(weights_out, torch.float32, slots, "weights_out", device),
                                      *space, self._stream()))
        return out

    def attend_workspace_bytes(self, batch: int, width: int, rows: int, max_rows: int, q_heads: int, dtype, window: int = 0, sinks: int = 0,
                               positions: bool = False, weights: bool = False) -> int:
        """What `attend` needs for `rows` rows, at most `max_rows` of a sequence, over tables [batch, width]; `positions` and
        `weights`: whether there are positions and weights_out."""
        return int(_attention_workspace("psc_kv_attention", self.pages, self.kv_heads, self.head_dim, self.page, batch, width, _DTYPES[dtype], rows,
                                        max_rows, q_heads, window, sinks, positions, weights))

    def attend_difference_workspace_bytes(self, batch: int, width: int, rows: int, max_rows: int, q_heads: int, dtype, window: int = 0,
                                          sinks: int = 0, positions: bool = False, weights: bool = False) -> int:
        """What `attend_difference` needs, as for `attend`."""
        return int(_attention_workspace("psc_kv_difference", self.pages, self.kv_heads, self.head_dim, self.page, batch, width, _DTYPES[dtype], rows,
                                        max_rows, q_heads, window, sinks, positions, weights))

    def evict_workspace_bytes(self, batch: int, width: int, budget: int) -> int:
        _ints(batch=batch, width=width, budget=budget)
        return int(_load().psc_kv_evict_workspace_bytes(_pack(0, 0, 0, 0, self.pages, self.kv_heads, self.head_dim, self.page, 0, batch, width, 0), budget))

    def evict(self, table, lengths, weights, budget: int, sinks: int = 0, recent: int = 0, positions=None, seen=None, out=None, workspace=None):
        """Cut every sequence's heads to the `budget` tokens of the largest `weights` (per slot), the tokens at positions
        below `sinks` and the `recent` last ones of the `seen` [batch] (None: lengths) always among them.  Returns
        (kept, lengths, positions, weights): the slot each kept token had [batch, kv_heads, budget], and the state after;
        `out`: those four, where `lengths`, `positions` and `weights` may be the tensors passed in."""
        c, batch, slots = self._args(table, lengths)
        device, lib = self._index, _load()
        _ints(budget=budget, sinks=sinks, recent=recent)
        if out is None:
            shape = (batch, self.kv_heads, budget)
            whole = torch.empty((2, *shape), dtype=torch.int32, device=self.device)
            out = (whole[0], torch.empty(batch, dtype=torch.int32, device=self.device), whole[1],
                   torch.empty(shape, dtype=torch.float32, device=self.device))
        kept, lengths_out, positions_out, weights_out = out
        wide = weights_out.shape
        if len(wide) != 3 or wide[:2] != slots[:2]:
            raise PscError(f"weights (out): expected [{slots[0]}, {slots[1]}, {budget} or more], got {list(wide)}")
        if workspace is None:
            workspace = _workspace(lib.psc_kv_evict_workspace_bytes(c, budget), self.device)
        _check(lib.psc_kv_evict(c, _array(weights, torch.float32, slots, "weights", device),
                                _array(positions, torch.int32, slots, "positions", device),
                                _array(seen, torch.int32, (batch,), "seen", device), budget, sinks, recent,
                                _array(kept, torch.int32, (batch, self.kv_heads, budget), "kept", device),
                                _array(lengths_out, torch.int32, (batch,), "lengths (out)", device),
                                _array(positions_out, torch.int32, wide, "positions (out)", device),
                                _array(weights_out, torch.float32, wide, "weights (out)", device), wide[2],
                                *_bytes(workspace, device), self._stream()))
        return out
