"""ChebBooster online stage on AMD MI355X (gfx950).

``libcheb.so`` (C ABI in ``include/cheb.h``) does all the work: fp64 host
weights, the device history ring, the full-step push and the skipped-step
prediction kernel.  This package is its Python face: the C entry points under
their own names (``_binding``) and a small tensor-level wrapper,
``ChebCache``, that takes torch tensors and streams and passes their
addresses through.  PyTorch provides device memory and streams only.
"""
from typing import List, Optional, Sequence

import numpy as np
import torch

from ._binding import (  # noqa: F401  (re-exported C entry points)
    CHEB_LAYOUT_INTERLEAVED, CHEB_LAYOUT_SLOTS, cheb_cache_arena_bytes_ex, cheb_cache_create_ex,
    cheb_cache_geometry, DEFAULT_LAUNCH_CONFIG, CHEB_QUANT_MXFP8, CHEB_QUANT_MXINT8,
    CHEB_QUANT_NONE, cheb_cache_create_quant, cheb_cache_layout_quant, cheb_cache_quant,
    cheb_cache_read, cheb_add_norm, cheb_norm, cheb_residual_norm, CHEB_MAX_NORM_DIM,
    CHEB_NORM_LAYER, CHEB_NORM_RMS, CHEB_OUT_FP8_ROW, CHEB_OUT_MXFP8,
    CHEB_BF16, CHEB_F16, CHEB_F32, CHEB_MAX_NODES, CHEB_MAX_OUTPUTS, CHEB_MAX_SLOTS, CHEB_RHO_ALTERNATING,
    CHEB_RHO_GENERAL, CHEB_SHORT_FULL, CHEB_TAYLOR, CHEB_SHORT_LOWER, ChebError, cheb_chebyshev_nodes,
    cheb_precompute_weights_variant,
    cheb_cache_abort_push, cheb_cache_arena_bytes, cheb_cache_begin_push, cheb_cache_commit, cheb_cache_create,
    cheb_cache_destroy,
    cheb_cache_dtype, cheb_cache_entry, cheb_cache_history, cheb_cache_layout, cheb_cache_push,
    cheb_cache_reset, cheb_cache_segment_offset, cheb_cache_slot_numel, cheb_combine,
    cheb_combine_multi, cheb_extrapolate, cheb_extrapolate_at, cheb_extrapolate_at_multi,
    cheb_extrapolate_multi, cheb_extrapolate_steps, cheb_get_launch_config, cheb_last_error,
    cheb_precompute_weights, cheb_residual_apply, cheb_residual_reduce, cheb_schedule,
    cheb_set_launch_config, cheb_table_build, cheb_table_build_mask,
    cheb_table_destroy, cheb_table_info, cheb_table_load, cheb_table_save, cheb_table_step,
    cheb_version,
)
from . import _binding

LIB_PATH = _binding.LIB_PATH

_DTYPES = {torch.bfloat16: CHEB_BF16, torch.float16: CHEB_F16, torch.float32: CHEB_F32}
_TORCH = {CHEB_BF16: torch.bfloat16, CHEB_F16: torch.float16, CHEB_F32: torch.float32}


def cheb_dtype(dtype: torch.dtype) -> int:
    try:
        return _DTYPES[dtype]
    except KeyError:
        raise ChebError(_binding.CHEB_E_DTYPE, f"unsupported dtype {dtype}") from None


# The current stream's handle without a Stream object around it (0.2 us for
# 1.5), where torch has the call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream: Optional[torch.cuda.Stream], device: Optional[int] = None) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device() if device is None else device)
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _made_for(stream: Optional[torch.cuda.Stream], device, make):
    """Buffers that a call makes itself and fills on `stream`.  They come from
    that stream's pool: a block of the current stream's pool may have been freed
    with work still queued on it, which `stream` does not wait for.  They are
    not handed out again before the current stream, whose program goes on with
    them, is done with them either."""
    if stream is None:
        return make()
    user = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        made = make()
    for t in made if isinstance(made, (tuple, list)) else (made,):
        t.record_stream(user)
    return made


def _check_device_tensor(t: torch.Tensor, what: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ChebError(_binding.CHEB_E_INVAL, f"{what} must be a GPU tensor")
    if not t.is_contiguous():
        raise ChebError(_binding.CHEB_E_INVAL, f"{what} must be contiguous")


def _plain(t, dtype: torch.dtype, numel: int) -> bool:
    """Whether t is a contiguous GPU tensor of that type and size."""
    return (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype
            and t.numel() == numel and t.is_contiguous())


def combine(srcs: Sequence[torch.Tensor], w, out: torch.Tensor,
            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out = sum_k w[k] * srcs[k] (elementwise, one launch of cheb_combine)."""
    if len(srcs) == 0:
        raise ChebError(_binding.CHEB_E_INVAL, "no sources")
    dt = cheb_dtype(out.dtype)
    _check_device_tensor(out, "out")
    dtype, numel = out.dtype, out.numel()
    for i, s in enumerate(srcs):
        if not _plain(s, dtype, numel):
            _check_device_tensor(s, f"srcs[{i}]")
            raise ChebError(_binding.CHEB_E_MISMATCH, f"srcs[{i}] differs from out in dtype or size")
    cheb_combine([s.data_ptr() for s in srcs], w, out.data_ptr(), numel, dt,
                 _stream_handle(stream))
    return out


def combine_multi(srcs: Sequence[torch.Tensor], w, outs: Sequence[torch.Tensor],
                  stream: Optional[torch.cuda.Stream] = None):
    """outs[m] = sum_k w[m][k] * srcs[k], all outputs from one pass
    (one launch of cheb_combine_multi)."""
    if len(srcs) == 0 or len(outs) == 0:
        raise ChebError(_binding.CHEB_E_INVAL, "no sources or no outputs")
    dt = cheb_dtype(outs[0].dtype)
    dtype, numel = outs[0].dtype, outs[0].numel()
    for i, t in enumerate(list(srcs) + list(outs)):
        if not _plain(t, dtype, numel):
            _check_device_tensor(t, f"tensor {i}")
            raise ChebError(_binding.CHEB_E_MISMATCH, f"tensor {i} differs in dtype or size")
    cheb_combine_multi([s.data_ptr() for s in srcs], w, [o.data_ptr() for o in outs],
                       outs[0].numel(), dt, _stream_handle(stream))
    return outs


def precompute_weights(hist_t, target_t) -> np.ndarray:
    return cheb_precompute_weights(hist_t, target_t)


class ChebTable:
    """The offline stage's weight table (schedule F, rows for every
    predicted step), built in the library or loaded from a file."""

    def __init__(self, T=None, s0=None, s1=None, r=None, n_hist=None, abscissa=None,
                 policy=CHEB_SHORT_FULL, _handle=None):
        if _handle is None:
            _handle = cheb_table_build(T, s0, s1, r, n_hist, abscissa, policy)
        self._h = _handle
        info = cheb_table_info(self._h)
        self.T, self.n_hist, self.policy, self.n_full = (
            info["T"], info["n_hist"], info["policy"], info["n_full"])

    @classmethod
    def from_mask(cls, is_full, n_hist, abscissa, policy=CHEB_SHORT_FULL):
        return cls(_handle=cheb_table_build_mask(is_full, n_hist, abscissa, policy))

    @classmethod
    def load(cls, path):
        return cls(_handle=cheb_table_load(path))

    def save(self, path):
        cheb_table_save(self._h, path)

    def step(self, s):
        return cheb_table_step(self._h, s)

    def runs(self):
        """Consecutive predicted steps sharing one history: [(first, count)],
        each cut to at most CHEB_MAX_OUTPUTS steps."""
        out, s = [], 0
        while s < self.T:
            pred, nodes, _ = self.step(s)
            if not pred:
                s += 1
                continue
            first = s
            while (s < self.T and s - first < CHEB_MAX_OUTPUTS and self.step(s)[0]
                   and self.step(s)[1] == nodes):
                s += 1
            out.append((first, s - first))
        return out

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            cheb_table_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _segment_args(segments: Sequence[torch.Tensor]):
    """(addresses, sizes, storage type) of one step's module outputs."""
    dtype = segments[0].dtype
    dt = cheb_dtype(dtype)
    ptrs, sizes = [], []
    for i, t in enumerate(segments):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype
                and t.is_contiguous()):
            _check_device_tensor(t, f"segments[{i}]")
            raise ChebError(_binding.CHEB_E_MISMATCH, "segments differ in dtype")
        ptrs.append(t.data_ptr())
        sizes.append(t.numel())
    return ptrs, sizes, dt


def residual_reduce(segments: Sequence[torch.Tensor], res_offset, x_out: torch.Tensor,
                    x_in: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """x_out = x_in + the mapped sum of one step's module outputs."""
    ptrs, sizes, dt = _segment_args(segments)
    _check_device_tensor(x_out, "x_out")
    cheb_residual_reduce(ptrs, sizes, res_offset, dt, None if x_in is None else x_in.data_ptr(),
                         x_out.data_ptr(), x_out.numel(), _stream_handle(stream))
    return x_out


_NORMS = {"rms": CHEB_NORM_RMS, "layer": CHEB_NORM_LAYER}
_OUT_8BIT = {"mxfp8": CHEB_OUT_MXFP8, "fp8_row": CHEB_OUT_FP8_ROW}


def norm_output(rows: int, dim: int, out=torch.bfloat16, device=None):
    """Buffers for a norm's output: a [rows, dim] tensor for a torch type, or
    for "mxfp8" and "fp8_row" the e4m3 codes and their scales, [rows,
    ceil(dim / 32)] powers of two or [rows] fp32."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    if isinstance(out, torch.dtype):
        cheb_dtype(out)
        return torch.empty(rows, dim, dtype=out, device=device)
    if out not in _OUT_8BIT:
        raise ChebError(_binding.CHEB_E_DTYPE, f"unknown output format {out!r}")
    y = torch.empty(rows, dim, dtype=torch.float8_e4m3fn, device=device)
    if out == "fp8_row":
        return y, torch.empty(rows, dtype=torch.float32, device=device)
    return y, torch.empty(rows, -(-dim // 32), dtype=torch.float8_e8m0fnu, device=device)


def _here(t, what: str, current: int):
    """Refuses what is no contiguous tensor of the current device."""
    if isinstance(t, torch.Tensor) and t.get_device() == current and t.is_contiguous():
        return
    _check_device_tensor(t, what)
    raise ChebError(_binding.CHEB_E_INVAL,
                    f"{what} is on {t.device}, the current device is {current}")


def _stream_here(stream: Optional[torch.cuda.Stream], current: int) -> int:
    """A stream of the current device."""
    if stream is not None and stream.device.index != current:
        raise ChebError(_binding.CHEB_E_INVAL,
                        f"the stream is on {stream.device}, the current device is {current}")
    return _stream_handle(stream, current)


def _norm_rows(t, what: str, dim: int, rows: int) -> int:
    """Groups of a gain or shift."""
    n = t.numel()
    if t.dtype is not torch.float32 or n == 0 or n % dim:
        raise ChebError(_binding.CHEB_E_MISMATCH, f"{what} must be float32 rows of {dim}")
    if rows % (n // dim):
        raise ChebError(_binding.CHEB_E_MISMATCH, f"{what}: {rows} rows in {n // dim} groups")
    return n // dim


def _norm_call(current, device, x_out, x_in, numel, dim, kind, eps, gain, shift, out, stream):
    """The norm's structure and its output's buffers; every tensor it takes is
    checked, and lies on the current device."""
    x_dt = CHEB_F32
    in_ptr = out_ptr = gain_ptr = shift_ptr = scale_ptr = None
    if x_in is not None:
        _here(x_in, "x_in", current)
        in_ptr, x_dt = x_in.data_ptr(), _DTYPES.get(x_in.dtype)
        if x_in.numel() != numel:
            raise ChebError(_binding.CHEB_E_MISMATCH,
                            f"x_in holds {x_in.numel()} elements, the sources {numel}")
    if x_out is not None:
        _here(x_out, "x_out", current)
        out_ptr, x_dt = x_out.data_ptr(), _DTYPES.get(x_out.dtype)
        if x_out.numel() != numel or (x_in is not None and x_in.dtype is not x_out.dtype):
            raise ChebError(_binding.CHEB_E_MISMATCH, "x_out differs from x_in or the sources")
    if x_dt is None:
        raise ChebError(_binding.CHEB_E_DTYPE, "unsupported dtype of the residual")
    if dim < 1 or numel % dim:
        raise ChebError(_binding.CHEB_E_MISMATCH, f"{numel} elements are no rows of {dim}")
    rows, groups = numel // dim, 0
    norm = _NORMS.get(kind)
    if norm is None:
        raise ChebError(_binding.CHEB_E_INVAL, f"unknown norm {kind!r}")
    if gain is not None:
        _here(gain, "gain", current)
        gain_ptr, groups = gain.data_ptr(), _norm_rows(gain, "gain", dim, rows)
    if shift is not None:
        _here(shift, "shift", current)
        shift_ptr, of_shift = shift.data_ptr(), _norm_rows(shift, "shift", dim, rows)
        if gain is not None and of_shift != groups:
            raise ChebError(_binding.CHEB_E_MISMATCH, "gain and shift differ in groups")
        groups = of_shift
    if type(out) is str or type(out) is torch.dtype:
        form = out
        out = _made_for(stream, device, lambda: norm_output(rows, dim, form, device))
    if isinstance(out, (tuple, list)) and len(out) == 2:
        y, scale = out
        _here(y, "out's codes", current)
        _here(scale, "out's scales", current)
        scale_ptr = scale.data_ptr()
        fmt = CHEB_OUT_FP8_ROW if scale.dtype is torch.float32 else CHEB_OUT_MXFP8
        want = rows if fmt == CHEB_OUT_FP8_ROW else rows * -(-dim // 32)
        if (y.dtype is not torch.float8_e4m3fn or scale.numel() != want
                or (fmt == CHEB_OUT_MXFP8 and scale.dtype is not torch.float8_e8m0fnu)):
            raise ChebError(_binding.CHEB_E_MISMATCH, "out differs from norm_output's")
    else:
        y, fmt = out, _DTYPES.get(getattr(out, "dtype", None))
        if fmt is None:
            raise ChebError(_binding.CHEB_E_DTYPE, "out is of no supported dtype")
        _here(y, "out", current)
    if y.numel() != numel:
        raise ChebError(_binding.CHEB_E_MISMATCH, f"out holds {y.numel()} elements, not {numel}")
    return cheb_norm(rows, dim, eps, in_ptr, out_ptr, gain_ptr, shift_ptr,
                     max(rows // groups, 1) if groups else 0, y.data_ptr(), scale_ptr, norm, x_dt,
                     fmt), out


def add_norm(srcs: Sequence[torch.Tensor], w, x_out: Optional[torch.Tensor] = None,
             x_in: Optional[torch.Tensor] = None, *, dim: Optional[int] = None,
             kind: str = "rms", eps: float = 1e-6, gain: Optional[torch.Tensor] = None,
             shift: Optional[torch.Tensor] = None, out=torch.bfloat16,
             stream: Optional[torch.cuda.Stream] = None):
    """x = x_in + sum_k w[k] * srcs[k], kept in x_out if given, and its norm,
    in one pass: (x_out, y).  ``kind`` is "rms" or "layer"; ``gain`` and
    ``shift`` are fp32 [dim] or [groups, dim], each group for as many rows.
    ``out`` names y's format (a torch type, "mxfp8", "fp8_row") or is
    norm_output's buffers."""
    if len(srcs) == 0 and x_in is None:
        raise ChebError(_binding.CHEB_E_INVAL, "neither sources nor x_in")
    like = srcs[0] if len(srcs) else x_in
    if not isinstance(like, torch.Tensor) or not like.is_cuda:
        _check_device_tensor(like, "srcs[0]" if len(srcs) else "x_in")
    current = torch.cuda.current_device()
    dtype, numel = like.dtype, like.numel()
    ptrs = []
    for s in srcs:
        _here(s, "a source", current)
        if s.dtype is not dtype or s.numel() != numel:
            raise ChebError(_binding.CHEB_E_MISMATCH,
                            f"srcs[{len(ptrs)}] differs in dtype or size")
        ptrs.append(s.data_ptr())
    if dim is None:
        dim = like.shape[-1] if like.dim() else 1
    norm, out = _norm_call(current, like.device, x_out, x_in, numel, dim, kind, eps, gain, shift,
                           out, stream)
    cheb_add_norm(ptrs, w, cheb_dtype(dtype), norm, _stream_here(stream, current))
    return x_out, out


class ResidualHistory:
    """Collapsed history: per full step, only the block stack's total
    contribution to the residual stream (fp32), in a ring of n entries.  A
    skipped step's residual is x_in plus the prediction from these entries,
    which by linearity equals the sum of every module's prediction."""

    def __init__(self, n_slots: int, res_offset: Sequence[int], res_numel: int, device=None):
        self.res_offset = [int(o) for o in res_offset]
        self.res_numel = int(res_numel)
        self.cache = ChebCache(n_slots, torch.float32, [self.res_numel], device=device)

    def push(self, t: float, segments: Sequence[torch.Tensor],
             stream: Optional[torch.cuda.Stream] = None):
        slot = cheb_cache_begin_push(self.cache.handle)
        try:
            ptrs, sizes, dt = _segment_args(segments)
            cheb_residual_reduce(ptrs, sizes, self.res_offset, dt, None, slot, self.res_numel,
                                 _stream_handle(stream))
        except Exception:
            self.cache.abort_push()
            raise
        self.cache.commit(t)

    def push_difference(self, t: float, x_after: torch.Tensor, x_before: torch.Tensor,
                        stream: Optional[torch.cuda.Stream] = None):
        """Entry taken from the residual stream itself.  A full step's block
        stack leaves x_after = x_before + (every module output added into
        the residual), so the entry is x_after - x_before: one launch of
        the combination kernel with weights (1, -1) over residual-sized fp32
        tensors, instead of a pass over every module output.  The difference
        is formed in fp64 and rounded once to fp32."""
        for name, x in (("x_after", x_after), ("x_before", x_before)):
            if x.dtype != torch.float32 or x.numel() != self.res_numel:
                raise ChebError(_binding.CHEB_E_MISMATCH,
                                f"{name} must be float32 with {self.res_numel} elements")
        slot = cheb_cache_begin_push(self.cache.handle)
        try:
            _check_device_tensor(x_after, "srcs[0]")
            _check_device_tensor(x_before, "srcs[1]")
            cheb_combine([x_after.data_ptr(), x_before.data_ptr()], [1.0, -1.0], slot,
                         self.res_numel, CHEB_F32, _stream_handle(stream))
        except Exception:
            self.cache.abort_push()
            raise
        self.cache.commit(t)

    def history(self):
        return self.cache.history()

    def predict(self, target_t: float, x_out: torch.Tensor, x_in: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None):
        w = cheb_precompute_weights(self.history(), [target_t])[0]
        self.cache.residual_apply(w, [0], x_out, x_in, stream=stream)
        return x_out, w

    def predict_norm(self, target_t: float, x_out: Optional[torch.Tensor] = None,
                     x_in: Optional[torch.Tensor] = None, *, dim: int, first: int = 0,
                     rows: Optional[int] = None, kind: str = "rms", eps: float = 1e-6,
                     gain: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                     out=torch.bfloat16, stream: Optional[torch.cuda.Stream] = None):
        """The skipped step's residual and its norm in one pass: (x_out, y, w).
        Rows of ``dim`` from the residual's element ``first`` on: all of it, or
        ``rows`` of them (the image tokens, say); x_in and x_out hold those.
        Other arguments as add_norm's."""
        w = _binding.weights_at(self.cache.handle, target_t)
        x_out, y = self.cache.residual_norm(w, 0, x_out, x_in, dim=dim, first=first, rows=rows,
                                            kind=kind, eps=eps, gain=gain, shift=shift, out=out,
                                            stream=stream)
        return x_out, y, w

    def close(self):
        self.cache.close()


_QUANTS = {None: CHEB_QUANT_NONE, "mxint8": CHEB_QUANT_MXINT8, "mxfp8": CHEB_QUANT_MXFP8}
_LAYOUTS = {"slots": CHEB_LAYOUT_SLOTS, "interleaved": CHEB_LAYOUT_INTERLEAVED}


class _NoPlace(ChebError, AttributeError):
    """Where a plain entry lies, asked of 8-bit entries."""


class ChebCache:
    """The history ring of one feature set, over a torch-allocated arena.

    ``seg_numel`` lists the element counts of the cached tensors in cache
    order.  Outputs (and, in the slot layout, entries) share one flat
    layout; ``segment_views`` cuts a flat buffer into per-segment views.
    ``layout`` is "slots" (contiguous entries; fused push possible) or
    "interleaved" (entries cut into 32 KiB chunks taken in turn; filled by
    ``push``).  ``quant`` is None (entries of ``dtype``) or a format of 8-bit
    entries, "mxint8" or "mxfp8": ``push`` then quantises tensors of ``dtype``
    in groups of 32 elements, and predictions, ``read`` and the residual update
    decode them; tensors start on multiples of 4096 elements.

    A call with ``stream`` works there, and the caller orders that stream with
    others as for any work; an output that the call makes itself may be dropped
    at any time.
    """

    def __init__(self, n_slots: int, dtype: torch.dtype, seg_numel: Sequence[int],
                 device=None, arena: Optional[torch.Tensor] = None, layout: str = "slots",
                 quant: Optional[str] = None):
        self.n_slots = int(n_slots)
        self.dtype = dtype
        self.cdtype = cheb_dtype(dtype)
        self.seg_numel = [int(n) for n in seg_numel]
        if layout not in _LAYOUTS:
            raise ChebError(_binding.CHEB_E_INVAL, f"unknown layout {layout!r}")
        self.layout = layout
        if quant not in _QUANTS:
            raise ChebError(_binding.CHEB_E_INVAL, f"unknown 8-bit format {quant!r}")
        self.quant = quant
        if quant is None:
            lay = cheb_cache_layout(self.n_slots, self.cdtype, self.seg_numel)
            self.slot_stride_bytes = int(lay["slot_stride_bytes"])
            self.arena_bytes = cheb_cache_arena_bytes_ex(self.n_slots, self.cdtype,
                                                         self.seg_numel, _LAYOUTS[layout])
        else:
            lay = cheb_cache_layout_quant(self.n_slots, self.cdtype, _QUANTS[quant],
                                          self.seg_numel, _LAYOUTS[layout])
            self.arena_bytes = int(lay["arena_bytes"])
        self.seg_offset = [int(o) for o in lay["seg_offset"]]
        self.slot_numel = int(lay["slot_numel"])
        if arena is None:
            device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
            arena = torch.empty(self.arena_bytes, dtype=torch.uint8, device=device)
        _check_device_tensor(arena, "arena")
        self.arena = arena
        self.device = arena.device
        if quant is not None:
            self._h = cheb_cache_create_quant(self.n_slots, self.cdtype, _QUANTS[quant],
                                              self.seg_numel, _LAYOUTS[layout], arena.data_ptr(),
                                              arena.numel() * arena.element_size())
            return
        self._h = cheb_cache_create_ex(self.n_slots, self.cdtype, self.seg_numel, _LAYOUTS[layout],
                                       arena.data_ptr(), arena.numel() * arena.element_size())
        _, self.chunk_elems, self.entry_stride_elems = cheb_cache_geometry(self._h)

    # -- lifetime ------------------------------------------------------------
    def close(self):
        if getattr(self, "_h", None) is not None:
            cheb_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __getattr__(self, name):
        if (name in ("slot_stride_bytes", "chunk_elems", "entry_stride_elems")
                and self.__dict__.get("quant") is not None):
            raise _NoPlace(_binding.CHEB_E_INVAL, f"{name}: 8-bit entries lie as the library "
                           "chooses, read() gives them")
        raise AttributeError(f"{type(self).__name__!r} object has no attribute {name!r}")

    @property
    def handle(self):
        return self._h

    def _check_here(self, stream: Optional[torch.cuda.Stream], *tensors: torch.Tensor):
        """Work on 8-bit entries, and reads of any, go to the current device: the
        cache, the stream and the tensors are all on it."""
        current = torch.cuda.current_device()
        if self.device.index != current or (stream is not None
                                            and stream.device.index != current):
            raise ChebError(_binding.CHEB_E_INVAL, f"the cache ({self.device}) or the stream is "
                            f"not on the current device, {current}")
        for t in tensors:
            if t.get_device() != current:
                raise ChebError(_binding.CHEB_E_INVAL, f"a tensor is on {t.device}, the cache "
                                f"on {self.device}")

    # -- buffers -------------------------------------------------------------
    def new_output(self) -> torch.Tensor:
        return torch.empty(self.slot_numel, dtype=self.dtype, device=self.device)

    def _new_output(self, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
        return _made_for(stream, self.device, self.new_output)

    def segment_views(self, flat: torch.Tensor, shapes=None) -> List[torch.Tensor]:
        views = []
        for s, (off, n) in enumerate(zip(self.seg_offset, self.seg_numel)):
            v = flat[off:off + n]
            views.append(v.view(shapes[s]) if shapes is not None else v)
        return views

    def _slot_tensor(self, addr: int) -> torch.Tensor:
        start = addr - self.arena.data_ptr()
        raw = self.arena[start:start + self.slot_numel * self.dtype.itemsize]
        return raw.view(self.dtype)

    def entry(self, idx: int) -> torch.Tensor:
        """The held entry of age index idx (0 = oldest) as a flat tensor: a
        view of its slot in the slot layout, a gathered copy of its chunks
        in the interleaved layout, the values of its codes where entries are
        held in 8 bits."""
        if self.quant is not None:
            return self.read(idx)
        addr = cheb_cache_entry(self._h, idx)
        if self.layout == "slots":
            return self._slot_tensor(addr)
        esz = self.dtype.itemsize
        start = (addr - self.arena.data_ptr()) // esz
        chunk, stride = self.chunk_elems, self.entry_stride_elems
        n_chunks = -(-self.slot_numel // chunk)
        if n_chunks == 0:
            return torch.empty(0, dtype=self.dtype, device=self.device)
        whole = self.arena.view(self.dtype)
        chunks = torch.as_strided(whole, (n_chunks, chunk), (stride, 1),
                                  storage_offset=whole.storage_offset() + start)
        return chunks.reshape(-1)[:self.slot_numel].clone()

    def read(self, idx: int, out: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The held entry of age index idx (0 = oldest) as a flat tensor of its
        own, whatever the layout; of 8-bit entries the values of the codes."""
        out = self._new_output(stream) if out is None else out
        self._check_out(out)
        self._check_here(stream, out)
        cheb_cache_read(self._h, idx, out.data_ptr(), _stream_handle(stream))
        return out

    # -- the online stage ------------------------------------------------------
    def push(self, t: float, segments: Sequence[torch.Tensor],
             stream: Optional[torch.cuda.Stream] = None):
        if len(segments) != len(self.seg_numel):
            raise ChebError(_binding.CHEB_E_MISMATCH, "segment count differs from the layout")
        dtype, ptrs = self.dtype, []
        if self.quant is not None:
            self._check_here(stream)
            device = self.device.index
        for s, n in zip(segments, self.seg_numel):
            if not (isinstance(s, torch.Tensor) and s.is_cuda and s.dtype is dtype
                    and s.numel() == n and s.is_contiguous()):
                _check_device_tensor(s, f"segments[{len(ptrs)}]")
                raise ChebError(_binding.CHEB_E_MISMATCH,
                                f"segments[{len(ptrs)}] differs from the layout")
            if self.quant is not None and s.get_device() != device:
                raise ChebError(_binding.CHEB_E_INVAL, f"segments[{len(ptrs)}] is on {s.device}, "
                                f"the cache on {self.device}")
            ptrs.append(s.data_ptr())
        cheb_cache_push(self._h, t, ptrs, _stream_handle(stream))

    def begin_push(self) -> torch.Tensor:
        """Flat view of the slot the next entry occupies (fused push)."""
        return self._slot_tensor(cheb_cache_begin_push(self._h))

    def commit(self, t: float):
        cheb_cache_commit(self._h, t)

    def abort_push(self):
        """Close an open fused push without recording an entry; the entry
        its slot held stays dropped."""
        cheb_cache_abort_push(self._h)

    def reset(self):
        cheb_cache_reset(self._h)

    def history(self) -> np.ndarray:
        return cheb_cache_history(self._h)

    def _check_out(self, out: torch.Tensor):
        _check_device_tensor(out, "out")
        if out.dtype != self.dtype or out.numel() < self.slot_numel:
            raise ChebError(_binding.CHEB_E_MISMATCH, "out differs from the slot layout")

    def extrapolate(self, w, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        out = self._new_output(stream) if out is None else out
        self._check_out(out)
        if self.quant is not None:
            self._check_here(stream, out)
        cheb_extrapolate(self._h, w, out.data_ptr(), _stream_handle(stream))
        return out

    def extrapolate_multi(self, w, outs: Optional[Sequence[torch.Tensor]] = None,
                          stream: Optional[torch.cuda.Stream] = None):
        w = np.asarray(w, dtype=np.float64).reshape(-1, self.n_slots)
        outs = [self._new_output(stream) for _ in range(w.shape[0])] if outs is None else list(outs)
        for o in outs:
            self._check_out(o)
        if self.quant is not None:
            self._check_here(stream, *outs)
        cheb_extrapolate_multi(self._h, w, [o.data_ptr() for o in outs],
                               _stream_handle(stream))
        return outs

    def extrapolate_at_multi(self, targets, outs: Optional[Sequence[torch.Tensor]] = None,
                             stream: Optional[torch.cuda.Stream] = None):
        targets = list(targets)
        outs = [self._new_output(stream) for _ in targets] if outs is None else list(outs)
        for o in outs:
            self._check_out(o)
        if self.quant is not None:
            self._check_here(stream, *outs)
        w = cheb_extrapolate_at_multi(self._h, targets, [o.data_ptr() for o in outs],
                                      _stream_handle(stream), n_slots=self.n_slots)
        return outs, w

    def extrapolate_steps(self, table: "ChebTable", first_step: int, n_steps: int = 1,
                          outs: Optional[Sequence[torch.Tensor]] = None,
                          stream: Optional[torch.cuda.Stream] = None):
        outs = [self._new_output(stream) for _ in range(n_steps)] if outs is None else list(outs)
        for o in outs:
            self._check_out(o)
        if self.quant is not None:
            self._check_here(stream, *outs)
        cheb_extrapolate_steps(self._h, table.handle, first_step, [o.data_ptr() for o in outs],
                               _stream_handle(stream))
        return outs

    def residual_apply(self, w, res_offset, x_out: torch.Tensor,
                       x_in: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """x_out = x_in + the block stack's predicted module outputs (one pass)."""
        _check_device_tensor(x_out, "x_out")
        if x_out.dtype != torch.float32:
            raise ChebError(_binding.CHEB_E_DTYPE, "the residual is float32")
        if x_in is not None:
            _check_device_tensor(x_in, "x_in")
            if x_in.dtype != torch.float32 or x_in.numel() != x_out.numel():
                raise ChebError(_binding.CHEB_E_MISMATCH, "x_in differs from x_out")
        if self.quant is not None:
            self._check_here(stream, x_out, x_out if x_in is None else x_in)
        cheb_residual_apply(self._h, w, res_offset, x_out.numel(),
                            None if x_in is None else x_in.data_ptr(), x_out.data_ptr(),
                            _stream_handle(stream))
        return x_out

    def residual_norm(self, w, seg: int, x_out: Optional[torch.Tensor] = None,
                      x_in: Optional[torch.Tensor] = None, *, dim: int, first: int = 0,
                      rows: Optional[int] = None, kind: str = "rms", eps: float = 1e-6,
                      gain: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                      out=torch.bfloat16, stream: Optional[torch.cuda.Stream] = None):
        """x = x_in + the prediction of cached tensor ``seg`` from its element
        ``first`` on, and its norm, in one pass: (x_out, y).  Rows of ``dim``,
        as many as fit or ``rows``; other arguments as add_norm's."""
        if not 0 <= seg < len(self.seg_numel):
            raise ChebError(_binding.CHEB_E_INVAL, f"segment {seg} out of range")
        w = np.asarray(w, dtype=np.float64)
        if w.size != self.n_slots:
            raise ChebError(_binding.CHEB_E_INVAL, f"{w.size} weights for {self.n_slots} entries")
        dim, left = int(dim), self.seg_numel[seg] - first
        if dim < 1 or first < 0 or left < 0 or (rows is not None and rows < 0):
            raise ChebError(_binding.CHEB_E_INVAL, f"no rows of {dim} from element {first} on")
        rows = left // dim if rows is None else int(rows)
        current = torch.cuda.current_device()
        _here(self.arena, "the cache", current)
        norm, out = _norm_call(current, self.device, x_out, x_in, rows * dim, dim, kind, eps, gain,
                               shift, out, stream)
        cheb_residual_norm(self._h, w, seg, first, norm, _stream_here(stream, current))
        return x_out, out

    def extrapolate_at(self, target_t: float, out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None):
        out = self._new_output(stream) if out is None else out
        self._check_out(out)
        if self.quant is not None:
            self._check_here(stream, out)
        w = cheb_extrapolate_at(self._h, target_t, out.data_ptr(), _stream_handle(stream),
                                n_slots=self.n_slots)
        return out, w


__all__ = [n for n in dir() if n.startswith("cheb_")] + [
    "ChebCache", "ChebTable", "ChebError", "ResidualHistory", "residual_reduce", "add_norm",
    "norm_output", "combine", "combine_multi", "precompute_weights", "CHEB_BF16",
    "CHEB_F32", "CHEB_MAX_SLOTS", "CHEB_MAX_OUTPUTS", "CHEB_MAX_NODES", "LIB_PATH"]
