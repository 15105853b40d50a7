"""ctypes binding of the sampling phase (include/paged_attn.h): rotary positions with several axes, the paged cache of keys and
values, and the attention of each sequence's newest tokens over its pages.

Tensors are torch device tensors.  Their types, shapes, devices and strides are checked by a small native module (csrc/py_sampling.cpp) and the
numbers in the library; either way a call that cannot run raises PrefixAttnError before anything is enqueued.  There is no CPU
fallback."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np

from . import binding
from .binding import PA_BF16, PA_F32, PrefixAttnError, _stream

MAX_AXES, MAX_PAIRS = 4, 128                # PA_ROPE_MAX_AXES, PA_ROPE_MAX_PAIRS of the header
LAYOUTS = {"halves": 0, "pairs": 1}         # pa_rope_layout_t
_DTYPES = {"f32": PA_F32, "bf16": PA_BF16}
_SHAPE, _UNSUPPORTED = 2, 3                 # PA_ERR_SHAPE, PA_ERR_UNSUPPORTED
EXPORTED_SYMBOLS = ("rope_axes_forward", "rope_axes_backward", "paged_attn_plan", "paged_attn_destroy", "paged_kv_append",
                    "paged_kv_append_rope", "paged_attn_forward", "paged_attn_schedule", "paged_attn_schedule_shape")
_lib = None
_native = None                              # the module built from csrc/py_sampling.cpp


class _RopeDesc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("num_axes", ctypes.c_int32), ("pair_axis", ctypes.c_uint8 * MAX_PAIRS)]


class _PagedDesc(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int64), ("max_pages_per_seq", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32), ("max_tokens", ctypes.c_int64), ("softmax_scale", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("device", ctypes.c_int32)]


def _load():
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load_library()
    i32, i64, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    lib.paged_attn_plan.restype = ctypes.c_int
    lib.paged_attn_plan.argtypes = [ctypes.POINTER(_PagedDesc), ctypes.POINTER(vp), ctypes.POINTER(sz)]
    lib.paged_attn_schedule.restype = i64
    lib.paged_attn_schedule.argtypes = [vp, vp, vp, i32, i64, i32, vp, i64]
    lib.paged_attn_schedule_shape.restype = ctypes.c_int
    lib.paged_attn_schedule_shape.argtypes = [vp, i32, i64, i32, *[ctypes.POINTER(i32)] * 3]
    lib.paged_attn_destroy.restype, lib.paged_attn_destroy.argtypes = None, [vp]
    _lib = lib
    return lib


def _load_native():
    """Imports the module that checks the calls' tensors; raises if it has not been built (python -m paper_2507_07966_amd.build)."""
    global _native
    _load()   # torch and the library first: the module links to both
    try:
        from . import _sampling
    except ImportError as e:
        raise ImportError(f"the module of the sampling calls cannot be loaded ({e}): build it with `python -m paper_2507_07966_amd.build`, which needs "
                          f"torch, Python's headers and g++") from e
    _native = _sampling
    return _native


def _refuse(status: int, where: str, what: str):
    raise PrefixAttnError(status, f"{where}: {what}")


def _check(where: str, refused) -> None:
    """`refused`: None, or the status and the text that csrc/py_sampling.cpp returns for a call that was not enqueued."""
    if refused is not None:
        status, what = refused
        raise PrefixAttnError(status, f"{where}: {what}" if what else where)


class RopeAxes:
    """What the rotation of a head is: see rope_axes()."""

    def __init__(self, desc: _RopeDesc):
        self._desc = desc
        self._address = ctypes.addressof(desc)
        self.head_dim, self.rotary_dim, self.num_axes = desc.head_dim, desc.rotary_dim, desc.num_axes
        self.layout = {v: k for k, v in LAYOUTS.items()}[desc.layout]
        self.pair_axis = tuple(desc.pair_axis[:desc.rotary_dim // 2])


def rope_axes(sections: Sequence[int], head_dim: int, rotary_dim: Optional[int] = None, layout: str = "halves",
              interleaved: bool = False) -> RopeAxes:
    """A rotary embedding of 1 to 4 axes (time, height and width of a video token): sections[a] pairs of channels turn with axis a,
    sum(sections) = rotary_dim / 2; the channels from rotary_dim (head_dim by default) on pass through.
    layout "halves": pair i is channels (i, i + rotary_dim / 2); "pairs": (2 i, 2 i + 1).
    interleaved: the axes take pairs in turn (0, 1, 2, 0, 1, 2, ...) until their sections are used up, instead of one
    run each."""
    sections = [int(n) for n in sections]
    rotary_dim = int(head_dim if rotary_dim is None else rotary_dim)
    if not 1 <= len(sections) <= MAX_AXES or min(sections) < 0 or 2 * sum(sections) != rotary_dim or rotary_dim > 2 * MAX_PAIRS:
        _refuse(_SHAPE, "rope_axes", f"sections {sections} have to be 1 to {MAX_AXES} counts of pairs that sum to "
                                     f"rotary_dim / 2 = {rotary_dim / 2:g}, at most {MAX_PAIRS}")
    if layout not in LAYOUTS:
        _refuse(_UNSUPPORTED, "rope_axes", f"layout has to be one of {sorted(LAYOUTS)}, not {layout!r}")
    if interleaved:
        left, axes = list(sections), []
        while len(axes) < sum(sections):
            for a in range(len(left)):
                if left[a]:
                    left[a] -= 1
                    axes.append(a)
    else:
        axes = [a for a, n in enumerate(sections) for _ in range(n)]
    d = _RopeDesc()
    d.head_dim, d.rotary_dim, d.layout, d.num_axes = int(head_dim), rotary_dim, LAYOUTS[layout], len(sections)
    if not 2 <= rotary_dim <= int(head_dim) <= 2 * MAX_PAIRS:
        _refuse(_SHAPE, "rope_axes", f"rotary_dim {rotary_dim} of head_dim {head_dim}: 2 <= rotary_dim <= head_dim <= {2 * MAX_PAIRS}")
    d.pair_axis[:len(axes)] = axes
    return RopeAxes(d)


def rope_axes_forward(rope: RopeAxes, q, k, positions, inv_freq, q_out, k_out, stream=None) -> None:
    """rope_axes_forward of the C ABI: the heads of q [T, Hq, D] and k [T, Hk, D] (or None, with k_out None) turned by positions
    [axes, T] int32 times inv_freq [rotary_dim / 2] fp32, into q_out and k_out (which may be q and k).  Heads are contiguous, tokens
    may be strided (slices of a fused projection).  Enqueues only."""
    _check("rope_axes_forward", (_native or _load_native()).rope(False, rope._address, q, k, positions, inv_freq, q_out, k_out, _stream(stream)))


def rope_axes_backward(rope: RopeAxes, dq_out, dk_out, positions, inv_freq, dq, dk, stream=None) -> None:
    """rope_axes_backward of the C ABI: the gradients dq, dk of q and k from those of q_out and k_out, same shapes."""
    _check("rope_axes_backward", (_native or _load_native()).rope(True, rope._address, dq_out, dk_out, positions, inv_freq, dq, dk, _stream(stream)))


class PagedAttnPlan:
    """Owner of a paged_attn_plan_t*; see paged_attn_plan()."""

    def __init__(self, handle, workspace_bytes, kw):
        self._h = handle
        self.workspace_bytes = int(workspace_bytes)
        self.__dict__.update(kw)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("plan was destroyed")
        return self._h

    def schedule(self, seq_lens, cu_new, num_tokens: int, shared_len: int = -1) -> np.ndarray:
        """The pieces of work that paged_attn_forward's workgroups take for these lengths (host arrays; shared_len -1: not given): int32
        [n, 8] = (share, sequence (-1: the shared keys), kv head, first stacked row, rows, first key, end of the keys, whole block)."""
        lib = _lib or _load()
        lens, cu = np.asarray(seq_lens), np.asarray(cu_new)
        if lens.ndim != 1 or cu.shape != (len(lens) + 1,):   # the library reads so many of them
            _refuse(_SHAPE, "schedule", f"seq_lens [n] and cu_new [n + 1], not {list(lens.shape)} and {list(cu.shape)}")
        for name, x in (("seq_lens", lens), ("cu_new", cu), ("num_tokens", np.asarray(num_tokens)), ("shared_len", np.asarray(shared_len))):
            if x.dtype.kind not in "iu" and x.size:
                _refuse(_UNSUPPORTED, "schedule", f"{name} has to be whole numbers, not {x.dtype}")
            if x.size and not -(1 << 31) <= int(x.min()) <= int(x.max()) < 1 << 31:
                _refuse(_SHAPE, "schedule", f"{name} does not fit 32 bits")
        lens, cu = (np.ascontiguousarray(x, dtype=np.int32) for x in (lens, cu))
        args = self.handle, lens.ctypes.data, cu.ctypes.data, len(lens), int(num_tokens), int(shared_len)
        n = lib.paged_attn_schedule(*args, None, 0)
        if n < 0:
            raise PrefixAttnError(-n, "paged_attn_schedule")
        out = np.zeros((n, 8), dtype=np.int32)
        lib.paged_attn_schedule(*args, out.ctypes.data, n)
        return out

    def schedule_shape(self, num_seqs: int, num_tokens: int, shared: bool = False):
        """Workgroups of such a call, rows of a block and keys of a tile."""
        if not (0 < num_seqs <= self.max_seqs and 0 < num_tokens <= self.max_tokens):
            _refuse(_SHAPE, "schedule_shape", f"{num_seqs} sequences and {num_tokens} tokens: 1 to {self.max_seqs} and {self.max_tokens} on this plan")
        v = [ctypes.c_int32() for _ in range(3)]
        st = (_lib or _load()).paged_attn_schedule_shape(self.handle, int(num_seqs), int(num_tokens), int(shared), *map(ctypes.byref, v))
        if st:
            raise PrefixAttnError(st, "paged_attn_schedule_shape")
        return tuple(x.value for x in v)

    def destroy(self):
        if self._h is not None:
            _load().paged_attn_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def paged_attn_plan(num_q_heads: int, num_kv_heads: int, head_dim: int, page_size: int, num_pages: int, max_pages_per_seq: int,
                    max_seqs: int, max_tokens: int, softmax_scale: float, dtype: str = "bf16", device: int = 0) -> PagedAttnPlan:
    """paged_attn_plan of the C ABI: the heads, the cache (num_pages pages of page_size tokens) and the largest call (max_seqs
    sequences of max_pages_per_seq pages, max_tokens new tokens in all).  dtype "bf16" | "f32"; device -1 = host-only plan."""
    lib = _load()
    d = _PagedDesc()
    kw = dict(num_q_heads=int(num_q_heads), num_kv_heads=int(num_kv_heads), head_dim=int(head_dim), page_size=int(page_size),
              num_pages=int(num_pages), max_pages_per_seq=int(max_pages_per_seq), max_seqs=int(max_seqs),
              max_tokens=int(max_tokens), softmax_scale=float(softmax_scale), device=int(device))
    for name, value in kw.items():
        setattr(d, name, value)
        if name != "softmax_scale" and getattr(d, name) != value:
            _refuse(_SHAPE, "paged_attn_plan", f"{name} = {value} is out of range")
    d.dtype = _DTYPES.get(dtype, -1)
    h, ws = ctypes.c_void_p(), ctypes.c_size_t()
    st = lib.paged_attn_plan(ctypes.byref(d), ctypes.byref(h), ctypes.byref(ws))
    if st:
        raise PrefixAttnError(st, "paged_attn_plan")
    return PagedAttnPlan(h.value, ws.value, dict(kw, dtype=dtype))


def paged_kv_append(plan: PagedAttnPlan, k, v, k_cache, v_cache, page_table, seq_lens, cu_new, stream=None) -> None:
    """paged_kv_append of the C ABI: the new tokens' k, v [T, Hkv, D] into their pages of the caches [num_pages, Hkv, page_size, D].
    page_table [B, max_pages_per_seq], seq_lens [B] (new tokens included) and cu_new [B + 1] (packed rows) are int32.  Enqueues only."""
    _check("paged_kv_append", (_native or _load_native()).append(plan.handle, None, None, k, v, None, None, None, k_cache, v_cache, page_table,
                                                                 seq_lens, cu_new, _stream(stream)))


def paged_kv_append_rope(plan: PagedAttnPlan, rope: RopeAxes, q, k, v, positions, inv_freq, q_out, k_cache, v_cache, page_table,
                         seq_lens, cu_new, stream=None) -> None:
    """paged_kv_append_rope of the C ABI: the keys rotated as they are stored, and q [T, Hq, D] rotated into q_out (which may be q;
    both None to leave queries alone).  positions [axes, T] int32 and inv_freq as in rope_axes_forward.  Enqueues only."""
    _check("paged_kv_append_rope", (_native or _load_native()).append(plan.handle, rope._address, q, k, v, positions, inv_freq, q_out, k_cache,
                                                                      v_cache, page_table, seq_lens, cu_new, _stream(stream)))


def paged_attn_forward(plan: PagedAttnPlan, q, k_cache, v_cache, page_table, seq_lens, cu_new, out, lse_out, workspace,
                       shared_len=None, stream=None) -> None:
    """paged_attn_forward of the C ABI: attention of the new tokens q [T, Hq, D] over the pages of their sequences, into out
    [T, Hq, D] and lse_out [Hq, T] fp32 (or None).  The new tokens' keys and values are in the cache already (paged_kv_append).
    shared_len: None, or an int32 tensor of one element: so many leading tokens of all sequences are in the same pages, which calls
    of at most 56 rows (tokens times Hq / Hkv) a sequence then read once for every 64 rows (fp32: 32) of all sequences together.
    `workspace`: uint8, at least plan.workspace_bytes.  Enqueues only."""
    _check("paged_attn_forward", (_native or _load_native()).attend(plan.handle, q, k_cache, v_cache, page_table, seq_lens, cu_new, out, lse_out,
                                                                    workspace, shared_len, _stream(stream)))
