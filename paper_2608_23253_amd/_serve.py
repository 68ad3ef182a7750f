"""ctypes binding of the operators on either side of the scoring path (the C ABI
declared in include/e2s_serve.h): rotary positions, the paged 8-bit key/value cache,
attention over it, and eviction from it.

Argument marshalling only, as in ``_lib``: functions with the C names minus the
``e2s_`` prefix take torch tensors on the GPU, allocate what they return, pass raw
device pointers and the current torch stream, and raise ``E2SError`` on a non-zero
status.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Optional

from . import _lib
from ._lib import _CURRENT_STREAM, _check, _dtype_code, _launch, _ptr, _raise, _torch

HEADER = os.path.join(os.path.dirname(_lib.PKG), "include", "e2s_serve.h")

ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}
MAX_PAIRS = 128

_I32, _I64, _F64, _P = ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p


class RotarySpec(ctypes.Structure):
    _fields_ = [("head_dim", _I32), ("rot_dim", _I32), ("layout", _I32), ("scaling", _I32),
                ("sections", _I32 * 3), ("reserved", _I32), ("amplitude", _F64), ("base", _F64),
                ("factor", _F64), ("original_len", _F64), ("low", _F64), ("high", _F64)]


class RotaryPlan(ctypes.Structure):
    """e2s_rotary_plan: the frequencies, kept by the caller (see rotary_plan)."""
    _fields_ = [("head_dim", _I32), ("rot_dim", _I32), ("layout", _I32), ("axes", _I32),
                ("amplitude", ctypes.c_float), ("reserved", _I32),
                ("axis", ctypes.c_uint8 * MAX_PAIRS), ("turns", _F64 * MAX_PAIRS)]


class RotaryShape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_tokens", _I32), ("q_heads", _I32), ("k_heads", _I32),
                ("dtype", _I32), ("inverse", _I32), ("q_stride", _I64 * 3),
                ("k_stride", _I64 * 3), ("q_out_stride", _I64 * 3), ("k_out_stride", _I64 * 3),
                ("pos_stride", _I64 * 3)]


class CacheDesc(ctypes.Structure):
    """e2s_cache."""
    _fields_ = [("num_pages", _I32), ("page_tokens", _I32), ("num_kv_heads", _I32),
                ("head_dim", _I32), ("k_page_stride", _I64), ("v_page_stride", _I64), ("k", _P),
                ("v", _P), ("k_scale", _P), ("v_scale", _P)]


class AppendShape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_tokens", _I32), ("src_tokens", _I32), ("dtype", _I32),
                ("max_pages", _I32), ("reserved", _I32), ("pages_stride", _I64),
                ("k_stride", _I64 * 3), ("v_stride", _I64 * 3)]


class AttendShape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_heads", _I32), ("num_queries", _I32), ("dtype", _I32),
                ("max_tokens", _I32), ("max_pages", _I32), ("causal", _I32), ("weights", _I32),
                ("scale", ctypes.c_float), ("reserved", _I32), ("pages_stride", _I64),
                ("q_stride", _I64 * 3), ("out_stride", _I64 * 3),
                ("weights_in_stride", _I64 * 2), ("weights_out_stride", _I64 * 2)]


class EvictShape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("max_tokens", _I32), ("budget", _I32), ("sinks", _I32),
                ("recent", _I32), ("max_pages", _I32), ("new_max_pages", _I32),
                ("left_tokens", _I32), ("pages_stride", _I64), ("new_pages_stride", _I64),
                ("weights_stride", _I64 * 2), ("left_stride", _I64 * 2)]


def _ref(t):
    return ctypes.POINTER(t)


SIGNATURES = {
    "e2s_rotary_plan_init": [_ref(RotarySpec), _ref(RotaryPlan)],
    "e2s_rotate_positions": [_P, _ref(RotaryPlan), _P, _P, _P, _P, _P, _P],
    "e2s_cache_append": [_ref(CacheDesc), _P, _P, _P, _P, _P, _P, _P, _P],
    "e2s_cache_attend_workspace_size": [_ref(CacheDesc), _P, _ref(ctypes.c_size_t)],
    "e2s_cache_attend": [_ref(CacheDesc), _P, _P, _P, _P, _P, _P, _P, _P, _P,
                         ctypes.c_size_t, _P],
    "e2s_cache_evict": [_ref(CacheDesc), _P, _P, _P, _P, _P, _P, _P, _P, _P],
    "e2s_serve_abi_version": [],
}
for _name, _args in SIGNATURES.items():
    _fn = getattr(_lib.lib(), _name)
    _fn.argtypes, _fn.restype = _args, ctypes.c_int
_LIB = _lib.lib()


# What a step passes is packed in the records' layout (native sizes and alignment): one call
# in place of one per field.
_ROTARY = struct.Struct("@6i15q")
_APPEND = struct.Struct("@6i7q")
_ATTEND = struct.Struct("@8ifi11q")
_EVICT = struct.Struct("@8i6q")


# (the binding loads without torch, too)
_Function = _lib._TORCH.autograd.Function if _lib._TORCH is not None else object


def _allocating_on(stream, device):
    """What a call allocates, and fills with zeros, belongs to the stream it runs on."""
    if stream is None:
        return _HERE
    torch = _torch()
    return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device))


_HERE = contextlib.nullcontext()


def _like(t, stream, order=None):
    torch = _torch()
    with _allocating_on(stream, t.device):
        return torch.empty_like(t, memory_format=order or torch.preserve_format)


_AD = _lib._TORCH.autograd.forward_ad if _lib._TORCH is not None else None


def _no_tangents(where, *tensors):
    """Forward-mode differentiation has no rule here: an error says so where a launch, which
    knows of values alone, would lose the tangents.  (Outside a dual level there are none: one
    look, where torch says which level it is in.)"""
    if getattr(_AD, "_current_level", 0) < 0:
        return
    for t in tensors:
        if t is not None and _AD.unpack_dual(t).tangent is not None:
            raise RuntimeError(f"{where} has no forward-mode derivative")


def _rows(t, name, dtype=None):
    """The strides of a [B, H, T, d] tensor of rows: any, the last dimension contiguous."""
    if not (isinstance(t, _torch().Tensor) and t.is_cuda and t.dim() == 4 and
            (dtype is None or t.dtype is dtype)):
        _check(t, name, dtype=dtype, ndim=4, contiguous=False)
    st = t.stride()
    if st[3] != 1 and t.shape[3] > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return st


def _moved(shape, a, b):
    """Whether rows of a shape lie elsewhere by strides b than by strides a (a dimension of one
    may have any)."""
    return a[:3] != b[:3] and any(n > 1 and x != y for n, x, y in zip(shape[:3], a, b))


def _vector(t, name, n):
    """The address of an int32 [n] of per-sequence numbers."""
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.int32 and
            t.dim() == 1 and t.is_contiguous()):
        _check(t, name, dtype=torch.int32, ndim=1)
    if t.shape[0] != n:
        raise ValueError(f"{name} must be [{n}] (got {tuple(t.shape)})")
    return t.data_ptr()


def _table(t, name, n):
    """The width and the row stride of an int32 [n, max_pages]."""
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.int32 and
            t.dim() == 2):
        _check(t, name, dtype=torch.int32, ndim=2, contiguous=False)
    (rows, width), st = t.shape, t.stride()
    if rows != n or width < 1 or (st[1] != 1 and width > 1):
        raise ValueError(f"{name} must be [{n}, max_pages] with contiguous rows")
    return width, st[0]


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

def rotary_plan(head_dim: int, rot_dim: Optional[int] = None, base: float = 10000.0,
                layout="half", scaling="none", factor: float = 1.0, original_len: float = 0.0,
                low: float = 1.0, high: float = 32.0, amplitude: float = 0.0,
                sections=None) -> RotaryPlan:
    """The frequencies of e2s_rotate_positions (see e2s_rotary_spec): rot_dim leading
    elements of a row turn (default: all).  scaling: "none", "linear", "base" or "ramp" (linear
    in a pair's turns, not in its number).
    sections: numbers of pairs that turn by each of three positions, or None."""
    spec = RotarySpec(head_dim, head_dim if rot_dim is None else rot_dim,
                      ROTARY_LAYOUTS[layout] if isinstance(layout, str) else int(layout),
                      ROTARY_SCALINGS[scaling] if isinstance(scaling, str) else int(scaling),
                      (_I32 * 3)(*(sections or (0, 0, 0))), 0, amplitude, base, factor,
                      original_len, low, high)
    plan = RotaryPlan()
    _raise(_LIB.e2s_rotary_plan_init(ctypes.byref(spec), ctypes.byref(plan)),
           "e2s_rotary_plan_init")
    return plan


class _Rotate(_Function):
    """The rotation, whose transpose is the rotation back."""

    @staticmethod
    def forward(ctx, q, k, positions, plan, inverse):
        ctx.save_for_backward(positions)
        ctx.plan, ctx.inverse = plan, inverse
        ctx.set_materialize_grads(False)
        return rotate_positions(q, k, positions, plan, inverse)

    @staticmethod
    def backward(ctx, *grads):
        # (a broadcast gradient has no contiguous rows)
        gq, gk = (g.contiguous() if need and g is not None and g.stride(3) != 1 else
                  g if need else None for g, need in zip(grads, ctx.needs_input_grad))
        if gq is None and gk is None:
            return None, None, None, None, None
        return (*rotate_positions(gq, gk, *ctx.saved_tensors, ctx.plan, not ctx.inverse), None,
                None, None)


def rotate_positions(q, k, positions, plan: RotaryPlan, inverse: bool = False, q_out=None,
                     k_out=None, stream: Optional[int] = None):
    """q [B, H, T, d] and k [B, Hkv, T, d] (either may be None; any strides with contiguous
    rows) turned by `positions`: int32 [T] or [B, T], with a leading 3 for a plan of three
    axes.  inverse turns back: the transpose, which takes a gradient of the outputs to that
    of the inputs.  Returns (q_out, k_out); an output may be its input.  Outputs that are
    not given have a gradient where the inputs ask for one."""
    torch = _torch()
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k is needed")
    _no_tangents("rotate_positions", q, k)
    if (x.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
        if q_out is not None or k_out is not None:
            raise ValueError("an output that is given has no gradient: give none, or call "
                             "under torch.no_grad()")
        with _allocating_on(stream, x.device):
            return _Rotate.apply(q, k, positions, plan, inverse)
    dtype, B, T, D = x.dtype, x.shape[0], x.shape[2], plan.head_dim
    heads, strides, out_strides, ptrs, outs = [], [], [], [], []
    for t, name, o in ((q, "q", q_out), (k, "k", k_out)):
        if t is None:
            if o is not None:
                raise ValueError(f"{name}_out without {name}")
            heads.append(0)
            strides += (0, 0, 0)
            out_strides += (0, 0, 0)
            ptrs += (None, None)
            outs.append(None)
            continue
        st = _rows(t, name, dtype)
        shape = t.shape
        if shape[0] != B or shape[2] != T or shape[3] != D:
            raise ValueError(f"{name} {tuple(shape)} must be [B, heads, T, {D}] "
                             "with one B and T")
        if o is None:
            o = _like(t, stream) if stream is not None else torch.empty_like(t)
            so = o.stride()
            if so[3] != 1:               # rows one element apart: torch may order them first
                o = _like(t, stream, torch.contiguous_format)
                so = o.stride()
        else:
            so = _rows(o, name + "_out", dtype)
            if o.shape != shape:
                raise ValueError(f"{name}_out must have {name}'s shape")
            if o.data_ptr() == t.data_ptr() and _moved(shape, st, so):
                raise ValueError(f"{name}_out in the place of {name} must have its strides")
        heads.append(shape[1])
        strides += st[:3]
        out_strides += so[:3]
        ptrs += (t.data_ptr(), o.data_ptr())
        outs.append(o)
    if not (isinstance(positions, torch.Tensor) and positions.is_cuda and
            positions.dtype is torch.int32):
        _check(positions, "positions", dtype=torch.int32, contiguous=False)
    lead = (3,) if plan.axes == 3 else ()
    shape, ps = positions.shape, positions.stride()
    if shape == lead + (B, T):
        ps = (ps[0] if lead else 0, ps[-2], ps[-1])
    elif shape == lead + (T,):
        ps = (ps[0] if lead else 0, 0, ps[-1])
    else:
        raise ValueError(f"positions must be {list(lead + (T,))} or {list(lead + (B, T))} "
                         f"(got {list(shape)})")
    if B > 0 and T > 0:
        sh = _ROTARY.pack(B, T, *heads, _dtype_code(x), 1 if inverse else 0, *strides,
                          *out_strides, *ps)
        _launch("e2s_rotate_positions", (q, k, positions, *outs), _LIB.e2s_rotate_positions, sh,
                ctypes.byref(plan), positions.data_ptr(), ptrs[0], ptrs[2], ptrs[1], ptrs[3],
                stream=stream)
    return outs[0], outs[1]


# ---------------------------------------------------------------------------
# the 8-bit cache
# ---------------------------------------------------------------------------

class PagedCache:
    """The 8-bit cache of one layer (e2s_cache): k, v [num_pages, Hkv, P, d]
    float8_e4m3fn and k_scale, v_scale [num_pages, Hkv] float32; a held value is its byte
    times its block's scale, a power of two (2^-100 .. 2^120: of any other that the caller
    puts there attention reads the exponent alone).  Which sequence a page belongs to is the
    caller's page table's to say."""

    def __init__(self, num_pages: int, num_kv_heads: int, head_dim: int, page_tokens: int = 64,
                 device="cuda"):
        torch = _torch()
        shape = (num_pages, num_kv_heads, page_tokens, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
                for _ in range(2))
        ks, vs = (torch.ones(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        self._hold(k, v, ks, vs)

    @classmethod
    def of(cls, k, v, k_scale, v_scale) -> "PagedCache":
        """A cache in memory that the caller allocated; the pages of k and v may lie apart
        (a pool that holds every layer's pages), what is in a page may not."""
        self = cls.__new__(cls)
        self._hold(k, v, k_scale, v_scale)
        return self

    def _hold(self, k, v, k_scale, v_scale):
        torch = _torch()
        for t, name in ((k, "k"), (v, "v")):
            _check(t, name, dtype=torch.float8_e4m3fn, ndim=4, contiguous=False)
            if t.shape != k.shape or t.numel() == 0:
                raise ValueError("k and v must have one shape [num_pages, Hkv, P, d], not empty")
            if not t[0].is_contiguous():
                raise ValueError(f"a page of {name} must be contiguous")
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _check(t, name, dtype=torch.float32, ndim=2)
            if t.shape != k.shape[:2]:
                raise ValueError(f"{name} must be [num_pages, Hkv]")
        _lib._device_of(k, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.num_kv_heads, self.page_tokens, self.head_dim = k.shape
        self.device = k.device
        page = k[0].numel()
        st = [t.stride(0) if self.num_pages > 1 else page for t in (k, v)]
        self.desc = CacheDesc(*k.shape[:1], self.page_tokens, self.num_kv_heads, self.head_dim,
                              st[0], st[1], k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                              v_scale.data_ptr())
        self.desc_ref = ctypes.byref(self.desc)


def cache_append(cache: PagedCache, pages, start, k, v, count=None, src_idx=None,
                 stream: Optional[int] = None):
    """New tokens into the cache (e2s_cache_append).  k, v [B, Hkv, N, d] (any strides with
    16-byte aligned rows) hold sequence b's tokens start[b], start[b] + 1, ...: all N, the
    first count[b], or the rows that src_idx [B, T] int32 names (e.g. prune()'s
    keep_idx).  pages [B, max_pages], start and count [B] are int32."""
    torch = _torch()
    G, D = cache.num_kv_heads, cache.head_dim
    ks = _rows(k, "k")
    vs = _rows(v, "v", k.dtype)
    B, N = k.shape[0], k.shape[2]
    if k.shape != (B, G, N, D) or v.shape != (B, G, N, D):
        raise ValueError(f"k and v must be [B, {G}, N, {D}]")
    width, row = _table(pages, "pages", B)
    start_at = _vector(start, "start", B)
    count_at = None if count is None else _vector(count, "count", B)
    T = N
    if src_idx is not None:
        _check(src_idx, "src_idx", dtype=torch.int32, ndim=2)
        if src_idx.shape[0] != B:
            raise ValueError("src_idx must be [B, T]")
        T = src_idx.shape[1]
    if B == 0 or T == 0:
        return
    sh = _APPEND.pack(B, T, N, _dtype_code(k), width, 0, row, *ks[:3], *vs[:3])
    _launch("e2s_cache_append", (cache.k, pages, start, k, v, count, src_idx),
            _LIB.e2s_cache_append, cache.desc_ref, sh, pages.data_ptr(), start_at, count_at,
            _ptr(src_idx), k.data_ptr(), v.data_ptr(), stream=stream)


class _Undifferentiated(_Function):
    """The outputs of call(), whose gradient is asked for in vain: an error says so where it
    would otherwise be lost."""

    @staticmethod
    def forward(ctx, q, call):
        return call()

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("attention over the 8-bit cache has no backward pass: call it under "
                           "torch.no_grad() or with detached queries")


class CacheAttention:
    """Repeated e2s_cache_attend calls of one shape: `batch` sequences of at most
    `max_tokens` cached tokens and `num_queries` queries.  It holds the workspace, so calls
    of one object on several streams are the caller's to order, and a stream that a call
    was given has to be there until the object is dropped."""

    def __init__(self, cache: PagedCache, batch: int, num_heads: int, num_queries: int,
                 max_tokens: int, dtype=None, scale: float = 0.0, causal: bool = True,
                 weights: bool = False):
        torch = _torch()
        self.cache = cache
        self.dtype = torch.bfloat16 if dtype is None else dtype
        code = _dtype_code(torch.empty(0, dtype=self.dtype))
        D, G = cache.head_dim, cache.num_kv_heads
        self.batch, self.max_tokens, self.weights = batch, max_tokens, bool(weights)
        self._q_shape = (batch, num_heads, num_queries, D)
        self._w_shape = (batch, G)
        self._head = (batch, num_heads, num_queries, code, max_tokens)
        self._tail = (int(bool(causal)), int(self.weights), float(scale), 0)
        # strides of a dense call: the workspace does not depend on them
        rows = (num_heads * num_queries * D, num_queries * D, D)
        sh = _ATTEND.pack(*self._head, 1, *self._tail, 1, *rows, *rows, G * max_tokens, max_tokens,
                          G * max_tokens, max_tokens)
        n = ctypes.c_size_t(0)
        _raise(_LIB.e2s_cache_attend_workspace_size(cache.desc_ref, sh, ctypes.byref(n)),
               "e2s_cache_attend_workspace_size")
        self.workspace = torch.empty(int(n.value), device=cache.device, dtype=torch.uint8)
        # streams whose work the allocator waits for before it gives the workspace away
        self._index = cache.device.index
        self._streams = {_CURRENT_STREAM(self._index)}

    def _used_on(self, stream: int):
        torch = _torch()
        self.workspace.record_stream(torch.cuda.ExternalStream(stream, device=self.cache.device))
        self._streams.add(stream)

    def _weights(self, t, name):
        torch = _torch()
        _check(t, name, dtype=torch.float32, ndim=3, contiguous=False)
        st = t.stride()
        if tuple(t.shape[:2]) != self._w_shape or t.shape[2] < self.max_tokens or \
                (st[2] != 1 and t.shape[2] > 1):
            raise ValueError(f"{name} must be [{self._w_shape[0]}, {self._w_shape[1]}, >= "
                             f"{self.max_tokens}] with contiguous rows")
        return st[:2]

    def __call__(self, q, pages, lengths, out=None, q_count=None, weights_in=None,
                 weights_out=None, stream: Optional[int] = None):
        """q [B, H, T, d] against each sequence's lengths[b] cached tokens: (out, weights_out
        or None).  See e2s_cache_attend for q_count, weights_in and weights_out; outputs not
        given are allocated, zeros where the call leaves entries as they were.  There is no
        backward pass: where q asks for a gradient, `out` is not given and a backward pass
        through the outputs is an error."""
        torch = _torch()
        qs = _rows(q, "q", self.dtype)
        _no_tangents("attention over the 8-bit cache", q)
        if q.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("attention over the cache has no gradient for `out`: call it "
                                 "under torch.no_grad() or with detached queries")
            if self.weights and weights_out is None:
                return _Undifferentiated.apply(q, lambda: self(
                    q, pages, lengths, None, q_count, weights_in, None, stream))
            return _Undifferentiated.apply(q, lambda: self(
                q, pages, lengths, None, q_count, weights_in, weights_out, stream)[0]), weights_out
        if q.shape != self._q_shape:
            raise ValueError(f"q must be {list(self._q_shape)} (got {list(q.shape)})")
        width, row = _table(pages, "pages", self.batch)
        lengths_at = _vector(lengths, "lengths", self.batch)
        count_at = None if q_count is None else _vector(q_count, "q_count", self.batch)
        if out is None:
            with _allocating_on(stream, q.device):
                out = torch.empty_like(q) if q_count is None else torch.zeros_like(q)
            os_ = out.stride()
        else:
            os_ = _rows(out, "out", self.dtype)
            if out.shape != self._q_shape:
                raise ValueError("out must have q's shape")
        wi = wo = (0, 0)
        if self.weights:
            if weights_out is None:
                with _allocating_on(stream, q.device):
                    weights_out = torch.zeros(self._w_shape + (self.max_tokens,),
                                              device=q.device, dtype=torch.float32)
            wo = self._weights(weights_out, "weights_out")
            if weights_in is not None:
                wi = self._weights(weights_in, "weights_in")
        elif weights_in is not None or weights_out is not None:
            raise ValueError("this CacheAttention was made without weights")
        if stream is None:
            stream = _CURRENT_STREAM(self._index)
        if stream not in self._streams:
            self._used_on(stream)
        sh = _ATTEND.pack(*self._head, width, *self._tail, row, *qs[:3], *os_[:3], *wi, *wo)
        _launch("e2s_cache_attend",
                (self.workspace, q, pages, lengths, out, q_count, weights_in, weights_out),
                _LIB.e2s_cache_attend, self.cache.desc_ref, sh, pages.data_ptr(), lengths_at,
                count_at, q.data_ptr(), out.data_ptr(), _ptr(weights_in), _ptr(weights_out),
                self.workspace.data_ptr(), self.workspace.numel(), stream=stream)
        return out, weights_out


def cache_attend(q, cache: PagedCache, pages, lengths, max_tokens: Optional[int] = None,
                 scale: float = 0.0, causal: bool = True, out=None, q_count=None,
                 want_weights: bool = False, weights_in=None, weights_out=None,
                 stream: Optional[int] = None):
    """One CacheAttention call: (out, weights or None).  max_tokens: no length is larger
    (default: what the page table can hold)."""
    _rows(q, "q")
    _table(pages, "pages", q.shape[0])
    if max_tokens is None:
        max_tokens = pages.shape[1] * cache.page_tokens
    weights = want_weights or weights_in is not None or weights_out is not None
    with _allocating_on(stream, q.device):
        call = CacheAttention(cache, q.shape[0], q.shape[1], q.shape[2], max_tokens, q.dtype,
                              scale, causal, weights)
    return call(q, pages, lengths, out, q_count, weights_in, weights_out, stream)


def cache_evict(cache: PagedCache, pages, lengths, weights, new_pages, budget: int,
                sinks: int = 0, recent: int = 0, weights_left=None,
                stream: Optional[int] = None):
    """Every sequence and key head cut to its `budget` tokens of largest weight, the first
    `sinks` and the last `recent` among them (e2s_cache_evict): weights [B, Hkv, >= the
    longest length] float32; the kept rows go to new_pages [B, .] int32.  Returns (keep_idx
    [B, Hkv, budget] int32, ascending, then -1; new lengths [B] int32; the kept tokens'
    weights [B, Hkv, budget] or as given, zeros behind them)."""
    torch = _torch()
    G = cache.num_kv_heads
    if not (isinstance(weights, torch.Tensor) and weights.is_cuda and
            weights.dtype is torch.float32 and weights.dim() == 3):
        _check(weights, "weights", dtype=torch.float32, ndim=3, contiguous=False)
    (B, g, N), ws = weights.shape, weights.stride()
    if g != G or (ws[2] != 1 and N > 1):
        raise ValueError(f"weights must be [B, {G}, N] with contiguous rows")
    width, row = _table(pages, "pages", B)
    new_width, new_row = _table(new_pages, "new_pages", B)
    lengths_at = _vector(lengths, "lengths", B)
    K = max(budget, 0)
    with _allocating_on(stream, weights.device):
        keep, kept = lengths.new_empty((B, G, K)), torch.empty_like(lengths)
        left = weights.new_empty((B, G, K)) if weights_left is None else weights_left
    if weights_left is not None:
        _check(weights_left, "weights_left", dtype=torch.float32, ndim=3, contiguous=False)
        if tuple(weights_left.shape[:2]) != (B, G) or \
                (weights_left.stride(2) != 1 and weights_left.shape[2] > 1):
            raise ValueError(f"weights_left must be [{B}, {G}, >= budget] with contiguous rows")
    sh = _EVICT.pack(B, N, budget, sinks, recent, width, new_width, left.shape[2], row,
                     new_row, *ws[:2], *left.stride()[:2])
    _launch("e2s_cache_evict",
            (cache.k, pages, lengths, weights, new_pages, keep, kept, left),
            _LIB.e2s_cache_evict, cache.desc_ref, sh, pages.data_ptr(), lengths_at,
            weights.data_ptr(), new_pages.data_ptr(), keep.data_ptr(), kept.data_ptr(),
            left.data_ptr(), stream=stream)
    return keep, kept, left
