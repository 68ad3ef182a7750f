"""ctypes binding of what a layer's step takes beside the operators of _serve (the C ABI
declared in include/e2s_step.h): norms of heads with the rotation of their positions, and
the paged 4-bit key/value cache.

Argument marshalling only, as in ``_serve``: functions with the C names minus the ``e2s_``
prefix take torch tensors on the GPU, allocate what they return, pass raw device pointers
and the current torch stream, and raise ``E2SError`` on a non-zero status.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

from . import _lib
from ._lib import _CURRENT_STREAM, _check, _dtype_code, _launch, _ptr, _raise, _torch
from ._serve import (_I32, _I64, _P, RotaryPlan, _allocating_on, _Function, _like, _moved,
                     _no_tangents, _ref, _rows, _table, _vector)

HEADER = os.path.join(os.path.dirname(_lib.PKG), "include", "e2s_step.h")


class NormRotateShape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_tokens", _I32), ("q_heads", _I32), ("k_heads", _I32),
                ("dtype", _I32), ("weight_dtype", _I32), ("eps", ctypes.c_float),
                ("reserved", _I32), ("q_stride", _I64 * 3), ("k_stride", _I64 * 3),
                ("q_grad_stride", _I64 * 3), ("k_grad_stride", _I64 * 3),
                ("q_out_stride", _I64 * 3), ("k_out_stride", _I64 * 3), ("pos_stride", _I64 * 3)]


class Cache4Desc(ctypes.Structure):
    """e2s_cache4."""
    _fields_ = [("num_pages", _I32), ("page_tokens", _I32), ("num_kv_heads", _I32),
                ("head_dim", _I32), ("k_page_stride", _I64), ("v_page_stride", _I64), ("k", _P),
                ("v", _P), ("k_scale", _P), ("v_scale", _P)]


class Read4Shape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_tokens", _I32), ("dtype", _I32), ("max_pages", _I32),
                ("pages_stride", _I64), ("k_out_stride", _I64 * 3), ("v_out_stride", _I64 * 3)]


class Attend4Shape(ctypes.Structure):
    _fields_ = [("batch", _I32), ("num_heads", _I32), ("num_queries", _I32), ("dtype", _I32),
                ("max_tokens", _I32), ("max_pages", _I32), ("causal", _I32),
                ("scale", ctypes.c_float), ("pages_stride", _I64), ("q_stride", _I64 * 3),
                ("out_stride", _I64 * 3)]


SIGNATURES = {
    "e2s_norm_rotate": [_P, _ref(RotaryPlan)] + [_P] * 8,
    "e2s_norm_rotate_backward_workspace_size": [_P, _ref(RotaryPlan), _I32,
                                                _ref(ctypes.c_size_t)],
    "e2s_norm_rotate_backward": [_P, _ref(RotaryPlan)] + [_P] * 12 + [ctypes.c_size_t, _P],
    "e2s_cache4_append": [_ref(Cache4Desc), _P, _P, _P, _P, _P, _P, _P, _P],
    "e2s_cache4_read": [_ref(Cache4Desc), _P, _P, _P, _P, _P, _P, _P],
    "e2s_cache4_attend_workspace_size": [_ref(Cache4Desc), _P, _ref(ctypes.c_size_t)],
    "e2s_cache4_attend": [_ref(Cache4Desc), _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P],
    "e2s_step_abi_version": [],
}
for _name, _args in SIGNATURES.items():
    _fn = getattr(_lib.lib(), _name)
    _fn.argtypes, _fn.restype = _args, ctypes.c_int
_LIB = _lib.lib()

# the records in their layout (native sizes and alignment), packed in one call
_NORM = struct.Struct("@6ifi21q")
_APPEND = struct.Struct("@6i7q")
_READ = struct.Struct("@4i7q")
_ATTEND = struct.Struct("@7if7q")


# ---------------------------------------------------------------------------
# norms and positions
# ---------------------------------------------------------------------------

def _weight(w, name, x, D):
    """The address of a norm's weight: [d], of the rows' type or float32."""
    torch = _torch()
    if w is None:
        return None
    if not (isinstance(w, torch.Tensor) and w.is_cuda and w.dim() == 1 and w.is_contiguous()):
        _check(w, name, ndim=1)
    if w.dtype is not x.dtype and w.dtype is not torch.float32:
        raise TypeError(f"{name} must be {x.dtype} or torch.float32 (got {w.dtype})")
    if w.shape[0] != D:
        raise ValueError(f"{name} must be [{D}] (got {tuple(w.shape)})")
    return w.data_ptr()


def _weight_code(q_weight, k_weight, code):
    """The weights' one dtype."""
    w = k_weight if q_weight is None else q_weight
    if w is None:
        return code
    if k_weight is not None and k_weight.dtype is not w.dtype:
        raise TypeError("q_weight and k_weight must be of one type")
    return 0 if w.dtype is _torch().float32 else code


def _positions(positions, plan, B, T):
    """The axis, sequence and token strides of a plan's positions."""
    torch = _torch()
    if not (isinstance(positions, torch.Tensor) and positions.is_cuda and
            positions.dtype is torch.int32):
        _check(positions, "positions", dtype=torch.int32, contiguous=False)
    lead = (3,) if plan.axes == 3 else ()
    shape, ps = positions.shape, positions.stride()
    if shape == lead + (B, T):
        return (ps[0] if lead else 0, ps[-2], ps[-1])
    if shape == lead + (T,):
        return (ps[0] if lead else 0, 0, ps[-1])
    raise ValueError(f"positions must be {list(lead + (T,))} or {list(lead + (B, T))} "
                     f"(got {list(shape)})")


_NONE = (0, 0, 0)


def _made_like(t, stream):
    """An output beside t, its rows contiguous, and its strides."""
    torch = _torch()
    o = _like(t, stream) if stream is not None else torch.empty_like(t)
    st = o.stride()
    if st[3] != 1:                       # rows one element apart: torch may order them first
        o = _like(t, stream, torch.contiguous_format)
        st = o.stride()
    return o, st[:3]


def _inputs(q, k, positions, plan, q_weight, k_weight, eps):
    """The checked inputs of a call: the head of its record, q's and k's strides, those of the
    positions, and the weights' addresses."""
    x = q if q is not None else k
    D = plan.head_dim
    heads, strides = [], []
    for t, name in ((q, "q"), (k, "k")):
        if t is None:
            heads.append(0)
            strides += _NONE
            continue
        strides += _rows(t, name, x.dtype)[:3]
        shape = t.shape
        if shape[0] != x.shape[0] or shape[2] != x.shape[2] or shape[3] != D:
            raise ValueError(f"{name} {tuple(shape)} must be [B, heads, T, {D}] with one B and T")
        heads.append(shape[1])
    B, T = x.shape[0], x.shape[2]
    ps = _positions(positions, plan, B, T)
    weights = _weight(q_weight, "q_weight", x, D), _weight(k_weight, "k_weight", x, D)
    code = _dtype_code(x)
    return ((B, T, *heads, code, _weight_code(q_weight, k_weight, code), eps, 0), strides, ps,
            weights)


def _forward(inputs, q, k, positions, plan, q_weight, k_weight, q_out, k_out, stream):
    head, strides, ps, weights = inputs
    out_strides, outs = [], []
    for i, (t, name, o) in enumerate(((q, "q", q_out), (k, "k", k_out))):
        if t is None:
            if o is not None:
                raise ValueError(f"{name}_out without {name}")
            out_strides += _NONE
        elif o is None:
            o, st = _made_like(t, stream)
            out_strides += st
        else:
            st = _rows(o, name + "_out", t.dtype)[:3]
            if o.shape != t.shape:
                raise ValueError(f"{name}_out must have {name}'s shape")
            if o.data_ptr() == t.data_ptr() and \
                    _moved(t.shape, tuple(strides[3 * i:3 * i + 3]), st):
                raise ValueError(f"{name}_out in the place of {name} must have its strides")
            out_strides += st
        outs.append(o)
    if head[0] > 0 and head[1] > 0:
        sh = _NORM.pack(*head, *strides, *_NONE, *_NONE, *out_strides, *ps)
        _launch("e2s_norm_rotate", (q, k, positions, q_weight, k_weight, *outs),
                _LIB.e2s_norm_rotate, sh, ctypes.byref(plan), positions.data_ptr(), _ptr(q),
                _ptr(k), *weights, _ptr(outs[0]), _ptr(outs[1]), stream=stream)
    return outs[0], outs[1]


def _backward(inputs, q_grad, k_grad, q, k, positions, plan, q_weight, k_weight, want, stream):
    """want: which weights' gradients."""
    torch = _torch()
    head, strides, ps, weights = inputs
    B, T = head[:2]
    grad_strides, out_strides, outs = [], [], []
    for t, g, name in ((q, q_grad, "q"), (k, k_grad, "k")):
        if t is None:
            grad_strides += _NONE
            out_strides += _NONE
            outs.append(None)
            continue
        grad_strides += _rows(g, name + "_grad", t.dtype)[:3]
        if g.shape != t.shape:
            raise ValueError(f"{name}_grad must have {name}'s shape")
        o, st = _made_like(t, stream)
        out_strides += st
        outs.append(o)
    x = q if q is not None else k
    dqw = dkw = work = None
    size = 0
    if want[0] or want[1]:
        with _allocating_on(stream, x.device):
            make = torch.empty_like if B > 0 and T > 0 else torch.zeros_like
            dqw = make(q_weight) if want[0] else None
            dkw = make(k_weight) if want[1] else None
    if B > 0 and T > 0:
        sh = _NORM.pack(*head, *strides, *grad_strides, *out_strides, *ps)
        plan_ref = ctypes.byref(plan)
        if want[0] or want[1]:
            n = ctypes.c_size_t(0)
            _raise(_LIB.e2s_norm_rotate_backward_workspace_size(sh, plan_ref, 1, ctypes.byref(n)),
                   "e2s_norm_rotate_backward_workspace_size")
            size = n.value
            with _allocating_on(stream, x.device):
                work = torch.empty(size, device=x.device, dtype=torch.uint8)
        _launch("e2s_norm_rotate_backward",
                (q, k, positions, q_weight, k_weight, q_grad, k_grad, *outs, dqw, dkw, work),
                _LIB.e2s_norm_rotate_backward, sh, plan_ref, positions.data_ptr(), _ptr(q),
                _ptr(k), *weights, _ptr(q_grad), _ptr(k_grad), _ptr(outs[0]), _ptr(outs[1]),
                _ptr(dqw), _ptr(dkw), _ptr(work), size, stream=stream)
    return outs[0], outs[1], dqw, dkw


def _whole_rows(t):
    """t, or a copy where its rows are not contiguous (a broadcast gradient's are not)."""
    if t.stride(3) == 1 or t.shape[3] == 1:
        return t
    return t.clone(memory_format=_torch().contiguous_format)


class _NormRotate(_Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, plan, eps):
        inputs = _inputs(q, k, positions, plan, q_weight, k_weight, eps)
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        ctx.plan, ctx.eps = plan, eps
        ctx.set_materialize_grads(False)
        return _forward(inputs, q, k, positions, plan, q_weight, k_weight, None, None, None)

    @staticmethod
    def backward(ctx, q_grad, k_grad):
        if _torch().is_grad_enabled():
            raise RuntimeError("norm_rotate has no second derivative: take its gradients "
                               "without create_graph")
        need_q, need_k, need_qw, need_kw = ctx.needs_input_grad[:4]
        if not (need_q or need_qw):
            q_grad = None
        if not (need_k or need_kw):
            k_grad = None
        if q_grad is None and k_grad is None:
            return (None,) * 7
        # What is unpacked need not be what was saved: a hook gives copies, which have strides of
        # their own, and a checkpoint makes tensors again.  So nothing that forward learned of
        # their memory is used: the record is made, and checked, from the tensors in hand.
        q, k, q_weight, k_weight, positions = ctx.saved_tensors
        # (a tensor whose output has no gradient takes no part)
        q, q_grad = (None, None) if q_grad is None else (_whole_rows(q), _whole_rows(q_grad))
        k, k_grad = (None, None) if k_grad is None else (_whole_rows(k), _whole_rows(k_grad))
        inputs = _inputs(q, k, positions, ctx.plan, q_weight, k_weight, ctx.eps)
        dq, dk, dqw, dkw = _backward(inputs, q_grad, k_grad, q, k, positions, ctx.plan, q_weight,
                                     k_weight, (need_qw and q is not None,
                                                need_kw and k is not None), None)
        return (dq if need_q else None, dk if need_k else None, dqw, dkw, None, None, None)


def norm_rotate(q, k, positions, plan: RotaryPlan, q_weight=None, k_weight=None,
                eps: float = 1e-6, q_out=None, k_out=None, stream: Optional[int] = None):
    """q [B, H, T, d] and k [B, Hkv, T, d] (either may be None; any strides with contiguous
    rows), every row divided by its root mean square (eps within the root), times its
    tensor's weight ([d], of the rows' type or float32, or None), and turned by `positions`
    as rotate_positions does (e2s_norm_rotate).  Returns (q_out, k_out); an output may be its
    input.  Outputs that are not given have a gradient where q, k or a weight asks for one
    (a first one: its own gradient is an error, as are tangents of forward-mode
    differentiation)."""
    torch = _torch()
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k is needed")
    _no_tangents("norm_rotate", q, k, q_weight, k_weight)
    if torch.is_grad_enabled() and (x.requires_grad or (k is not None and k.requires_grad) or
                                    (q_weight is not None and q_weight.requires_grad) or
                                    (k_weight is not None and k_weight.requires_grad)):
        if q_out is not None or k_out is not None:
            raise ValueError("an output that is given has no gradient: give none, or call "
                             "under torch.no_grad()")
        with _allocating_on(stream, x.device):
            return _NormRotate.apply(q, k, q_weight, k_weight, positions, plan, eps)
    inputs = _inputs(q, k, positions, plan, q_weight, k_weight, eps)
    return _forward(inputs, q, k, positions, plan, q_weight, k_weight, q_out, k_out, stream)


def norm_rotate_backward(q_grad, k_grad, q, k, positions, plan: RotaryPlan, q_weight=None,
                         k_weight=None, eps: float = 1e-6, want_q_weight: bool = True,
                         want_k_weight: bool = True, stream: Optional[int] = None):
    """The gradients of norm_rotate's inputs from those of its outputs
    (e2s_norm_rotate_backward): (q's, k's, q_weight's, k_weight's), None for a tensor or weight
    that is None, and for the weight of a tensor that is.  want_q_weight, want_k_weight: False
    leaves that weight's out.  It keeps no state, so it may be captured in a graph by itself;
    autograd calls it."""
    if q is None and k is None:
        raise ValueError("q or k is needed")
    for t, g, name in ((q, q_grad, "q"), (k, k_grad, "k")):
        if (t is None) != (g is None):
            raise ValueError(f"{name} and {name}_grad go together")
    _no_tangents("norm_rotate_backward", q_grad, k_grad, q, k, q_weight, k_weight)
    inputs = _inputs(q, k, positions, plan, q_weight, k_weight, eps)
    want = (q_weight is not None and q is not None and want_q_weight,
            k_weight is not None and k is not None and want_k_weight)
    return _backward(inputs, q_grad, k_grad, q, k, positions, plan, q_weight, k_weight, want,
                     stream)


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------

class PagedCache4:
    """The 4-bit cache of one layer (e2s_cache4), by the tables that the header lays out:
    k [num_pages, Hkv, P, d/2] and v [num_pages, Hkv, P/32, d, 16] uint8, two elements to a
    byte; k_scale [num_pages, Hkv, P/16, 4, d/32, 4] uint8, exponents + 127; v_scale
    [num_pages, Hkv, P] bfloat16.  Which sequence a page belongs to is the caller's page
    table's to say."""

    def __init__(self, num_pages: int, num_kv_heads: int, head_dim: int, page_tokens: int = 64,
                 device="cuda"):
        torch = _torch()
        lead = (num_pages, num_kv_heads)
        k, v, ks = (torch.zeros(lead + s, dtype=torch.uint8, device=device) for s in (
            (page_tokens, head_dim // 2), (page_tokens // 32, head_dim, 16),
            (page_tokens // 16, 4, head_dim // 32, 4)))
        vs = torch.ones(lead + (page_tokens,), dtype=torch.bfloat16, device=device)
        self._hold(k, ks + 127, v, vs)

    @classmethod
    def of(cls, k, k_scale, v, v_scale) -> "PagedCache4":
        """A cache in memory that the caller allocated; the pages of k and v may lie apart (a
        pool that holds every layer's pages), what is in a page may not."""
        self = cls.__new__(cls)
        self._hold(k, k_scale, v, v_scale)
        return self

    def _hold(self, k, k_scale, v, v_scale):
        torch = _torch()
        _check(k, "k", dtype=torch.uint8, ndim=4, contiguous=False)
        _check(v, "v", dtype=torch.uint8, ndim=5, contiguous=False)
        pages, G, P, half = k.shape
        if k.numel() == 0 or P % 32 != 0 or half % 16 != 0:
            raise ValueError("k must be [num_pages, Hkv, P, d/2], not empty, P and d multiples "
                             "of 32")
        if tuple(v.shape) != (pages, G, P // 32, 2 * half, 16):
            raise ValueError("v must be [num_pages, Hkv, P/32, d, 16]")
        for t, name in ((k, "k"), (v, "v")):
            if not t[0].is_contiguous():
                raise ValueError(f"a page of {name} must be contiguous")
        _check(k_scale, "k_scale", dtype=torch.uint8, ndim=6)
        _check(v_scale, "v_scale", dtype=torch.bfloat16, ndim=3)
        if tuple(k_scale.shape) != (pages, G, P // 16, 4, half // 16, 4):
            raise ValueError("k_scale must be [num_pages, Hkv, P/16, 4, d/32, 4]")
        if tuple(v_scale.shape) != (pages, G, P):
            raise ValueError("v_scale must be [num_pages, Hkv, P]")
        _lib._device_of(k, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.num_kv_heads, self.page_tokens, self.head_dim = pages, G, P, 2 * half
        self.device = k.device
        st = [t.stride(0) if pages > 1 else t[0].numel() for t in (k, v)]
        self.desc = Cache4Desc(pages, P, G, 2 * half, st[0], st[1], k.data_ptr(), v.data_ptr(),
                               k_scale.data_ptr(), v_scale.data_ptr())
        self.desc_ref = ctypes.byref(self.desc)


def cache4_append(cache: PagedCache4, pages, start, k, v, count=None, src_idx=None,
                  stream: Optional[int] = None):
    """New tokens into the 4-bit cache (e2s_cache4_append).  k, v [B, Hkv, N, d] (any strides
    with 16-byte aligned rows) hold sequence b's tokens start[b], start[b] + 1, ...: all N,
    the first count[b], or the rows that src_idx [B, T] int32 names (e.g. prune()'s
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
    _launch("e2s_cache4_append", (cache.k, pages, start, k, v, count, src_idx),
            _LIB.e2s_cache4_append, cache.desc_ref, sh, pages.data_ptr(), start_at, count_at,
            _ptr(src_idx), k.data_ptr(), v.data_ptr(), stream=stream)


def cache4_read(cache: PagedCache4, pages, start, num_tokens: int, count=None, dtype=None,
                k_out=None, v_out=None, stream: Optional[int] = None):
    """The held keys and values of every sequence's tokens start[b] .. start[b] + num_tokens,
    or the first count[b] of them (e2s_cache4_read): (k, v) [B, Hkv, num_tokens, d] of dtype
    (default bfloat16; float32 holds them exactly).  Outputs not given are allocated, zeros
    where the call leaves rows as they were."""
    torch = _torch()
    if not isinstance(pages, torch.Tensor) or pages.dim() != 2:
        _check(pages, "pages", dtype=torch.int32, ndim=2, contiguous=False)
    B = pages.shape[0]
    width, row = _table(pages, "pages", B)
    start_at = _vector(start, "start", B)
    count_at = None if count is None else _vector(count, "count", B)
    given = next((t for t in (k_out, v_out) if t is not None), None)
    if dtype is None:
        dtype = torch.bfloat16 if given is None else given.dtype
    shape = (B, cache.num_kv_heads, num_tokens, cache.head_dim)
    outs, strides = [], []
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        if t is None:
            with _allocating_on(stream, cache.device):
                t = (torch.empty if count is None else torch.zeros)(shape, dtype=dtype,
                                                                    device=cache.device)
        st = _rows(t, name, dtype)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {list(shape)} (got {list(t.shape)})")
        outs.append(t)
        strides += st[:3]
    if B == 0 or num_tokens == 0:
        return outs[0], outs[1]
    sh = _READ.pack(B, num_tokens, _dtype_code(outs[0]), width, row, *strides)
    _launch("e2s_cache4_read", (cache.k, pages, start, count, *outs), _LIB.e2s_cache4_read,
            cache.desc_ref, sh, pages.data_ptr(), start_at, count_at, outs[0].data_ptr(),
            outs[1].data_ptr(), stream=stream)
    return outs[0], outs[1]


class _Undifferentiated4(_Function):
    """The output of call(), whose gradient is asked for in vain: an error says so where it
    would otherwise be lost."""

    @staticmethod
    def forward(ctx, q, call):
        return call()

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("attention over the 4-bit cache has no backward pass: call it under "
                           "torch.no_grad() or with detached queries")


class Cache4Attention:
    """Repeated e2s_cache4_attend calls of one shape: `batch` sequences of at most
    `max_tokens` cached tokens and `num_queries` queries.  It holds the workspace, so calls
    of one object on several streams are the caller's to order, and a stream that a call was
    given has to be there until the object is dropped."""

    def __init__(self, cache: PagedCache4, batch: int, num_heads: int, num_queries: int,
                 max_tokens: int, dtype=None, scale: float = 0.0, causal: bool = True):
        torch = _torch()
        self.cache = cache
        self.dtype = torch.bfloat16 if dtype is None else dtype
        code = _dtype_code(torch.empty(0, dtype=self.dtype))
        D = cache.head_dim
        self.batch, self.max_tokens = batch, max_tokens
        self._q_shape = (batch, num_heads, num_queries, D)
        self._head = (batch, num_heads, num_queries, code, max_tokens)
        self._tail = (int(bool(causal)), float(scale))
        # strides of a dense call: the workspace does not depend on them
        rows = (num_heads * num_queries * D, num_queries * D, D)
        sh = _ATTEND.pack(*self._head, 1, *self._tail, 1, *rows, *rows)
        n = ctypes.c_size_t(0)
        _raise(_LIB.e2s_cache4_attend_workspace_size(cache.desc_ref, sh, ctypes.byref(n)),
               "e2s_cache4_attend_workspace_size")
        self.workspace = torch.empty(int(n.value), device=cache.device, dtype=torch.uint8)
        # streams whose work the allocator waits for before it gives the workspace away
        self._index = cache.device.index
        self._streams = {_CURRENT_STREAM(self._index)}

    def _used_on(self, stream: int):
        torch = _torch()
        self.workspace.record_stream(torch.cuda.ExternalStream(stream, device=self.cache.device))
        self._streams.add(stream)

    def __call__(self, q, pages, lengths, out=None, q_count=None, stream: Optional[int] = None):
        """q [B, H, T, d] against each sequence's lengths[b] cached tokens: out.  See
        e2s_cache4_attend for q_count; an output not given is allocated, zeros where the call
        leaves rows as they were.  There is no backward pass: where q asks for a gradient,
        `out` is not given and a backward pass through the output is an error."""
        torch = _torch()
        qs = _rows(q, "q", self.dtype)
        _no_tangents("attention over the 4-bit cache", q)
        if q.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("attention over the cache has no gradient for `out`: call it "
                                 "under torch.no_grad() or with detached queries")
            return _Undifferentiated4.apply(
                q, lambda: self(q, pages, lengths, None, q_count, stream))
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
        if stream is None:
            stream = _CURRENT_STREAM(self._index)
        if stream not in self._streams:
            self._used_on(stream)
        sh = _ATTEND.pack(*self._head, width, *self._tail, row, *qs[:3], *os_[:3])
        _launch("e2s_cache4_attend", (self.workspace, q, pages, lengths, out, q_count),
                _LIB.e2s_cache4_attend, self.cache.desc_ref, sh, pages.data_ptr(), lengths_at,
                count_at, q.data_ptr(), out.data_ptr(), self.workspace.data_ptr(),
                self.workspace.numel(), stream=stream)
        return out


def cache4_attend(q, cache: PagedCache4, pages, lengths, max_tokens: Optional[int] = None,
                  scale: float = 0.0, causal: bool = True, out=None, q_count=None,
                  stream: Optional[int] = None):
    """One Cache4Attention call: out.  max_tokens: no length is larger (default: what the
    page table can hold)."""
    _rows(q, "q")
    _table(pages, "pages", q.shape[0])
    if max_tokens is None:
        max_tokens = pages.shape[1] * cache.page_tokens
    with _allocating_on(stream, q.device):
        call = Cache4Attention(cache, q.shape[0], q.shape[1], q.shape[2], max_tokens, q.dtype,
                               scale, causal)
    return call(q, pages, lengths, out, q_count, stream)
