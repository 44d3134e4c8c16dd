"""Operators of a regularised feed-forward block: argument marshalling and
autograd plumbing only; every step runs in libslorr.so.

  gated_ffn          y = (act(x Wg^T) * (x Wu^T)) Wd^T
  block_norm         RMS or layer norm of a block's input
  block_join         y = x + alpha * scale * gate * dropout(norm(f)) and the next
                     block's norm of y, in one kernel
  dropout            dropout from a counter-based generator; no mask is stored
  FeedForwardBlock   these as a module, whose projections are the weights that
                     Regularizer and DecoupledSlorr take

Tensors are float32 or bfloat16, all of a call of one dtype, on one GPU; the
last dimension is the row. Activations may be strided (a layout that the
kernels do not read in place is copied); weights are contiguous (one that does
not start at a multiple of 16 bytes is copied in every call). Calls run on
the current stream of the tensors' device and can be captured into a graph.
Gradients are formed for the inputs that require them. Each is written anew by
fixed-order sums: no atomics, so results repeat bit for bit. They can be taken
once: differentiating them again raises RuntimeError, and so do forward-mode
derivatives and tracing (torch.jit.trace, make_fx); torch.compile ends its graphs
where they stand. To capture a
backward() into a graph, let no eager graph of the same leaves live: torch would
tie the capture to the stream of the older graph.

Dropout draws its numbers from rng, an int64 tensor (key, offset) on the device,
and an integer site that sets the calls of one step apart. The backward pass
draws them again, so rng keeps its values until then: a training loop advances
the offset once per step, by more than its largest site.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct
import weakref
from typing import List, NamedTuple, Optional, Tuple

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import check, lib

__all__ = ["gated_ffn", "block_norm", "block_join", "dropout", "FeedForwardBlock"]

_DTYPE = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}
_ACT = {"silu": _lib.SILU, "gelu": _lib.GELU, "gelu_tanh": _lib.GELU_TANH}
_NORM = {"rms": _lib.RMS, "layer": _lib.LAYER}
_MAX_STRIDE = (1 << 22) - 8
_MAX_NORM = 8192
_MOST_F32 = (2.0 - 2.0 ** -23) * 2.0 ** 127
_MOST_P = (65535.5 - 2.0 ** -20) / 65536          # p counts in steps of 2^-16


_is_tracing = getattr(torch._C, "_is_tracing", torch.jit.is_tracing)           # (without its Python frame)
_modes = getattr(torch._C, "_len_torch_dispatch_stack", lambda: 0)


def _check_transforms(*tensors) -> None:
    """Refuses what cannot see the kernels: forward-mode derivatives, whose tangents
    would be lost, and traces, which would hold the outputs' allocation alone."""
    if _is_tracing() or (_modes() and torch._C._get_dispatch_mode(torch._C._TorchDispatchModeKey.PROXY) is not None):
        raise RuntimeError("the block operators cannot be traced (a captured graph holds them)")
    if getattr(forward_ad, "_current_level", 0) >= 0:
        for t in tensors:
            if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
                raise RuntimeError("the block operators have no forward-mode derivative")


def _check_first(x: torch.Tensor, name: str) -> None:
    if not isinstance(x, torch.Tensor) or x.dtype not in _DTYPE:
        raise ValueError(f"{name} must be a float32 or bfloat16 tensor")
    if not x.is_cuda:
        raise ValueError(f"{name} must be on a GPU")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"{name} must have a last dimension of at least 1")


def _check_like(t: torch.Tensor, shape, x: torch.Tensor, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype != x.dtype or t.device != x.device:
        raise ValueError(f"{name} must be a {x.dtype} {tuple(shape)} tensor on {x.device}")


def _check_dense(t: torch.Tensor, shape, x: torch.Tensor, name: str) -> None:
    _check_like(t, shape, x, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _rows(t: torch.Tensor, dim: int) -> Tuple[torch.Tensor, int]:
    """t's values as rows of dim at a fixed stride, 16-byte aligned: the tensor
    to read (t itself where it is laid out so) and the stride."""
    if t.is_contiguous():
        return (t, dim) if t.data_ptr() % 16 == 0 else (t.clone(), dim)
    m = t.reshape(-1, dim)
    n, ld = m.shape[0], m.stride(0)
    if (dim > 1 and m.stride(1) != 1) or (n > 1 and not dim <= ld <= _MAX_STRIDE) or m.data_ptr() % 16:
        m = m.clone(memory_format=torch.contiguous_format)
        ld = dim
    return m, ld if n > 1 else dim


class _Once(torch.autograd.Function):
    """Gradients as they are, which refuse to be differentiated (anchor requires a gradient)."""

    @staticmethod
    def forward(ctx, anchor, *grads):
        return grads

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the block operators' gradients can be taken once only")


def _once(backward):
    """A backward pass whose results, where a graph of them is asked for (create_graph), end in _Once."""

    def run(ctx, *grads):
        _check_transforms(*grads)
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        with torch.no_grad():
            out = backward(ctx, *grads)
        return _Once.apply(torch.empty(0, requires_grad=True), *out)

    return run


_HERE = contextlib.nullcontext()


def _device(t: torch.Tensor):
    """t's device as the current one (nothing to do where it is)."""
    return _HERE if torch.cuda.current_device() == t.device.index else torch.cuda.device(t.device)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # current_stream() without its Stream object


def _stream(t: torch.Tensor) -> int:
    return _raw_stream(t.device.index) if _raw_stream else torch.cuda.current_stream(t.device).cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    p = t.data_ptr()
    if not p and t.numel():                       # (to the library a null pointer is an absent tensor)
        raise ValueError("a tensor has no memory")
    return p


def _returned(t: torch.Tensor, shape, dtype: torch.dtype, device: int) -> torch.Tensor:
    """A saved tensor as it comes back. saved_tensors_hooks may return another one, at another address and in
    another layout: the backward calls lay the tensors out again. Anything else about it has to be as it was."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        raise RuntimeError(f"a saved tensor of {dtype} {tuple(shape)} came back as {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _returned_dense(t: Optional[torch.Tensor], *of) -> Optional[torch.Tensor]:
    """The same of a tensor that is read as contiguous (None: none was saved)."""
    return None if t is None else _aligned(_returned(t, *of))


def _bytes(n: int, like: torch.Tensor) -> torch.Tensor:
    return like.new_empty(n, dtype=torch.uint8)


def _new(shape, like: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of that shape (empty_like where it can be: the shortest way to one)."""
    return torch.empty_like(like) if like.shape == shape and like.is_contiguous() else like.new_empty(shape)


# ------------------------------------------------------------- feed-forward

def _ffn_block(x, ldx, w_gate, act, lddy=0):
    inner, dim = w_gate.shape
    return _lib.Ffn(x.numel() // dim, dim, inner, _DTYPE[x.dtype], act, ldx, lddy)


def _at16(t):
    """t, or a copy where its values do not start at a multiple of 16 bytes."""
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _ffn_forward(x, shape, ldx, w_gate, w_up, w_down, act, keep):
    """y and, with keep, the state of the backward pass. x is laid out by _rows."""
    with _device(x):
        w_gate, w_up, w_down = _at16(w_gate), _at16(w_up), _at16(w_down)
        d = _ffn_block(x, ldx, w_gate, act)
        st, ws = ctypes.c_size_t(), ctypes.c_size_t()
        check(lib().slorr_ffn_sizes(d, st, ws, None), "slorr_ffn_sizes")
        y = _new(shape, x)
        state = _bytes(st.value, x) if keep else None
        work = _bytes(ws.value, x)
        check(lib().slorr_ffn_forward(d, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
                                      y.data_ptr(), _ptr(state), work.data_ptr(), ws.value, _stream(x)),
              "slorr_ffn_forward")
    return y, state


class _GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act):
        rows, ldx = _rows(x, w_gate.shape[1])
        y, state = _ffn_forward(rows, x.shape, ldx, w_gate, w_up, w_down, act, True)
        ctx.act, ctx.shape, ctx.laid, ctx.inner, ctx.state_bytes = act, x.shape, rows.shape, w_gate.shape[0], state.shape
        ctx.save_for_backward(rows, w_gate, w_up, w_down, state)
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, state = ctx.saved_tensors
        need, dim, inner, of = ctx.needs_input_grad, ctx.shape[-1], ctx.inner, (dy.dtype, dy.get_device())
        with _device(dy):
            x, ldx = _rows(_returned(x, ctx.laid, *of), dim)
            w_gate, w_up = _returned_dense(w_gate, (inner, dim), *of), _returned_dense(w_up, (inner, dim), *of)
            w_down = _returned_dense(w_down, (dim, inner), *of)
            state = _returned_dense(state, ctx.state_bytes, torch.uint8, of[1])
            dy, lddy = _rows(dy, dim)
            d = _ffn_block(x, ldx, w_gate, ctx.act, lddy)
            ws = ctypes.c_size_t()
            check(lib().slorr_ffn_sizes(d, None, None, ws), "slorr_ffn_sizes")
            grads = [_new(ctx.shape, x) if need[0] else None]
            grads += [torch.empty_like(w) if n else None for w, n in zip((w_gate, w_up, w_down), need[1:])]
            work = _bytes(ws.value, x)
            check(lib().slorr_ffn_backward(d, dy.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(),
                                           w_down.data_ptr(), state.data_ptr(), *map(_ptr, grads), work.data_ptr(),
                                           ws.value, _stream(x)), "slorr_ffn_backward")
        return (*grads, None)


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
              act: str = "silu") -> torch.Tensor:
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T over the rows of x (..., dim).

    w_gate, w_up: (inner, dim), w_down: (dim, inner), contiguous. act: "silu",
    "gelu" or "gelu_tanh". In bfloat16 the inner activations are rounded to
    bfloat16 between the products. In float32 an infinity comes out as a NaN,
    but for calls of up to 64 tokens without gradients, where it stays one.
    Without gradients nothing is kept."""
    _check_transforms(x, w_gate, w_up, w_down)
    _check_first(x, "x")
    if act not in _ACT:
        raise ValueError(f"act must be one of {list(_ACT)}")
    dim = x.shape[-1]
    if not isinstance(w_gate, torch.Tensor) or w_gate.dim() != 2 or w_gate.shape[0] < 1:
        raise ValueError("w_gate must be a matrix of at least one row")
    inner = w_gate.shape[0]
    _check_dense(w_gate, (inner, dim), x, "w_gate")
    _check_dense(w_up, (inner, dim), x, "w_up")
    _check_dense(w_down, (dim, inner), x, "w_down")
    if torch.is_grad_enabled() and (x.requires_grad or w_gate.requires_grad or w_up.requires_grad
                                    or w_down.requires_grad):
        return _GatedFfn.apply(x, w_gate, w_up, w_down, _ACT[act])
    rows, ldx = _rows(x, dim)
    return _ffn_forward(rows, x.shape, ldx, w_gate, w_up, w_down, _ACT[act], False)[0]


# --------------------------------------------------------------------- join

_JOIN = ("x", "f", "post_weight", "post_bias", "gate", "scale", "pre_weight", "pre_bias")
_ROWS, _VECTORS = (0, 1, 4), (2, 3, 5, 6, 7)


class _Call(NamedTuple):
    """A join without its tensors. (A plain tuple: torch.compile, which splits these functions, loses a ctypes
    structure's values on the way from one to the next.)"""
    rows: int
    dim: int
    dtype: int
    norm: int
    flags: int
    gate_rows: int
    eps: float
    alpha: float
    p: float
    site: int

    def struct(self, strides):
        return _lib.Join.from_buffer_copy(_PACKED.pack(*self[:6], *strides, *self[6:]))


_PACKED = struct.Struct("@qiiiIqqqqffdq")           # _lib.Join: packed at half of what its constructor takes
assert _PACKED.size == ctypes.sizeof(_lib.Join)


def _join_run(d: _Call, shape, tensors, strides, rng):
    """The forward call on laid-out inputs: y (None without f), z (None without PRE) and the inputs' addresses."""
    x, at = tensors[0], [*map(_ptr, tensors)]
    with _device(x):
        y = None if tensors[1] is None else _new(shape, x)
        z = _new(shape, x) if d.flags & _lib.JOIN_PRE else None
        check(lib().slorr_join_forward(d.struct(strides), _lib.JoinTensors(*at), _ptr(rng), _ptr(y), _ptr(z),
                                       _stream(x)), "slorr_join_forward")
    return y, z, at


class _Join(torch.autograd.Function):
    """forward(d, rng, *tensors): d describes the call, tensors in the order of
    _JOIN. Returns (y, z), or what there is of them."""

    @staticmethod
    def forward(ctx, d, rng, *tensors):
        laid, strides = _join_layout(d.dim, tensors)
        y, z, at = _join_run(d, tensors[0].shape, laid, strides, rng)
        ctx.d, ctx.strides, ctx.at = d, strides, at
        ctx.refs = [None if t is None else weakref.ref(t) for t in (rng, *laid)]
        ctx.shapes = [None if tensors[i] is None else tensors[i].shape for i in _ROWS]
        ctx.save_for_backward(rng, *laid)
        ctx.set_materialize_grads(False)
        return (y, z) if y is not None and z is not None else z if y is None else y

    @staticmethod
    @_once
    def backward(ctx, *douts):
        rng, *laid = ctx.saved_tensors
        d, some = ctx.d, douts[0] if douts[0] is not None else douts[-1]
        if some is None:
            return (None,) * (2 + len(laid))
        of = (some.dtype, some.get_device())
        with _device(some):
            strides, at = ctx.strides, [*map(_ptr, laid)]
            if at != ctx.at or not all(t is None or r() is t for r, t in zip(ctx.refs, (rng, *laid))):
                # not the tensors that were saved (checks and strides that cost a call 8 us)
                for i, shape in zip(_ROWS, ctx.shapes):
                    if laid[i] is not None:
                        _returned(laid[i], shape if laid[i].shape == shape else (shape.numel() // d.dim, d.dim), *of)
                for i in _VECTORS:
                    laid[i] = _returned_dense(laid[i], (d.dim,), *of)
                rng = _returned_dense(rng, (2,), torch.int64, of[1])
                laid, strides = _join_layout(d.dim, laid)
                at = [*map(_ptr, laid)]
            x = laid[0]
            dy = douts[0] if laid[1] is not None else None
            dz = douts[-1] if d.flags & _lib.JOIN_PRE else None
            if dy is not None:
                dy = _aligned(dy)
            if dz is not None:
                dz = _aligned(dz)
            need, grads = ctx.needs_input_grad[2:], [None] * len(laid)
            for i in _VECTORS:
                if need[i]:
                    grads[i] = torch.empty_like(laid[i])
            for i, shape in zip(_ROWS, ctx.shapes):
                if need[i]:
                    grads[i] = _new(shape, laid[i])
            ws, call = ctypes.c_size_t(), d.struct(strides)
            check(lib().slorr_join_workspace(call, ws), "slorr_join_workspace")
            work = _bytes(ws.value, x)
            check(lib().slorr_join_backward(call, _lib.JoinTensors(*at), _ptr(rng), _ptr(dy), _ptr(dz),
                                            _lib.JoinTensors(*map(_ptr, grads)), work.data_ptr(), ws.value,
                                            _stream(x)), "slorr_join_backward")
        return (None, None, *grads)


def _aligned(t: torch.Tensor) -> torch.Tensor:
    return t if t.is_contiguous() and t.data_ptr() % 16 == 0 else _at16(t.contiguous())


def _join_layout(dim, tensors):
    """The inputs as the library reads them, and the row strides of x, f and gate (0: absent)."""
    out, strides = list(tensors), [0, 0, 0]
    for k, i in enumerate(_ROWS):
        if out[i] is not None:
            out[i], strides[k] = _rows(out[i], dim)
    for i in _VECTORS:
        if out[i] is not None:
            out[i] = _at16(out[i])
    return out, strides


def _gate_rows(gate: torch.Tensor, x: torch.Tensor) -> int:
    """Rows of a gate over x: (dim,), or x's shape with trailing dimensions
    before the last set to 1."""
    if gate.dim() == 1:
        return 1
    if gate.dim() == x.dim():
        lead, rows = True, 1
        for g, n in zip(gate.shape[:-1], x.shape[:-1]):
            if lead and g == n:
                rows *= g
            elif g == 1:
                lead = False
            else:
                rows = 0
                break
        else:
            return rows
    raise ValueError("gate must have shape (dim,), or x's shape with its trailing dimensions before the last set to 1")


def _check_rng(p: float, rng, x: torch.Tensor) -> None:
    if not 0.0 <= p <= _MOST_P:
        raise ValueError("p must be in [0, 1), at most 1 - 2^-16 once rounded")
    if rng is None:
        if p > 0.0:
            raise ValueError("dropout needs rng")
    elif not isinstance(rng, torch.Tensor) or rng.dtype != torch.int64 or rng.shape != (2,) or not rng.is_contiguous() or rng.device != x.device:
        raise ValueError(f"rng must be an int64 tensor of two values on {x.device}")


def _join_call(x, f, kind, eps, post, pre, tensors, alpha, p, rng, site):
    if kind not in _NORM:
        raise ValueError(f"kind must be one of {list(_NORM)}")
    dim, gate = x.shape[-1], tensors[4]
    if dim > _MAX_NORM:
        raise ValueError(f"the last dimension must be at most {_MAX_NORM}")
    if not (0.0 <= eps <= _MOST_F32 and abs(alpha) <= _MOST_F32):
        raise ValueError("eps must be >= 0, eps and alpha finite in float32")
    if f is not None:
        _check_like(f, x.shape, x, "f")
    for i in _VECTORS:
        if tensors[i] is not None:
            _check_dense(tensors[i], (dim,), x, _JOIN[i])
    gate_rows = 0
    if gate is not None:
        if not isinstance(gate, torch.Tensor) or gate.dim() < 1:
            raise ValueError("gate must be a tensor")
        _check_like(gate, (*gate.shape[:-1], dim), x, "gate")
        gate_rows = _gate_rows(gate, x)
    d = _Call(x.numel() // dim, dim, _DTYPE[x.dtype], _NORM[kind], (_lib.JOIN_POST if post else 0) | (_lib.JOIN_PRE if pre else 0),
              gate_rows, float(eps), float(alpha), float(p), ctypes.c_int64(int(site)).value)      # (site: modulo 2^64)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return _Join.apply(d, rng, *tensors)
    y, z, _ = _join_run(d, x.shape, *_join_layout(dim, tensors), rng)
    return (y, z) if y is not None and z is not None else z if y is None else y


def block_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               kind: str = "rms", eps: float = 1e-5) -> torch.Tensor:
    """The norm of a block's input over the last dimension (at most 8192):
    kind "rms" or "layer", times weight plus bias (each (dim,) or None)."""
    _check_transforms(x, weight, bias)
    _check_first(x, "x")
    return _join_call(x, None, kind, eps, False, True, (x, None, None, None, None, None, weight, bias), 1.0, 0.0, None, 0)


def block_join(x: torch.Tensor, f: torch.Tensor, *, post: Optional[bool] = None,
               post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
               gate: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, alpha: float = 1.0,
               pre: Optional[bool] = None, pre_weight: Optional[torch.Tensor] = None,
               pre_bias: Optional[torch.Tensor] = None, kind: str = "rms", eps: float = 1e-5, p: float = 0.0,
               rng: Optional[torch.Tensor] = None, site: int = 0) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """The join between two blocks: y = x + alpha * scale * gate * dropout(u),
    u = norm(f) * post_weight + post_bias (u = f with post=False), and
    z = norm(y) * pre_weight + pre_bias (None with pre=False). Returns (y, z).

    x, f: (..., dim), dim at most 8192. post, pre: whether the norm is there; by
    default where one of its vectors is given. Vectors and scale: (dim,). gate:
    (dim,), x's shape, or x's shape with trailing dimensions before the last set
    to 1 (one gate row per sequence). p, rng, site: residual dropout, as in
    dropout(), as a factor 0 or 1 / (1 - p): an infinite u stays a NaN where it is
    dropped."""
    _check_transforms(x, f, post_weight, post_bias, gate, scale, pre_weight, pre_bias)
    _check_first(x, "x")
    if f is None:
        raise ValueError("f is required (block_norm is the norm alone)")
    post = (post_weight is not None or post_bias is not None) if post is None else bool(post)
    pre = (pre_weight is not None or pre_bias is not None) if pre is None else bool(pre)
    if not post and (post_weight is not None or post_bias is not None):
        raise ValueError("post_weight or post_bias with post=False")
    if not pre and (pre_weight is not None or pre_bias is not None):
        raise ValueError("pre_weight or pre_bias with pre=False")
    _check_rng(p, rng, x)
    out = _join_call(x, f, kind, eps, post, pre, (x, f, post_weight, post_bias, gate, scale, pre_weight, pre_bias),
                     alpha, p, rng, site)
    return out if pre else (out, None)


# ------------------------------------------------------------------ dropout

def _dropout_run(x: torch.Tensor, p: float, rng, site: int) -> torch.Tensor:
    with _device(x):
        x = _aligned(x)
        y = torch.empty_like(x)
        check(lib().slorr_dropout(x.numel(), _DTYPE[x.dtype], p, _ptr(rng), site, x.data_ptr(), y.data_ptr(), _stream(x)),
              "slorr_dropout")
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, rng, site):
        ctx.p, ctx.site = p, site
        ctx.save_for_backward(rng)
        return _dropout_run(x, p, rng, site)

    @staticmethod
    @_once
    def backward(ctx, dy):
        rng = _returned_dense(ctx.saved_tensors[0], (2,), torch.int64, dy.get_device())
        return _dropout_run(dy, ctx.p, rng, ctx.site), None, None, None


def dropout(x: torch.Tensor, p: float, rng: Optional[torch.Tensor], site: int = 0) -> torch.Tensor:
    """x / (1 - p) where an element is kept, else 0. Element e of x (in row-major
    order) is kept by its 16-bit number of the Philox4x32-10 sequence with key
    rng[0] and offset rng[1] + site, so p counts in steps of 2^-16 (rounded to
    the nearest; the factor is that of the rounded p)."""
    _check_transforms(x)
    _check_first(x, "x")
    _check_rng(p, rng, x)
    if torch.is_grad_enabled() and x.requires_grad:
        return _Dropout.apply(x, float(p), rng, int(site))
    return _dropout_run(x, float(p), rng, int(site))


# ------------------------------------------------------------------- module

class FeedForwardBlock(torch.nn.Module):
    """A pre-norm gated feed-forward block with its residual path:
    forward(x) = x + scale * dropout(norm(ffn(norm(x)))).

    matrices() are the projections, the weights to regularise. post: a norm
    after the feed-forward; scale: a residual scale per channel, starting at
    that value (None: none); p: residual dropout in training, from rng and site
    (see dropout)."""

    def __init__(self, dim: int, inner: int, act: str = "silu", kind: str = "rms", eps: float = 1e-5,
                 post: bool = False, scale: Optional[float] = None, p: float = 0.0, device=None,
                 dtype: torch.dtype = torch.bfloat16):
        super().__init__()
        if act not in _ACT or kind not in _NORM:
            raise ValueError(f"act must be one of {list(_ACT)}, kind one of {list(_NORM)}")
        if not (1 <= dim <= _MAX_NORM and inner >= 1 and 0.0 <= p <= _MOST_P and dtype in _DTYPE):
            raise ValueError(f"dim must be in [1, {_MAX_NORM}], inner at least 1, p in [0, 1), dtype float32 or bfloat16")
        kw = dict(device=device, dtype=dtype)
        self.act, self.kind, self.eps, self.p = act, kind, eps, p

        def matrix(r, c):
            return torch.nn.Parameter(torch.randn(r, c, **kw) * c ** -0.5)

        def vector(value):
            return torch.nn.Parameter(torch.full((dim,), float(value), **kw))

        self.w_gate, self.w_up, self.w_down = matrix(inner, dim), matrix(inner, dim), matrix(dim, inner)
        self.pre_weight = vector(1)
        self.pre_bias = vector(0) if kind == "layer" else None
        self.post_weight = vector(1) if post else None
        self.post_bias = vector(0) if post and kind == "layer" else None
        self.scale = None if scale is None else vector(scale)

    def matrices(self) -> List[torch.nn.Parameter]:
        return [self.w_gate, self.w_up, self.w_down]

    def forward(self, x: torch.Tensor, rng: Optional[torch.Tensor] = None, site: int = 0) -> torch.Tensor:
        z = block_norm(x, self.pre_weight, self.pre_bias, kind=self.kind, eps=self.eps)
        f = gated_ffn(z, self.w_gate, self.w_up, self.w_down, act=self.act)
        p = self.p if self.training else 0.0
        return block_join(x, f, post_weight=self.post_weight, post_bias=self.post_bias, scale=self.scale, kind=self.kind,
                          eps=self.eps, p=p, rng=rng if p > 0.0 else None, site=site)[0]
