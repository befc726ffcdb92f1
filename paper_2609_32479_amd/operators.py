"""Binding of the sequence-layer operators: linear attention with decay, normed and
rotated queries and keys, the gated feed-forward block (include/trackfit.h).

Argument marshalling only, as in the package itself: every function checks its
tensors, allocates the outputs and the workspace that the caller did not pass, and
enqueues the HIP kernels on ``stream`` (default: the tensors' device's current
stream).  What it allocates belongs to that stream, so that a workspace that is
freed when the function returns is not used by other streams' work too early.

The functions record nothing for autograd.  With gradients enabled the forward calls
refuse tensors that require one, whose gradients would silently be lost: call them under
``torch.no_grad()`` and take the gradients from the ``_backward`` functions, whose own
results have no graph either.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math

import torch

__all__ = ["decay_attention", "decay_attention_backward", "decay_attention_step", "qk_norm_rotate",
           "qk_norm_rotate_backward", "gated_ffn", "gated_ffn_backward", "SEQ_BAD_OFFSETS", "DecayConfig", "QKNormConfig",
           "GatedConfig"]

SEQ_BAD_OFFSETS = 1
_ELEMS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_vp, _i64, _i32, _sz, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float


class DecayConfig(ctypes.Structure):
    _fields_ = [("elem", _i32), ("n_heads", _i32), ("n_qk_heads", _i32), ("d_k", _i32), ("d_v", _i32),
                ("reverse", _i32), ("scale", _f32), ("clear", _i32)]


class QKNormConfig(ctypes.Structure):
    _fields_ = [("elem", _i32), ("n_q_heads", _i32), ("n_k_heads", _i32), ("head_dim", _i32), ("rotary_dim", _i32),
                ("interleaved", _i32), ("eps", _f32), ("base", ctypes.c_double), ("clear", _i32)]


class GatedConfig(ctypes.Structure):
    _fields_ = [("elem", _i32), ("width", _i32), ("inner", _i32), ("activation", _i32)]


EXPORTED = ("tf_decay_workspace_size", "tf_decay_backward_workspace_size", "tf_decay_attention",
            "tf_decay_attention_backward", "tf_decay_attention_step", "tf_qk_norm_rotate", "tf_qk_norm_workspace_size",
            "tf_qk_norm_rotate_backward", "tf_gated_ffn", "tf_gated_ffn_workspace_size", "tf_gated_ffn_backward")
_ACTIVATIONS = {"silu": 0, "gelu": 1}


def declare(L) -> None:
    """Set the C prototypes on the loaded library."""
    dc, nc, gc = ctypes.POINTER(DecayConfig), ctypes.POINTER(QKNormConfig), ctypes.POINTER(GatedConfig)
    t = [_vp, _i64]  # a tensor and its row stride
    protos = {
        "tf_decay_workspace_size": (_sz, [dc, _i64]),
        "tf_decay_backward_workspace_size": (_sz, [dc, _i64, _i32, _i32]),
        "tf_decay_attention": (ctypes.c_int, [dc, *t, *t, *t, *t, _i64, _vp, _i32, _vp, _vp, _sz, *t, _vp, _vp, _vp]),
        "tf_decay_attention_backward": (ctypes.c_int, [dc, *t, *t, *t, *t, *t, _i64, _vp, _i32, _vp, _vp, _vp, _sz, *t, *t,
                                                       *t, _vp, _vp, _vp, _vp]),
        "tf_decay_attention_step": (ctypes.c_int, [dc, *t, *t, *t, *t, _i32, _vp, _vp, *t, _vp]),
        "tf_qk_norm_workspace_size": (_sz, [nc, _i64]),
        "tf_qk_norm_rotate": (ctypes.c_int, [nc, *t, *t, _i64, _vp, _vp, _vp, _vp, _i32, *t, *t, _vp]),
        "tf_qk_norm_rotate_backward": (ctypes.c_int, [nc, *t, *t, *t, *t, _i64, _vp, _vp, _vp, _vp, _i32, _vp, _sz, *t, *t,
                                                      _vp, _vp, _vp]),
        "tf_gated_ffn": (ctypes.c_int, [gc, *t, _i64, _vp, _vp, _i64, *t, _vp]),
        "tf_gated_ffn_workspace_size": (_sz, [gc, _i64]),
        "tf_gated_ffn_backward": (ctypes.c_int, [gc, *t, *t, _i64, _vp, _vp, _i64, _vp, _sz, *t, _vp, _vp, _i64, _vp]),
    }
    for name, (res, args) in protos.items():
        f = getattr(L, name)
        f.restype, f.argtypes = res, args


_loaded = None


def _lib():
    global _loaded
    if _loaded is None:
        from . import lib
        _loaded = lib()
    return _loaded


def _check(status: int, what: str):
    if status:
        from . import TrackfitError
        raise TrackfitError(status, what)


@functools.lru_cache(maxsize=256)
def _config(kind, *fields):
    """A configuration of these plain values and a pointer to it (the library only reads it)."""
    cfg = kind(*fields)
    for (name, of), x in zip(kind._fields_, fields):  # ctypes keeps an int's low bits
        if of is _i32 and getattr(cfg, name) != x:
            raise ValueError(f"{name} {x} is not a 32-bit number")
    return cfg, ctypes.byref(cfg)


class _On:
    """The tensor's device, with ``stream`` as its current stream; entering gives the stream's handle."""
    __slots__ = ("tensor", "stream", "stack")

    def __init__(self, tensor: torch.Tensor, stream):
        self.tensor, self.stream, self.stack = tensor, stream, None

    def __enter__(self) -> int:
        index, stream = self.tensor.get_device(), self.stream
        if stream is None and index == torch._C._cuda_getDevice():  # nothing to switch
            return torch._C._cuda_getCurrentRawStream(index)
        with contextlib.ExitStack() as stack:  # (left again if something below fails)
            stack.enter_context(torch.cuda.device(index))
            if stream is None:
                handle = torch.cuda.current_stream().cuda_stream
            else:
                if not hasattr(stream, "cuda_stream"):
                    stream = torch.cuda.ExternalStream(int(stream))
                if stream.device.index != index:  # (its memory and its kernels would be another device's)
                    raise ValueError(f"the stream is on {stream.device}, the tensors on {self.tensor.device}")
                stack.enter_context(torch.cuda.stream(stream))
                handle = stream.cuda_stream
            self.stack = stack.pop_all()
        return int(handle)

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()


_on = _On


def _same(name: str, x, like: torch.Tensor, dtype=None):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if x.get_device() != like.get_device():
        raise ValueError(f"{name} is on {x.device}, the others on {like.device}")
    if dtype is not None and x.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {x.dtype}")


def _elem(x) -> int:
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("the operators take GPU tensors")
    if x.dtype not in _ELEMS:
        raise TypeError(f"unsupported element type {x.dtype}: float32, bfloat16 or float16")
    return _ELEMS[x.dtype]


_grad_enabled = torch.is_grad_enabled


def _no_graph(what: str, **tensors):
    for name, x in tensors.items():
        if x is not None and x.requires_grad:
            raise RuntimeError(f"{what} records no gradient, and {name} requires one: call it under torch.no_grad() and take "
                               f"gradients from the _backward function")


def _rows3(name: str, x: torch.Tensor, like: torch.Tensor, rows=None, heads=None, width=None) -> int:
    """Check a [rows, heads, width] tensor whose rows are contiguous; returns its row stride."""
    _same(name, x, like, like.dtype)
    shape = x.shape
    if len(shape) != 3 or (rows is not None and shape[0] != rows) or (heads is not None and shape[1] != heads) or \
            (width is not None and shape[2] != width):
        want = ", ".join("?" if v is None else str(v) for v in (rows, heads, width))
        raise ValueError(f"{name} must have shape [{want}], not {list(shape)}")
    _, h, w = shape
    n = h * w
    if x.is_contiguous():
        return n
    sr, sh, sw = x.stride()
    if (w > 1 and sw != 1) or (h > 1 and sh != w):
        raise ValueError(f"{name}'s rows [heads, width] must be contiguous")
    if shape[0] <= 1:
        return n  # (one row: any stride)
    if sr < n:
        raise ValueError(f"{name}'s rows overlap")
    return sr


def _new(name: str, x, like: torch.Tensor, shape, dtype) -> torch.Tensor:
    """The output tensor: a new one, or the caller's, checked to be contiguous."""
    if x is None:
        return like.new_empty(shape, dtype=dtype)
    _same(name, x, like, dtype)
    if tuple(x.shape) != tuple(shape) or not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape {list(shape)}")
    return x


def _rows_out(name: str, x, like: torch.Tensor, shape):
    """The output rows (new, or the caller's, which may be strided) and their stride."""
    if x is None:
        return like.new_empty(shape), shape[1] * shape[2]
    return x, _rows3(name, x, like, *shape)


def _offsets(offsets, like: torch.Tensor) -> int:
    _same("offsets", offsets, like, torch.int32)
    if offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 vector of at least one element")
    if offsets.numel() > 2 ** 31:
        raise ValueError("offsets must be those of fewer than 2^31 sequences")
    return offsets.numel() - 1


def _workspace(ws, need: int, like: torch.Tensor) -> torch.Tensor:
    if ws is None:
        return like.new_empty((max(need, 256),), dtype=torch.uint8)
    _same("workspace", ws, like)
    if not ws.is_contiguous() or ws.numel() * ws.element_size() < need:
        raise ValueError(f"workspace must be contiguous and hold {need} bytes")
    return ws


def _bytes(ws: torch.Tensor) -> int:
    return ws.numel() * ws.element_size()


def _ptr(x):
    return None if x is None else x.data_ptr()


def _decays(g: torch.Tensor, like: torch.Tensor, rows: int, heads: int) -> int:
    _same("log_decay", g, like, torch.float32)
    if g.dim() == 1 and g.shape[0] == heads and (heads == 1 or g.stride(0) == 1):
        return 0
    if g.dim() != 2 or tuple(g.shape) != (rows, heads) or (heads > 1 and g.stride(1) != 1):
        raise ValueError(f"log_decay must have shape [{heads}] or [{rows}, {heads}] with contiguous rows")
    if rows <= 1:
        return heads
    if g.stride(0) < heads:
        raise ValueError("log_decay's rows overlap (one decay a head is a vector)")
    return g.stride(0)


def _flags(flags, like):
    if flags is not None:
        _same("flags", flags, like, torch.int32)
        if flags.numel() < 1:
            raise ValueError("flags must hold one element")


def _state(name: str, s, like: torch.Tensor, n: int, heads: int, dk: int, dv: int):
    if s is None:
        return
    _same(name, s, like, torch.float32)
    if tuple(s.shape) != (n, heads, dk, dv) or not s.is_contiguous():
        raise ValueError(f"{name} must be contiguous float32 of shape [{n}, {heads}, {dk}, {dv}]")


def _decay_inputs(q, k, v, scale, reverse, clear=0):
    """Check q, k, v; returns the configuration and their row strides.  clear: the outputs, a bit each, that get zeros in
    the rows outside of all sequences (those that the call allocates)."""
    elem = _elem(q)
    if q.dim() != 3 or not isinstance(v, torch.Tensor) or v.dim() != 3:
        raise ValueError("q, k and v must have shape [rows, heads, width]")
    rows, qk_heads, dk = q.shape
    heads, dv = v.shape[1], v.shape[2]
    strides = (_rows3("q", q, q), _rows3("k", k, q, rows, qk_heads, dk), _rows3("v", v, q, rows))
    scale = float(scale) if scale is not None else dk ** -0.5 if dk else 1.0  # (heads without a width: refused by the library)
    return _config(DecayConfig, elem, heads, qk_heads, dk, dv, int(bool(reverse)), scale, clear), strides


def decay_attention(q, k, v, log_decay, offsets, scale=None, reverse=False, initial_state=None, return_state=False,
                    out=None, final_state=None, workspace=None, flags=None, stream=None):
    """Linear attention with a decay for each head over packed sequences: per
    sequence and head, S_t = exp(g_t) S_{t-1} + k_t v_t^T and o_t = scale S_t^T q_t.

    q, k [rows, qk_heads, d_k], v [rows, heads, d_v] (fp32, bf16 or fp16; rows may be
    strided, as slices of one projection are), log_decay float32 [rows, heads] or
    [heads], offsets int32 [n + 1].  scale: d_k ** -0.5 by default.  reverse: from
    each sequence's last row to its first.  initial_state float32 [n, heads, d_k, d_v]
    or None.  Returns (out [rows, heads, d_v], the last states or None); rows outside
    of all sequences are left as they are in a given ``out``, and zeros in a new one.
    The last states are returned if ``return_state`` is set or ``final_state`` is given.
    ``flags`` (int32 GPU tensor) is OR-ed with SEQ_BAD_OFFSETS when the offsets make no
    sequences (the outputs are NaN then).
    """
    (cfg, at), (qs, ks, vs) = _decay_inputs(q, k, v, scale, reverse, int(out is None))
    rows, n = q.shape[0], _offsets(offsets, q)
    gs = _decays(log_decay, q, rows, cfg.n_heads)
    _state("initial_state", initial_state, q, n, cfg.n_heads, cfg.d_k, cfg.d_v)
    _flags(flags, q)
    if _grad_enabled():
        _no_graph("decay_attention", q=q, k=k, v=v, log_decay=log_decay, initial_state=initial_state, out=out,
                  final_state=final_state)
    with _on(q, stream) as s:
        out, os = _rows_out("out", out, q, (rows, cfg.n_heads, cfg.d_v))
        if return_state or final_state is not None:
            final_state = _new("final_state", final_state, q, (n, cfg.n_heads, cfg.d_k, cfg.d_v), torch.float32)
        ws = _workspace(workspace, int(_lib().tf_decay_workspace_size(at, rows)), q)
        _check(_lib().tf_decay_attention(
            at, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, log_decay.data_ptr(), gs, rows,
            offsets.data_ptr(), n, _ptr(initial_state), ws.data_ptr(), _bytes(ws), out.data_ptr(), os, _ptr(final_state),
            _ptr(flags), s), "tf_decay_attention")
    return out, final_state


def decay_attention_backward(d_out, q, k, v, log_decay, offsets, scale=None, reverse=False, initial_state=None,
                             d_state=None, dq=None, dk=None, dv=None, d_log_decay=None, d_initial=None, workspace=None,
                             flags=None, stream=None):
    """Gradients of decay_attention's inputs: (dq, dk, dv, d_log_decay, d_initial).

    d_out as out, d_state as the last states (None: they are not used), the other
    arguments those of the forward call.  d_initial is None without an initial_state.
    Rows outside of all sequences are zeros in the gradients that the call allocates, and
    left as they are in given ones.
    """
    clear = (dq is None) | (dk is None) << 1 | (dv is None) << 2 | (d_log_decay is None) << 3
    (cfg, at), (qs, ks, vs) = _decay_inputs(q, k, v, scale, reverse, clear)
    rows, n, h = q.shape[0], _offsets(offsets, q), cfg.n_heads
    gs = _decays(log_decay, q, rows, h)
    _state("initial_state", initial_state, q, n, h, cfg.d_k, cfg.d_v)
    _state("d_state", d_state, q, n, h, cfg.d_k, cfg.d_v)
    ds = _rows3("d_out", d_out, q, rows, h, cfg.d_v)
    _flags(flags, q)
    with _on(q, stream) as s:
        dq, dqs = _rows_out("dq", dq, q, tuple(q.shape))
        dk, dks = _rows_out("dk", dk, q, tuple(q.shape))
        dv, dvs = _rows_out("dv", dv, q, (rows, h, cfg.d_v))
        d_log_decay = _new("d_log_decay", d_log_decay, q, tuple(log_decay.shape), torch.float32)
        if initial_state is not None or d_initial is not None:
            d_initial = _new("d_initial", d_initial, q, (n, h, cfg.d_k, cfg.d_v), torch.float32)
        need = int(_lib().tf_decay_backward_workspace_size(at, rows, n, int(d_state is not None)))
        ws = _workspace(workspace, need, q)
        _check(_lib().tf_decay_attention_backward(
            at, d_out.data_ptr(), ds, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
            log_decay.data_ptr(), gs, rows, offsets.data_ptr(), n, _ptr(initial_state), _ptr(d_state), ws.data_ptr(),
            _bytes(ws), dq.data_ptr(), dqs, dk.data_ptr(), dks, dv.data_ptr(), dvs, d_log_decay.data_ptr(),
            _ptr(d_initial), _ptr(flags), s), "tf_decay_attention_backward")
    return dq, dk, dv, d_log_decay, d_initial


def decay_attention_step(q, k, v, log_decay, state, scale=None, state_out=None, out=None, stream=None):
    """One row of every sequence, for serving: q, k [n, qk_heads, d_k], v [n, heads,
    d_v], log_decay [n, heads] or [heads], state float32 [n, heads, d_k, d_v].
    Returns (out [n, heads, d_v], the new states).  ``state_out`` may be ``state``,
    which is then updated in place; by default the new states are a new tensor."""
    (cfg, at), (qs, ks, vs) = _decay_inputs(q, k, v, scale, False)
    n = q.shape[0]
    gs = _decays(log_decay, q, n, cfg.n_heads)
    if state is None:
        raise ValueError("state must be a GPU tensor")
    _state("state", state, q, n, cfg.n_heads, cfg.d_k, cfg.d_v)
    if _grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or log_decay.requires_grad or
                            state.requires_grad or out is not None or state_out is not None):
        _no_graph("decay_attention_step", q=q, k=k, v=v, log_decay=log_decay, state=state, out=out, state_out=state_out)
    with _on(q, stream) as s:
        out, os = _rows_out("out", out, q, (n, cfg.n_heads, cfg.d_v))
        if state_out is not state:  # (in place: checked above)
            state_out = _new("state_out", state_out, state, state.shape, torch.float32)
        _check(_lib().tf_decay_attention_step(
            at, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, log_decay.data_ptr(), gs, n,
            state.data_ptr(), state_out.data_ptr(), out.data_ptr(), os, s), "tf_decay_attention_step")
    return out, state_out


def _norm_inputs(q, k, q_gain, k_gain, offsets, positions, rotary_dim, base, interleaved, eps, q_out, k_out):
    elem = _elem(q)
    if q.dim() != 3:
        raise ValueError("q and k must have shape [rows, heads, width]")
    rows, hq, d = q.shape
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q and k must have shape [rows, heads, width]")
    qs, ks = _rows3("q", q, q), _rows3("k", k, q, rows, None, d)
    for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
        _same(name, g, q, torch.float32)
        if tuple(g.shape) != (d,) or not g.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 vector of {d}")
    if positions is not None:
        _same("positions", positions, q, torch.int32)
        if tuple(positions.shape) != (rows,) or not positions.is_contiguous():
            raise ValueError(f"positions must be a contiguous int32 vector of {rows}")
    n = _offsets(offsets, q) if offsets is not None else 0
    rot = d if rotary_dim is None else int(rotary_dim)
    if not math.isfinite(float(base)):
        raise ValueError("base must be finite")
    clear = int(q_out is None) | int(k_out is None) << 1 if offsets is not None else 0
    return _config(QKNormConfig, elem, hq, k.shape[1], d, rot, int(bool(interleaved)), float(eps), float(base), clear), qs, ks, n


def qk_norm_rotate(q, k, q_gain, k_gain, offsets=None, positions=None, rotary_dim=None, base=10000.0, interleaved=False,
                   eps=1e-6, q_out=None, k_out=None, stream=None):
    """Queries and keys normalised per head (root mean square, float32 gains [d])
    and rotated by their positions, in one pass; returns (q, k) of the same shapes.

    q [rows, q_heads, d], k [rows, k_heads, d].  A row's position is its entry of
    ``positions`` (int32 [rows]), else it counts from its sequence's first row
    (``offsets``), else from row 0.  The first ``rotary_dim`` values (default: all) are
    rotated, in pairs (j, j + rotary_dim / 2), or of neighbours if ``interleaved``.
    With offsets only the sequences' rows are written; the others are zeros in tensors
    that the call allocates.  ``q_out`` and ``k_out`` may be q and k.
    """
    (cfg, at), qs, ks, n = _norm_inputs(q, k, q_gain, k_gain, offsets, positions, rotary_dim, base, interleaved, eps, q_out,
                                        k_out)
    if _grad_enabled() and (q.requires_grad or k.requires_grad or q_gain.requires_grad or k_gain.requires_grad or
                            q_out is not None or k_out is not None):
        _no_graph("qk_norm_rotate", q=q, k=k, q_gain=q_gain, k_gain=k_gain, q_out=q_out, k_out=k_out)
    with _on(q, stream) as s:
        q_out, qos = _rows_out("q_out", q_out, q, tuple(q.shape))
        k_out, kos = _rows_out("k_out", k_out, q, tuple(k.shape))
        _check(_lib().tf_qk_norm_rotate(
            at, q.data_ptr(), qs, k.data_ptr(), ks, q.shape[0], q_gain.data_ptr(), k_gain.data_ptr(),
            _ptr(positions), _ptr(offsets), n, q_out.data_ptr(), qos, k_out.data_ptr(), kos, s), "tf_qk_norm_rotate")
    return q_out, k_out


def qk_norm_rotate_backward(dq_out, dk_out, q, k, q_gain, k_gain, offsets=None, positions=None, rotary_dim=None,
                            base=10000.0, interleaved=False, eps=1e-6, dq=None, dk=None, dq_gain=None, dk_gain=None,
                            workspace=None, stream=None):
    """Gradients of qk_norm_rotate's inputs from those of its outputs: (dq, dk,
    dq_gain, dk_gain); q, k and the rest as in the forward call.  ``dq`` and ``dk``
    may be ``dq_out`` and ``dk_out``.  With offsets, rows outside of all sequences are
    zeros in gradients that the call allocates and left as they are in given ones."""
    (cfg, at), qs, ks, n = _norm_inputs(q, k, q_gain, k_gain, offsets, positions, rotary_dim, base, interleaved, eps, dq, dk)
    rows, d = q.shape[0], q.shape[2]
    dqos = _rows3("dq_out", dq_out, q, *q.shape)
    dkos = _rows3("dk_out", dk_out, q, *k.shape)
    with _on(q, stream) as s:
        dq, dqs = _rows_out("dq", dq, q, tuple(q.shape))
        dk, dks = _rows_out("dk", dk, q, tuple(k.shape))
        dq_gain = _new("dq_gain", dq_gain, q, (d,), torch.float32)
        dk_gain = _new("dk_gain", dk_gain, q, (d,), torch.float32)
        ws = _workspace(workspace, int(_lib().tf_qk_norm_workspace_size(at, rows)), q)
        _check(_lib().tf_qk_norm_rotate_backward(
            at, dq_out.data_ptr(), dqos, dk_out.data_ptr(), dkos, q.data_ptr(), qs, k.data_ptr(), ks, rows,
            q_gain.data_ptr(), k_gain.data_ptr(), _ptr(positions), _ptr(offsets), n, ws.data_ptr(), _bytes(ws),
            dq.data_ptr(), dqs, dk.data_ptr(), dks, dq_gain.data_ptr(), dk_gain.data_ptr(), s), "tf_qk_norm_rotate_backward")
    return dq, dk, dq_gain, dk_gain


def _matrix(name: str, x, like: torch.Tensor, rows=None, cols=None) -> int:
    """Check a [rows, cols] matrix with unit column stride; returns its row stride."""
    _same(name, x, like, like.dtype)
    if x.dim() != 2 or (rows is not None and x.shape[0] != rows) or (cols is not None and x.shape[1] != cols):
        want = ", ".join("?" if v is None else str(v) for v in (rows, cols))
        raise ValueError(f"{name} must have shape [{want}], not {list(x.shape)}")
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if x.shape[0] <= 1:
        return x.shape[1]
    if x.stride(0) < x.shape[1]:
        raise ValueError(f"{name}'s rows overlap")
    return x.stride(0)


def _gated_inputs(x, w_gate, w_up, activation):
    elem = _elem(x)
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(_ACTIVATIONS)}")
    xs = _matrix("x", x, x)
    ws = _matrix("w_gate", w_gate, x, None, x.shape[1])
    wu = _matrix("w_up", w_up, x, w_gate.shape[0], x.shape[1])
    if ws != wu:
        raise ValueError("w_gate and w_up must have the same row stride")
    return _config(GatedConfig, elem, x.shape[1], w_gate.shape[0], _ACTIVATIONS[activation]), xs, ws


def gated_ffn(x, w_gate, w_up, activation="silu", out=None, stream=None):
    """act(x w_gate^T) * (x w_up^T) in one kernel: x [rows, width], both weights
    [inner, width], of one type (fp32, bf16, fp16); activation "silu" or "gelu" (a
    Phi(a)).  Returns [rows, inner]."""
    (cfg, at), xs, ws = _gated_inputs(x, w_gate, w_up, activation)
    if _grad_enabled() and (x.requires_grad or w_gate.requires_grad or w_up.requires_grad or out is not None):
        _no_graph("gated_ffn", x=x, w_gate=w_gate, w_up=w_up, out=out)
    with _on(x, stream) as s:
        if out is None:
            out = x.new_empty((x.shape[0], cfg.inner))
        os = _matrix("out", out, x, x.shape[0], cfg.inner)
        _check(_lib().tf_gated_ffn(at, x.data_ptr(), xs, x.shape[0], w_gate.data_ptr(), w_up.data_ptr(), ws,
                                   out.data_ptr(), os, s), "tf_gated_ffn")
    return out


def gated_ffn_backward(d_out, x, w_gate, w_up, activation="silu", dx=None, dw_gate=None, dw_up=None, workspace=None,
                       stream=None):
    """Gradients of gated_ffn's inputs: (dx, dw_gate, dw_up).  The projections are
    computed again from x and the weights."""
    (cfg, at), xs, ws = _gated_inputs(x, w_gate, w_up, activation)
    rows = x.shape[0]
    ds = _matrix("d_out", d_out, x, rows, cfg.inner)
    with _on(x, stream) as s:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx
        dw_gate = torch.empty_like(w_gate, memory_format=torch.contiguous_format) if dw_gate is None else dw_gate
        dw_up = torch.empty_like(w_up, memory_format=torch.contiguous_format) if dw_up is None else dw_up
        dxs = _matrix("dx", dx, x, *x.shape)
        dws = _matrix("dw_gate", dw_gate, x, *w_gate.shape)
        if _matrix("dw_up", dw_up, x, *w_up.shape) != dws:
            raise ValueError("dw_gate and dw_up must have the same row stride")
        wk = _workspace(workspace, int(_lib().tf_gated_ffn_workspace_size(at, rows)), x)
        _check(_lib().tf_gated_ffn_backward(
            at, d_out.data_ptr(), ds, x.data_ptr(), xs, rows, w_gate.data_ptr(), w_up.data_ptr(), ws,
            wk.data_ptr(), _bytes(wk), dx.data_ptr(), dxs, dw_gate.data_ptr(), dw_up.data_ptr(), dws, s),
            "tf_gated_ffn_backward")
    return dx, dw_gate, dw_up
