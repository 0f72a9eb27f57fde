"""Torch binding of the dense operators of the C ABI: layer norm, affine map with an epilogue,
packed attention (argument marshalling only; bsa_layernorm_*, bsa_linear_* and bsa_attention_* of
include/bsa.h hold the contracts).

Tensors are bfloat16 or float32 on one GPU. A call runs on ``stream`` (a torch stream of the
tensors' device), or else on that device's current stream; outputs and workspaces are allocated
on the stream that the call runs on, so they are reused in its order. Operators are plain
functions: a forward returns what its backward takes.
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from . import _lib
from ._lib import BSA_BF16, BSA_F32, check

__all__ = ["ACTIVATIONS", "layernorm_forward", "layernorm_backward", "linear_forward", "linear_backward",
           "attention_forward", "attention_backward"]

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

_CODES = {torch.bfloat16: BSA_BF16, torch.float32: BSA_F32}
_HERE = contextlib.nullcontext()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _tensor(t, name, dtype=None, dev=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is None:
        if t.dtype not in _CODES:
            raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    elif t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")


def _shaped(t, name, shape, dtype, dev):
    _tensor(t, name, dtype, dev)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _rows(t, name, cols=None, dtype=None, dev=None, rows=None):
    """(rows, columns, elements between rows) of a [..., columns] tensor: contiguous, or 2-D with
    contiguous rows."""
    _tensor(t, name, dtype, dev)
    if t.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    n = t.shape[-1]
    if cols is not None and n != cols:
        raise ValueError(f"{name} must have {cols} columns, got {n}")
    if n == 0:
        raise ValueError(f"{name} must have at least one column")
    m = t.numel() // n
    if rows is not None and m != rows:
        raise ValueError(f"{name} must have {rows} rows, got {m}")
    if t.is_contiguous() or m <= 1:
        if t.stride(-1) == 1 or n == 1:
            return m, n, n
    elif t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= n:
        return m, n, t.stride(0)
    raise ValueError(f"{name} must be contiguous, or 2-D with contiguous rows that do not overlap")


def _on(dev, stream):
    """Context in which allocations and the call go to `stream` (default: dev's current stream)."""
    if stream is not None:
        if stream.device != dev:
            raise ValueError(f"stream must be on {dev}, got {stream.device}")
        return torch.cuda.stream(stream)
    if dev.index != torch._C._cuda_getDevice():
        return torch.cuda.device(dev)
    return _HERE


def _queue(dev):
    """The device's current stream as the C ABI takes it (torch.cuda.current_stream builds a Stream
    object: 1.8 us of a call's 10)."""
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _workspace(nbytes, dev):
    return torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None


# ---- layer norm ----

def layernorm_forward(x, gain, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x [..., C]; gain, bias [C] float32. Returns (y, mean, rstd),
    mean and rstd float32 of shape [...]."""
    lib = _lib.load()
    rows, cols, ld = _rows(x, "x")
    dev = x.device
    _shaped(gain, "gain", (cols,), torch.float32, dev)
    if bias is not None:
        _shaped(bias, "bias", (cols,), torch.float32, dev)
    p = _lib.bsa_layernorm_t(rows, cols, _CODES[x.dtype], eps, ld, cols, 0, 0)
    with _on(dev, stream):
        y = torch.empty(x.shape, dtype=x.dtype, device=dev)
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=dev)
        rstd = torch.empty_like(mean)
        check(lib.bsa_layernorm_forward(C.byref(p), x.data_ptr(), gain.data_ptr(), _ptr(bias), y.data_ptr(),
                                        mean.data_ptr(), rstd.data_ptr(), _queue(dev)), "bsa_layernorm_forward")
    return y, mean, rstd


def layernorm_backward(x, gain, mean, rstd, dy, bias: bool = True, stream=None):
    """Returns dict(dx, dgain, dbias): dx in x's type and shape, dgain and dbias [C] float32 (dbias None
    with bias = False)."""
    lib = _lib.load()
    rows, cols, ld = _rows(x, "x")
    dev = x.device
    _, _, lddy = _rows(dy, "dy", cols, x.dtype, dev, rows)
    _shaped(gain, "gain", (cols,), torch.float32, dev)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _shaped(t, name, x.shape[:-1], torch.float32, dev)
    p = _lib.bsa_layernorm_t(rows, cols, _CODES[x.dtype], 1.0, ld, 0, lddy, cols)   # eps: not read
    need = C.c_size_t()
    check(lib.bsa_layernorm_sizes(C.byref(p), C.byref(need)), "bsa_layernorm_sizes")
    with _on(dev, stream):
        ws = _workspace(need.value, dev)
        dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dgain = torch.empty(cols, dtype=torch.float32, device=dev)
        dbias = torch.empty_like(dgain) if bias else None
        check(lib.bsa_layernorm_backward(C.byref(p), x.data_ptr(), gain.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                         dy.data_ptr(), dx.data_ptr(), dgain.data_ptr(), _ptr(dbias), _ptr(ws),
                                         need.value, _queue(dev)), "bsa_layernorm_backward")
    return dict(dx=dx, dgain=dgain, dbias=dbias)


# ---- affine map ----

def _linear_params(x, w, act):
    m, k, ldx = _rows(x, "x")
    _tensor(w, "w", x.dtype, x.device)
    if w.dim() != 2:
        raise ValueError("w must be [n, k]")
    n, _, ldw = _rows(w, "w", k)
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return _lib.bsa_linear_t(m, k, n, _CODES[x.dtype], ACTIVATIONS[act], ldx, ldw, 0, 0, 0)


def _linear_sizes(lib, p):
    a, b = C.c_size_t(), C.c_size_t()
    check(lib.bsa_linear_sizes(C.byref(p), C.byref(a), C.byref(b)), "bsa_linear_sizes")
    return a.value, b.value


def linear_forward(x, w, bias=None, residual=None, act: str = "none", save_pre: bool = False, stream=None):
    """y = act(x w^T + bias) + residual for x [..., k], w [n, k], bias [n], residual [..., n]. Returns (y, pre);
    pre [..., n] is what linear_backward needs of a map with an activation (save_pre; else None)."""
    lib = _lib.load()
    p = _linear_params(x, w, act)
    dev, dt = x.device, x.dtype
    if bias is not None:
        _shaped(bias, "bias", (p.n,), dt, dev)
    if residual is not None:
        _, _, p.ld_res = _rows(residual, "residual", p.n, dt, dev, p.m)
    need, _ = _linear_sizes(lib, p)
    with _on(dev, stream):
        ws = _workspace(need, dev)
        y = torch.empty((*x.shape[:-1], p.n), dtype=dt, device=dev)
        pre = torch.empty_like(y) if save_pre and p.act else None
        check(lib.bsa_linear_forward(C.byref(p), x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(residual), y.data_ptr(),
                                     _ptr(pre), _ptr(ws), need, _queue(dev)), "bsa_linear_forward")
    return y, pre


def linear_backward(x, w, dy, pre=None, act: str = "none", bias: bool = False, need_dx: bool = True,
                    need_dw: bool = True, stream=None):
    """Gradients of linear_forward given dy [..., n]: dict(dx, dw, db), each in x's type (None where not
    asked for; bias: form db). The residual's gradient is dy itself."""
    lib = _lib.load()
    p = _linear_params(x, w, act)
    dev, dt = x.device, x.dtype
    _, _, p.ld_dy = _rows(dy, "dy", p.n, dt, dev, p.m)
    if p.act:
        if pre is None:
            raise ValueError("pre is needed: run linear_forward with save_pre=True")
        _rows(pre, "pre", p.n, dt, dev, p.m)
        if not pre.is_contiguous():
            raise ValueError("pre must be contiguous")
    _, need = _linear_sizes(lib, p)
    with _on(dev, stream):
        ws = _workspace(need, dev)
        dx = torch.empty(x.shape, dtype=dt, device=dev) if need_dx else None
        dw = torch.empty(w.shape, dtype=dt, device=dev) if need_dw else None
        db = torch.empty(p.n, dtype=dt, device=dev) if bias else None
        check(lib.bsa_linear_backward(C.byref(p), x.data_ptr(), w.data_ptr(), _ptr(pre) if p.act else None,
                                      dy.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db), _ptr(ws), need, _queue(dev)),
              "bsa_linear_backward")
    return dict(dx=dx, dw=dw, db=db)


# ---- packed attention ----

def _heads(t, name, dtype=None, dev=None, shape=None):
    """(elements between rows, between heads) of a [rows, heads, head_dim] tensor."""
    _tensor(t, name, dtype, dev)
    if t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, head_dim]")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    packed = t.shape[1] * t.shape[2], t.shape[2]
    if t.is_contiguous():
        return packed
    if t.stride(2) != 1:
        raise ValueError(f"{name} must be contiguous along head_dim")
    # the stride of a dimension of one entry says nothing
    row, head = (t.stride(i) if t.shape[i] != 1 else packed[i] for i in (0, 1))
    if row == 0 and head == 0:    # the C ABI's packed tensor
        raise ValueError(f"{name} may be broadcast over its rows or its heads, not over both: pass {name}.contiguous()")
    if row % (16 // t.element_size()) or head % (16 // t.element_size()):
        raise ValueError(f"{name}'s rows and heads must lie multiples of 16 bytes apart")
    return row, head


def _attention_params(q, k, v, cu_q, cu_k, used_k, causal, softmax_scale, zero_rest):
    q_row, q_head = _heads(q, "q")
    dev, dt = q.device, q.dtype
    tq, h, d = q.shape
    k_row, k_head = _heads(k, "k", dt, dev)
    if k.shape[2] != d or k.shape[1] == 0:
        raise ValueError(f"k must have head_dim {d} and at least one head, got {tuple(k.shape)}")
    v_row, v_head = _heads(v, "v", dt, dev, k.shape)
    if cu_k is None:
        if tq != k.shape[0]:
            raise ValueError("cu_k is needed where k has other rows than q")
        cu_k = cu_q
    _tensor(cu_q, "cu_q", torch.int32, dev)
    if cu_q.dim() != 1 or cu_q.numel() < 2 or not cu_q.is_contiguous():
        raise ValueError("cu_q must be a contiguous [sequences + 1] tensor")
    seqs = cu_q.numel() - 1
    _shaped(cu_k, "cu_k", (seqs + 1,), torch.int32, dev)
    if used_k is not None:
        _shaped(used_k, "used_k", (seqs,), torch.int32, dev)
    return _lib.bsa_attention_t(seqs, h, k.shape[1], d, tq, k.shape[0], int(bool(causal)), _CODES[dt], softmax_scale,
                                int(zero_rest), q_row, q_head, k_row, k_head, v_row, v_head, 0, 0, 0, 0)


def _attention_sizes(lib, p):
    a, b = C.c_size_t(), C.c_size_t()
    check(lib.bsa_attention_sizes(C.byref(p), C.byref(a), C.byref(b)), "bsa_attention_sizes")
    return a.value, b.value


def attention_forward(q, k, v, cu_q, cu_k=None, used_k=None, causal: bool = False, softmax_scale: float = 0.0,
                      o=None, lse=None, stream=None):
    """Attention over packed sequences: q [rows, heads, d], k and v [key rows, kv_heads, d] (kv_heads divides
    heads; strided views of a fused projection are fine, tensors broadcast over rows and heads are refused), cu_q
    and cu_k [sequences + 1] int32 first rows of the sequences and the end (cu_k None: the same rows as cu_q),
    used_k [sequences] int32 the key rows in use of each sequence's cache. causal: the last query of a sequence
    sees its last key. softmax_scale 0: 1 / sqrt(d). Returns (o, lse): o like q, lse [heads, rows] float32. Rows
    in no sequence are 0 (lse -inf); in an o and lse that the caller passes they keep what they held."""
    lib = _lib.load()
    if (o is None) != (lse is None):
        raise ValueError("pass both o and lse, or neither")
    p = _attention_params(q, k, v, cu_q, cu_k, used_k, causal, softmax_scale, o is None)
    cu_k = cu_q if cu_k is None else cu_k
    dev = q.device
    if o is not None:
        p.o_row, p.o_head = _heads(o, "o", q.dtype, dev, q.shape)
        _shaped(lse, "lse", (p.heads, p.total_q), torch.float32, dev)
    need, _ = _attention_sizes(lib, p)
    with _on(dev, stream):
        ws = _workspace(need, dev)
        if o is None:
            o = torch.empty(q.shape, dtype=q.dtype, device=dev)
            lse = torch.empty((p.heads, p.total_q), dtype=torch.float32, device=dev)
        check(lib.bsa_attention_forward(C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_q.data_ptr(),
                                        cu_k.data_ptr(), _ptr(used_k), o.data_ptr(), lse.data_ptr(), _ptr(ws), need,
                                        _queue(dev)), "bsa_attention_forward")
    return o, lse


def attention_backward(q, k, v, o, lse, d_o, cu_q, cu_k=None, used_k=None, causal: bool = False,
                       softmax_scale: float = 0.0, stream=None):
    """Gradients of attention_forward given d_o (like o; one that is broadcast over rows and heads, as o.sum((0, 1))
    gives, is passed as d_o.contiguous()): dict(dq, dk, dv), contiguous, in q's type; dk and dv are summed over a
    key head's query heads. Rows in no sequence and unused cache rows are 0."""
    lib = _lib.load()
    p = _attention_params(q, k, v, cu_q, cu_k, used_k, causal, softmax_scale, True)
    cu_k = cu_q if cu_k is None else cu_k
    dev = q.device
    p.o_row, p.o_head = _heads(o, "o", q.dtype, dev, q.shape)
    p.do_row, p.do_head = _heads(d_o, "d_o", q.dtype, dev, q.shape)
    _shaped(lse, "lse", (p.heads, p.total_q), torch.float32, dev)
    _, need = _attention_sizes(lib, p)
    with _on(dev, stream):
        ws = _workspace(need, dev)
        dq = torch.empty(q.shape, dtype=q.dtype, device=dev)
        dk = torch.empty(k.shape, dtype=k.dtype, device=dev)
        dv = torch.empty(v.shape, dtype=v.dtype, device=dev)
        check(lib.bsa_attention_backward(C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                         lse.data_ptr(), d_o.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(),
                                         _ptr(used_k), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), need,
                                         _queue(dev)), "bsa_attention_backward")
    return dict(dq=dq, dk=dk, dv=dv)
