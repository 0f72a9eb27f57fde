"""Torch binding of the dense operators of the C ABI: layer norm, affine map with an epilogue, gated
map, rotary positions with head norms, packed attention, and a cache of 8 bits for it (argument
marshalling only; bsa_layernorm_*, bsa_linear_*, bsa_gated_*, bsa_rotary_*, bsa_attention_* and
bsa_cache_* of include/bsa.h hold the contracts).

Tensors are bfloat16 or float32 on one GPU. A call runs on ``stream`` (a torch stream of the
tensors' device), or else on that device's current stream; outputs and workspaces are allocated
on the stream that the call runs on, so they are reused in its order. Operators are plain
functions: a forward returns what its backward takes.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import operator
from typing import NamedTuple

import torch

from . import _lib
from ._lib import BSA_BF16, BSA_F32, check

__all__ = ["ACTIVATIONS", "layernorm_forward", "layernorm_backward", "linear_forward", "linear_backward",
           "gated_forward", "gated_backward", "rotary_frequencies", "rotary_forward", "rotary_backward",
           "attention_forward", "attention_backward", "Cache", "cache_alloc", "cache_write", "cache_read",
           "cache_attention_forward"]

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

_CODES = {torch.bfloat16: BSA_BF16, torch.float32: BSA_F32}
_HERE = contextlib.nullcontext()


# Parameter records of calls whose arguments have passed the checks, by all that the checks read of them (shapes, strides,
# types, devices, plain numbers; never addresses or values of tensors). The calls of a serving step are as short on the GPU as their
# host path is long: with it a rotary_forward of 32 tokens takes 8 us of the host, without 14, a gated_forward 6.6, without 12.
_checked = {}


def _remember(key, record):
    if len(_checked) >= 4096:      # shapes that keep changing: start over
        _checked.clear()
    _checked[key] = record
    return record


def _signature(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.device)


def _fresh(t):
    """A contiguous tensor of t's shape, type and device."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


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


# ---- gated map ----

def _gated_params(x, w, act):
    m, k, ldx = _rows(x, "x")
    _tensor(w, "w", x.dtype, x.device)
    if w.dim() != 2 or w.shape[0] % 2:
        raise ValueError("w must be [2 n, k]")
    n2, _, ldw = _rows(w, "w", k)
    if not isinstance(act, str) or act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return _lib.bsa_gated_t(m, k, n2 // 2, _CODES[x.dtype], ACTIVATIONS[act], ldx, ldw, 0, 0)


def _gated_sizes(lib, p):
    a, b = C.c_size_t(), C.c_size_t()
    check(lib.bsa_gated_sizes(C.byref(p), C.byref(a), C.byref(b)), "bsa_gated_sizes")
    return a.value, b.value


def gated_forward(x, w, bias=None, act: str = "silu", save_pre: bool = False, stream=None):
    """y = act(g) u, [g | u] = x w^T + bias, for x [..., k], w [2 n, k] (the gate's n rows first), bias [2 n]. Returns
    (y [..., n], pre); pre [..., 2 n] is what gated_backward needs (save_pre; else None)."""
    lib = _lib.load()
    try:
        key = ("gated_forward", _signature(x), _signature(w), _signature(bias), act)
        record = _checked.get(key)
    except (AttributeError, TypeError):      # no tensors: the checks say so
        key = record = None
    if record is None:
        p = _gated_params(x, w, act)
        if bias is not None:
            _shaped(bias, "bias", (2 * p.n,), x.dtype, x.device)
        record = _remember(key, (p, _gated_sizes(lib, p)[0]))
    p, need = record
    dev, dt = x.device, x.dtype
    with _on(dev, stream):
        ws = _workspace(need, dev)
        y = torch.empty((*x.shape[:-1], p.n), dtype=dt, device=dev)
        pre = torch.empty((*x.shape[:-1], 2 * p.n), dtype=dt, device=dev) if save_pre else None
        check(lib.bsa_gated_forward(C.byref(p), x.data_ptr(), w.data_ptr(), _ptr(bias), y.data_ptr(), _ptr(pre), _ptr(ws),
                                    need, _queue(dev)), "bsa_gated_forward")
    return y, pre


def gated_backward(x, w, dy, pre, act: str = "silu", bias: bool = False, need_dx: bool = True, need_dw: bool = True,
                   stream=None):
    """Gradients of gated_forward given dy [..., n]: dict(dx, dw, db), each in x's type (None where not asked for;
    bias: form db)."""
    lib = _lib.load()
    try:
        key = ("gated_backward", _signature(x), _signature(w), _signature(dy), _signature(pre), act)
        record = _checked.get(key)
    except (AttributeError, TypeError):
        key = record = None
    if record is None:
        p = _gated_params(x, w, act)
        _, _, p.ld_dy = _rows(dy, "dy", p.n, x.dtype, x.device, p.m)
        if pre is None:
            raise ValueError("pre is needed: run gated_forward with save_pre=True")
        _rows(pre, "pre", 2 * p.n, x.dtype, x.device, p.m)
        if not pre.is_contiguous():
            raise ValueError("pre must be contiguous")
        record = _remember(key, (p, _gated_sizes(lib, p)[1]))
    p, need = record
    dev, dt = x.device, x.dtype
    with _on(dev, stream):
        ws = _workspace(need, dev)
        dx = torch.empty(x.shape, dtype=dt, device=dev) if need_dx else None
        dw = torch.empty(w.shape, dtype=dt, device=dev) if need_dw else None
        db = torch.empty(2 * p.n, dtype=dt, device=dev) if bias else None
        check(lib.bsa_gated_backward(C.byref(p), x.data_ptr(), w.data_ptr(), pre.data_ptr(), dy.data_ptr(), _ptr(dx),
                                     _ptr(dw), _ptr(db), _ptr(ws), need, _queue(dev)), "bsa_gated_backward")
    return dict(dx=dx, dw=dw, db=db)


# ---- rotary positions ----

def rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: float = 0.0,
                       low: float = 1.0, high: float = 32.0, axes: int = 1, device="cuda"):
    """(freq, magnitude) for rotary_forward: freq [rot / 2] float64, for each of `axes` axes the same
    base^(-i / n), i < n = rot / 2 / axes. For contexts `factor` times longer than the `trained` positions, scaling
    "linear" divides every frequency by factor (position interpolation), "base" raises the base so that the
    slowest pair's is divided by it and the fastest pair's kept, and "ramp" divides those of the pairs that turn
    less than `low` times in the trained positions, keeps those that turn more than `high` times, goes linearly
    between, and makes magnitude 0.1 ln(factor) + 1 (Peng et al. 2023)."""
    if rot < 2 or rot % 2 or axes < 1 or rot // 2 % axes:
        raise ValueError("rot must be even and axes divide rot / 2")
    if not base > 0 or not factor >= 1:
        raise ValueError("base must be > 0 and factor >= 1")
    n = rot // 2 // axes
    if scaling == "base" and n > 1:
        base = base * factor ** (n / (n - 1))
    f = torch.tensor([base ** (-i / n) for i in range(n)], dtype=torch.float64)
    magnitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        if not trained > 0 or not 0 <= low < high:
            raise ValueError("scaling by a ramp needs trained > 0 and 0 <= low < high")
        if factor > 1:
            keep = ((f * (trained / (2 * math.pi)) - low) / (high - low)).clamp_(0, 1)
            f = f * keep + f / factor * (1 - keep)
        magnitude = 0.1 * math.log(factor) + 1
    elif scaling not in ("none", "base"):
        raise ValueError(f"scaling must be none, linear, base or ramp, got {scaling!r}")
    return f.repeat(axes).to(device), magnitude


def _any_heads(t, name, dtype, dev, shape=None):
    """(elements between rows, between heads) of a [rows, heads, head_dim] tensor of any strides."""
    _tensor(t, name, dtype, dev)
    if t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, head_dim]")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    packed = t.shape[1] * t.shape[2], t.shape[2]
    if t.is_contiguous():
        return packed
    if t.stride(2) != 1 and t.shape[2] != 1:
        raise ValueError(f"{name} must be contiguous along head_dim")
    # the stride of a dimension of one entry says nothing
    row, head = (t.stride(i) if t.shape[i] != 1 else packed[i] for i in (0, 1))
    if row == 0 and head == 0:    # the C ABI's packed tensor
        raise ValueError(f"{name} may be broadcast over its rows or its heads, not over both: pass {name}.contiguous()")
    return row, head


def _rotary_params(q, k, positions, freq, gain_q, gain_k, eps, interleaved, magnitude):
    """For q and k, or gradients like them; their strides stay to be filled in."""
    _tensor(q, "q")
    dev = q.device
    if q.dim() != 3:
        raise ValueError("q must be [rows, heads, head_dim]")
    rows, heads, d = q.shape
    kv = 0
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 3 or k.shape[0] != rows or k.shape[2] != d or k.shape[1] == 0:
            raise ValueError(f"k must be [{rows}, kv_heads, {d}]")
        kv = k.shape[1]
    elif gain_k is not None:
        raise ValueError("gain_k needs k")
    _tensor(freq, "freq", torch.float64, dev)
    if freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous [rot / 2] tensor")
    if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.float32):
        raise ValueError("positions must be an int32 or float32 tensor")
    if positions.dim() not in (1, 2) or positions.shape[0] != rows or not positions.is_contiguous():
        raise ValueError(f"positions must be a contiguous [{rows}] or [{rows}, axes] tensor")
    _tensor(positions, "positions", positions.dtype, dev)
    axes = 1 if positions.dim() == 1 else positions.shape[1]
    for name, g in (("gain_q", gain_q), ("gain_k", gain_k)):
        if g is not None:
            _shaped(g, name, (d,), torch.float32, dev)
    return _lib.bsa_rotary_t(rows, heads, kv, d, 2 * freq.numel(), axes, int(positions.dtype == torch.float32),
                             int(bool(interleaved)), _CODES[q.dtype], eps, magnitude, *[0] * 12)


def rotary_forward(q, k, positions, freq, gain_q=None, gain_k=None, eps: float = 1e-6, interleaved: bool = False,
                   magnitude: float = 1.0, y_q=None, y_k=None, stream=None):
    """Queries q [rows, heads, d] and keys k [rows, kv_heads, d] (or None), each head's root mean square normed to its
    gain [d] (float32; None: not normed), their first rot = 2 len(freq) values rotated by position * freq: pairs
    (i, i + rot / 2), or with interleaved (2 i, 2 i + 1); magnitude scales the rotated values. positions [rows] int32
    or float32, or [rows, axes] with each axis turning its own run of the pairs. Strided views of a fused
    projection are fine. Returns (y_q, y_k), which may be given: q and k themselves too."""
    lib = _lib.load()
    sig = _signature
    eps, interleaved, magnitude = float(eps), bool(interleaved), float(magnitude)
    try:
        key = ("rotary_forward", sig(q), sig(k), sig(positions), sig(freq), sig(gain_q), sig(gain_k), eps, interleaved,
               magnitude, sig(y_q), sig(y_k))
        p = _checked.get(key)
    except (AttributeError, TypeError):      # no tensors: the checks say so
        key = p = None
    if p is None:
        p = _rotary_params(q, k, positions, freq, gain_q, gain_k, eps, interleaved, magnitude)
        dev, dt = q.device, q.dtype
        p.q_row, p.q_head = _any_heads(q, "q", dt, dev)
        if k is not None:
            p.k_row, p.k_head = _any_heads(k, "k", dt, dev)
        elif y_k is not None:
            raise ValueError("y_k needs k")
        if y_q is not None:
            p.oq_row, p.oq_head = _any_heads(y_q, "y_q", dt, dev, q.shape)
        if y_k is not None:
            p.ok_row, p.ok_head = _any_heads(y_k, "y_k", dt, dev, k.shape)
        _remember(key, p)
    dev = q.device
    with _on(dev, stream):
        y_q = _fresh(q) if y_q is None else y_q
        y_k = _fresh(k) if y_k is None and k is not None else y_k
        check(lib.bsa_rotary_forward(C.byref(p), q.data_ptr(), _ptr(k), positions.data_ptr(), freq.data_ptr(), _ptr(gain_q),
                                     _ptr(gain_k), y_q.data_ptr(), _ptr(y_k), _queue(dev)), "bsa_rotary_forward")
    return y_q, y_k


def rotary_backward(dy_q, dy_k, positions, freq, q=None, k=None, gain_q=None, gain_k=None, eps: float = 1e-6,
                    interleaved: bool = False, magnitude: float = 1.0, dq=None, dk=None, stream=None):
    """Gradients of rotary_forward given those of its outputs: dict(dq, dk, dgain_q, dgain_k). q (k) as it was before
    the forward is needed with gain_q (gain_k). dq and dk may be given: views of a fused gradient, or dy_q and
    dy_k themselves."""
    lib = _lib.load()
    sig = _signature
    eps, interleaved, magnitude = float(eps), bool(interleaved), float(magnitude)
    try:
        key = ("rotary_backward", sig(dy_q), sig(dy_k), sig(positions), sig(freq), sig(q), sig(k), sig(gain_q), sig(gain_k), eps,
               interleaved, magnitude, sig(dq), sig(dk))
        record = _checked.get(key)
    except (AttributeError, TypeError, ValueError):
        key = record = None
    if record is None:
        p = _rotary_params(dy_q, dy_k, positions, freq, gain_q, gain_k, eps, interleaved, magnitude)
        dev, dt = dy_q.device, dy_q.dtype
        p.dq_row, p.dq_head = _any_heads(dy_q, "dy_q", dt, dev)
        if dy_k is not None:
            p.dk_row, p.dk_head = _any_heads(dy_k, "dy_k", dt, dev)
        elif dk is not None:
            raise ValueError("dk needs dy_k")
        if gain_q is not None:
            if q is None:
                raise ValueError("q is needed with gain_q")
            p.q_row, p.q_head = _any_heads(q, "q", dt, dev, dy_q.shape)
        if gain_k is not None:
            if k is None:
                raise ValueError("k is needed with gain_k")
            p.k_row, p.k_head = _any_heads(k, "k", dt, dev, dy_k.shape)
        if dq is not None:
            p.oq_row, p.oq_head = _any_heads(dq, "dq", dt, dev, dy_q.shape)
        if dk is not None:
            p.ok_row, p.ok_head = _any_heads(dk, "dk", dt, dev, dy_k.shape)
        need = C.c_size_t()
        if gain_q is not None or gain_k is not None:
            check(lib.bsa_rotary_sizes(C.byref(p), C.byref(need)), "bsa_rotary_sizes")
        record = _remember(key, (p, need.value))
    p, need = record
    dev = dy_q.device
    with _on(dev, stream):
        ws = _workspace(need, dev)
        dq = _fresh(dy_q) if dq is None else dq
        dk = _fresh(dy_k) if dk is None and dy_k is not None else dk
        dgain_q = None if gain_q is None else torch.empty_like(gain_q)
        dgain_k = None if gain_k is None else torch.empty_like(gain_k)
        check(lib.bsa_rotary_backward(C.byref(p), None if gain_q is None else q.data_ptr(),
                                      None if gain_k is None else k.data_ptr(), positions.data_ptr(), freq.data_ptr(),
                                      _ptr(gain_q), _ptr(gain_k), dy_q.data_ptr(), _ptr(dy_k), dq.data_ptr(), _ptr(dk),
                                      _ptr(dgain_q), _ptr(dgain_k), _ptr(ws), need, _queue(dev)),
              "bsa_rotary_backward")
    return dict(dq=dq, dk=dk, dgain_q=dgain_q, dgain_k=dgain_k)


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


# ---- cache of 8 bits ----

class Cache(NamedTuple):
    """Keys and values of packed sequences' caches as float8_e4m3fn [rows, kv_heads, d] (rows and heads multiples of 16
    bytes apart) and the codes of their scales, uint8 [kv_heads, rows]: k[t, h] stands for k[t, h].float() *
    2^(k_exp[h, t] - 127)."""
    k: torch.Tensor
    v: torch.Tensor
    k_exp: torch.Tensor
    v_exp: torch.Tensor


def cache_alloc(rows: int, kv_heads: int, head_dim: int, device="cuda") -> Cache:
    """A cache of `rows` rows in all (the capacities of its sequences, one behind another), zeroed."""
    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.uint8, device=device)
    k, v = (zeros(rows, kv_heads, head_dim).view(torch.float8_e4m3fn) for _ in range(2))
    return Cache(k, v, zeros(kv_heads, rows), zeros(kv_heads, rows))


def _cache_bytes(t, name, dev, shape=None):
    """(bytes between rows, between heads) of a cache's keys or values."""
    row, head = _any_heads(t, name, torch.float8_e4m3fn, dev, shape)
    if row % 16 or head % 16:
        raise ValueError(f"{name}'s rows and heads must lie multiples of 16 bytes apart")
    return row, head


def _cache_strides(cache, dev):
    ck = _cache_bytes(cache.k, "cache.k", dev)
    cv = _cache_bytes(cache.v, "cache.v", dev, cache.k.shape)
    rows, kv, _ = cache.k.shape
    _shaped(cache.k_exp, "cache.k_exp", (kv, rows), torch.uint8, dev)
    _shaped(cache.v_exp, "cache.v_exp", (kv, rows), torch.uint8, dev)
    return ck + cv


def _offsets(cu_q, cu_k, used_k, dev):
    _tensor(cu_q, "cu_q", torch.int32, dev)
    if cu_q.dim() != 1 or cu_q.numel() < 2 or not cu_q.is_contiguous():
        raise ValueError("cu_q must be a contiguous [sequences + 1] tensor")
    seqs = cu_q.numel() - 1
    _shaped(cu_k, "cu_k", (seqs + 1,), torch.int32, dev)
    if used_k is not None:
        _shaped(used_k, "used_k", (seqs,), torch.int32, dev)
    return seqs


def _call_key(name, cache, cu_q, cu_k, used_k, *more):
    sig = _signature
    k, v, k_exp, v_exp = cache
    return name, sig(k), sig(v), sig(k_exp), sig(v_exp), sig(cu_q), sig(cu_k), sig(used_k), more


def cache_write(cache, k, v, cu_q, cu_k, used_k=None, stream=None):
    """Quantises new rows k, v [rows, kv_heads, d] into the cache: those of sequence s, [cu_q[s], cu_q[s+1]), become the
    last of the used_k[s] rows in use behind its first row cu_k[s] (used_k None: of all up to cu_k[s+1]), where
    cache_attention_forward with the same offsets finds them. Other rows keep what they held."""
    lib = _lib.load()
    try:
        key = _call_key("cache_write", cache, cu_q, cu_k, used_k, _signature(k), _signature(v))
        p = _checked.get(key)
    except (AttributeError, TypeError, ValueError):
        key = p = None
    if p is None:
        k_row, k_head = _heads(k, "k")
        dev, dt = k.device, k.dtype
        v_row, v_head = _heads(v, "v", dt, dev, k.shape)
        strides = _cache_strides(cache, dev)
        rows, kv, d = cache.k.shape
        if k.shape[1:] != cache.k.shape[1:]:
            raise ValueError(f"k must have {kv} heads of {d}, got {tuple(k.shape)}")
        p = _remember(key, _lib.bsa_cache_t(_offsets(cu_q, cu_k, used_k, dev), kv, d, _CODES[dt], k.shape[0], rows, k_row,
                                            k_head, v_row, v_head, *strides))
    dev = k.device
    with _on(dev, stream):
        check(lib.bsa_cache_write(C.byref(p), k.data_ptr(), v.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), _ptr(used_k),
                                  cache.k.data_ptr(), cache.v.data_ptr(), cache.k_exp.data_ptr(), cache.v_exp.data_ptr(),
                                  _queue(dev)), "bsa_cache_write")


def cache_read(cache, rows: int, cu_q, cu_k, used_k=None, dtype=torch.bfloat16, stream=None):
    """The values of the cache rows that cache_write with these offsets writes: (k, v) [rows, kv_heads, d] in dtype
    (bfloat16 or float32; exact in both). Rows in no sequence are 0. With cu_q the running sum of used_k: all that
    the caches hold."""
    lib = _lib.load()
    rows = operator.index(rows)
    try:
        key = _call_key("cache_read", cache, cu_q, cu_k, used_k, rows, dtype)
        p = _checked.get(key)
    except (AttributeError, TypeError, ValueError):
        key = p = None
    if p is None:
        if dtype not in _CODES:
            raise ValueError(f"dtype must be bfloat16 or float32, got {dtype}")
        if rows < 0:
            raise ValueError("rows must be >= 0")
        _tensor(cache.k, "cache.k", torch.float8_e4m3fn)
        dev = cache.k.device
        strides = _cache_strides(cache, dev)
        total, kv, d = cache.k.shape
        p = _remember(key, _lib.bsa_cache_t(_offsets(cu_q, cu_k, used_k, dev), kv, d, _CODES[dtype], rows, total, 0, 0, 0, 0,
                                            *strides))
    dev = cache.k.device
    with _on(dev, stream):
        k = torch.empty((rows, p.kv_heads, p.head_dim), dtype=dtype, device=dev)
        v = torch.empty_like(k)
        check(lib.bsa_cache_read(C.byref(p), cache.k.data_ptr(), cache.v.data_ptr(), cache.k_exp.data_ptr(),
                                 cache.v_exp.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), _ptr(used_k), k.data_ptr(),
                                 v.data_ptr(), _queue(dev)), "bsa_cache_read")
    return k, v


def cache_attention_forward(q, cache, cu_q, cu_k, used_k=None, causal: bool = False, softmax_scale: float = 0.0, o=None,
                            lse=None, stream=None):
    """attention_forward of q [rows, heads, d] with the values of an 8-bit cache as keys and values. Returns (o, lse)."""
    lib = _lib.load()
    if (o is None) != (lse is None):
        raise ValueError("pass both o and lse, or neither")
    causal, softmax_scale = bool(causal), float(softmax_scale)
    try:
        key = _call_key("cache_attention_forward", cache, cu_q, cu_k, used_k, _signature(q), causal, softmax_scale, _signature(o),
                        _signature(lse))
        record = _checked.get(key)
    except (AttributeError, TypeError, ValueError):
        key = record = None
    if record is None:
        q_row, q_head = _heads(q, "q")
        dev, dt = q.device, q.dtype
        tq, h, d = q.shape
        strides = _cache_strides(cache, dev)
        rows, kv, _ = cache.k.shape
        if cache.k.shape[2] != d or kv == 0:
            raise ValueError(f"the cache must have head_dim {d} and at least one head, got {tuple(cache.k.shape)}")
        p = _lib.bsa_attention_t(_offsets(cu_q, cu_k, used_k, dev), h, kv, d, tq, rows, int(causal), _CODES[dt],
                                 softmax_scale, int(o is None), q_row, q_head, *strides, 0, 0, 0, 0)
        if o is not None:
            p.o_row, p.o_head = _heads(o, "o", dt, dev, q.shape)
            _shaped(lse, "lse", (h, tq), torch.float32, dev)
        need = C.c_size_t()
        check(lib.bsa_cache_attention_sizes(C.byref(p), C.byref(need)), "bsa_cache_attention_sizes")
        record = _remember(key, (p, need.value))
    p, need = record
    dev = q.device
    with _on(dev, stream):
        ws = _workspace(need, dev)
        if o is None:
            o = _fresh(q)
            lse = torch.empty((p.heads, p.total_q), dtype=torch.float32, device=dev)
        check(lib.bsa_cache_attention_forward(C.byref(p), q.data_ptr(), cache.k.data_ptr(), cache.v.data_ptr(),
                                              cache.k_exp.data_ptr(), cache.v_exp.data_ptr(), cu_q.data_ptr(),
                                              cu_k.data_ptr(), _ptr(used_k), o.data_ptr(), lse.data_ptr(), _ptr(ws), need,
                                              _queue(dev)), "bsa_cache_attention_forward")
    return o, lse
