"""ctypes binding of a recurrent layer's other operators: the short causal
convolution, the selective state space scan, linear attention with a decay for
each head, each for packed sequences and for one token per sequence, and low-rank adapters beside a shared projection
(``include/gdn_ssm.h``, ``include/gdn_linear.h``, ``include/gdn_lora.h``).

Argument checks and marshalling only, as in ``binding``.  Token rows may be
strided (columns of a projection's rows are passed as views, nothing is
copied); a call works on torch's current stream of its tensors' device,
whichever device is current.  These are serving operators: no gradient is
recorded.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

import torch

from .binding import (ConvShape, GDN_F32, LinearShape, LoraShape, SSMShape, _adapter_ids, _check, _dtype_code, _need, _ptr,
                      _seqlens, _stream, _workspace, _WORKSPACES, load_library)

GDN_ERR_WORKSPACE = 5

_ACTIVATIONS = {None: 0, "none": 0, "silu": 1}


def _on_device(fn, at=0):
    """Runs the call with the device of its argument number ``at`` current (kernels
    launch on the current device); free where it is current already."""
    name = fn.__code__.co_varnames[at]

    @functools.wraps(fn)
    def call(*args, **kwargs):
        first = args[at] if len(args) > at else kwargs.get(name)
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            raise ValueError(f"{fn.__name__} works on tensors in GPU memory")
        if first.get_device() == torch._C._cuda_getDevice():
            return fn(*args, **kwargs)
        with torch.cuda.device(first.device):
            return fn(*args, **kwargs)
    return call


def _rows(t, name, dtype, device, shape):
    """Checks a tensor of token rows ([T, ...] with dense rows); returns the
    distance of two rows in elements.  ``shape``: the row's shape."""
    # the usual tensor at once; anything else is looked at in turn
    if type(t) is torch.Tensor and t.dtype is dtype and t.device == device:
        size, strides = t.shape, t.stride()
        if len(shape) == 1:
            usual, width = len(size) == 2 and size[1] == shape[0] and strides[1] == 1, shape[0]
        else:
            usual = len(size) == 3 and size[2] == shape[1] and size[1] == shape[0] and strides[2] == 1 and \
                strides[1] == shape[1]
            width = shape[0] * shape[1]
        if usual:
            if size[0] <= 1:
                return width
            if strides[0] >= width:
                return strides[0]
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape[1:]) != shape:
        raise ValueError(f"{name} must be [T, {', '.join(map(str, shape))}], got {list(t.shape)}")
    width, strides = 1, t.stride()
    for d in range(len(shape) - 1, -1, -1):
        if shape[d] != 1 and strides[d + 1] != width:
            raise ValueError(f"the rows of {name} must be dense")
        width *= shape[d]
    if t.shape[0] <= 1:
        return width
    if strides[0] < width:
        raise ValueError(f"the rows of {name} must not overlap")
    return strides[0]


def _flat(t, name, shape, device):
    """Checks an optional fp32 parameter."""
    if t is None or (type(t) is torch.Tensor and t.shape == shape and t.dtype is torch.float32 and
                     t.device == device and t.is_contiguous()):
        return
    _need(t, name, torch.float32, device, len(shape))
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _offsets(cu_seqlens, cu_seqlens_host, device, tokens):
    cu, host = _seqlens(cu_seqlens, cu_seqlens_host, device)
    end = ctypes.c_int32.from_address(host.data_ptr() + 4 * (host.numel() - 1)).value   # host[-1], a quarter of its time
    if end > tokens:
        raise ValueError(f"cu_seqlens ends at {end}, behind the {tokens} token rows")
    return cu, host


def _run_with_workspace(call, size, shape, host, device, stream, given):
    """``call(workspace, its bytes)`` with the caller's workspace, or with the one
    kept per thread, device and stream; the library refuses a workspace that is too small
    before it enqueues anything, and only then its size is asked for.  (While a
    graph is captured, ``_workspace`` gives memory of the graph's.)"""
    if given is not None:
        if not isinstance(given, torch.Tensor) or given.device != device or not given.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {device}")
        _check(call(given.data_ptr(), given.numel() * given.element_size()))
        return
    if not torch._C._cuda_isCurrentStreamCapturing():
        kept = _WORKSPACES.kept.get((device.index, stream))
        status = call(None, 0) if kept is None else call(kept.data_ptr(), kept.numel())
        if status != GDN_ERR_WORKSPACE:
            _check(status)
            return
    need = ctypes.c_size_t(0)
    _check(size(ctypes.byref(shape), host, ctypes.byref(need)))
    ws = _workspace(need.value, device, stream)
    _check(call(ws.data_ptr(), ws.numel()))


# ---------------------------------------------------------------- short convolution

def _conv_args(x, weight, bias, activation, out):
    device = x.device
    if x.dim() != 2:
        raise ValueError("x must be [T, C]")
    T, C = x.shape
    _need(weight, "weight", torch.float32, device, 2)
    W = weight.shape[1]
    if weight.shape[0] != C:
        raise ValueError(f"weight must be [{C}, W], got {list(weight.shape)}")
    _flat(bias, "bias", (C,), device)
    if activation not in _ACTIVATIONS:
        raise ValueError("activation must be 'silu' or 'none'")
    ldx = _rows(x, "x", x.dtype, device, (C,))
    if out is None:
        out, ldy = torch.empty((T, C), dtype=x.dtype, device=device), C
    else:
        ldy = _rows(out, "out", x.dtype, device, (C,))
        if out.shape[0] != T:
            raise ValueError("out must hold as many token rows as x")
    return device, T, C, W, out, (C, W, _dtype_code(x), _ACTIVATIONS[activation], ldx, ldy)


def _history(t, name, n, W, C, dtype, device):
    if t is None or (type(t) is torch.Tensor and t.shape == (n, W - 1, C) and t.dtype is dtype and
                     t.device == device and t.is_contiguous()):
        return
    _need(t, name, dtype, device, 3)
    if t.shape != (n, W - 1, C):
        raise ValueError(f"{name} must be [N, W - 1, C]")


@_on_device
def causal_conv(x: torch.Tensor, weight: torch.Tensor, cu_seqlens, cu_seqlens_host=None,
                bias: Optional[torch.Tensor] = None, history_in: Optional[torch.Tensor] = None,
                activation: Optional[str] = "silu", out: Optional[torch.Tensor] = None,
                history_out: Optional[torch.Tensor] = None, write_history: bool = True):
    """Causal depthwise convolution of packed sequences on torch's current stream.

    x [T, C] (bf16 or fp32; rows may be strided, e.g. columns of a
    projection's rows), weight [C, W] fp32 with W of 2 to 4 taps (tap j
    multiplies token t - W + 1 + j), bias [C] fp32, ``history_in`` [N, W - 1, C]
    in x's dtype: the inputs before each sequence's first token, oldest first
    (None = zeros).  ``activation``: 'silu' or 'none'.  Returns ``(out [T, C],
    history_out [N, W - 1, C] or None)``; ``history_out`` holds the last W - 1
    inputs, from which ``causal_conv_step`` or a later call continues, and may
    be ``history_in``.  Rows of ``out`` behind the last sequence are left alone.
    """
    lib = load_library()
    device, T, C, W, out, shape = _conv_args(x, weight, bias, activation, out)
    cu, host = _offsets(cu_seqlens, cu_seqlens_host, device, T)
    n = host.numel() - 1
    _history(history_in, "history_in", n, W, C, x.dtype, device)
    if write_history and history_out is None:
        history_out = torch.empty((n, max(W - 1, 0), C), dtype=x.dtype, device=device)
    _history(history_out, "history_out", n, W, C, x.dtype, device)
    _check(lib.gdn_causal_conv(ctypes.byref(ConvShape(n, *shape)), host.data_ptr(), cu.data_ptr(), x.data_ptr(),
                               weight.data_ptr(), _ptr(bias), _ptr(history_in), out.data_ptr(), _ptr(history_out),
                               _stream(device)))
    return out, history_out


@_on_device
def causal_conv_step(x: torch.Tensor, weight: torch.Tensor, history_in: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, activation: Optional[str] = "silu",
                     out: Optional[torch.Tensor] = None, history_out: Optional[torch.Tensor] = None):
    """``causal_conv`` for one token per sequence: x [N, C], history_in [N, W - 1, C]
    (None = zeros).  Returns ``(out [N, C], history_out)``; pass
    ``history_out=history_in`` to update in place."""
    lib = load_library()
    device, n, C, W, out, shape = _conv_args(x, weight, bias, activation, out)
    _history(history_in, "history_in", n, W, C, x.dtype, device)
    if history_out is None:
        history_out = torch.empty((n, max(W - 1, 0), C), dtype=x.dtype, device=device)
    _history(history_out, "history_out", n, W, C, x.dtype, device)
    _check(lib.gdn_causal_conv_step(ctypes.byref(ConvShape(n, *shape)), x.data_ptr(), weight.data_ptr(),
                                    _ptr(bias), _ptr(history_in), out.data_ptr(), history_out.data_ptr(),
                                    _stream(device)))
    return out, history_out


# ---------------------------------------------------------------- state space scan

def _ssm_args(x, dt, a_log, B, C, d_skip, dt_bias, out):
    device, dtype = x.device, x.dtype
    if x.dim() != 3 or not isinstance(B, torch.Tensor) or B.dim() != 3:
        raise ValueError("x must be [T, H, head_dim] and B [T, G, d_state]")
    T, H, P = x.shape
    G, N = B.shape[1], B.shape[2]
    if not isinstance(dt, torch.Tensor) or dt.dtype not in (dtype, torch.float32):
        raise ValueError("dt must be a float32 tensor or one of x's dtype")
    ldx, ldb = _rows(x, "x", dtype, device, (H, P)), _rows(B, "B", dtype, device, (G, N))
    ldc = ldb if C is None else _rows(C, "C", dtype, device, (G, N))
    ldy = H * P if out is None else _rows(out, "out", dtype, device, (H, P))
    lddt = _rows(dt, "dt", dt.dtype, device, (H,))
    if B.shape[0] != T or dt.shape[0] != T or (C is not None and C.shape[0] != T) or \
            (out is not None and out.shape[0] != T):
        raise ValueError("dt, B, C and out must hold the same tokens as x")
    if a_log is None:
        raise TypeError("a_log must be a torch.Tensor")
    _flat(a_log, "a_log", (H,), device)
    _flat(d_skip, "d_skip", (H,), device)
    _flat(dt_bias, "dt_bias", (H,), device)
    code = _dtype_code(x)
    return device, T, H, P, N, (H, G, N, P, code, GDN_F32 if dt.dtype is torch.float32 else code, ldx, lddt, ldb, ldc,
                                ldy)


def _state(t, name, shape, device, dims="[N, H, d_state, head_dim]"):
    if t is None or (type(t) is torch.Tensor and t.shape == shape and t.dtype is torch.float32 and
                     t.device == device and t.is_contiguous()):
        return
    _need(t, name, torch.float32, device, 4)
    if t.shape != shape:
        raise ValueError(f"{name} must be {dims}")


@_on_device
def ssm_scan(x: torch.Tensor, dt: torch.Tensor, a_log: torch.Tensor, B: torch.Tensor, C: Optional[torch.Tensor],
             cu_seqlens, cu_seqlens_host=None, d_skip: Optional[torch.Tensor] = None,
             dt_bias: Optional[torch.Tensor] = None, state_in: Optional[torch.Tensor] = None, outputs: bool = True,
             out: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None, write_state: bool = True,
             workspace: Optional[torch.Tensor] = None):
    """Selective state space scan of packed sequences on torch's current stream.

    Per token and head: delta = softplus(dt + dt_bias), M = exp(-exp(a_log)
    delta) M + B (delta x)^T, y = M^T C + d_skip x.  x [T, H, head_dim], B and C
    [T, G, d_state] (bf16 or fp32, token rows may be strided; head h reads
    group h / (H / G)), dt [T, H] fp32 or x's dtype, a_log, d_skip and dt_bias
    [H] fp32, state_in [N, H, d_state, head_dim] fp32 (None = zero states).
    Returns ``(y [T, H, head_dim] in x's dtype, state_out)``; with
    ``outputs=False`` only the states are computed (a replayed tail's; y is
    None, C is not read and may be None).  ``state_out`` may be ``state_in``.
    Rows of ``out`` behind the last sequence are left alone.
    """
    lib = load_library()
    if not outputs:
        if out is not None or not write_state:
            raise ValueError("outputs=False computes the states alone: out must be None and write_state true")
        C = d_skip = None
    elif C is None:
        raise TypeError("C must be a torch.Tensor")
    device, T, H, P, N, shape = _ssm_args(x, dt, a_log, B, C, d_skip, dt_bias, out)
    cu, host = _offsets(cu_seqlens, cu_seqlens_host, device, T)
    n = host.numel() - 1
    if outputs and out is None:
        out = torch.empty((T, H, P), dtype=x.dtype, device=device)
    _state(state_in, "state_in", (n, H, N, P), device)
    if write_state and state_out is None:
        state_out = torch.empty((n, H, N, P), dtype=torch.float32, device=device)
    _state(state_out, "state_out", (n, H, N, P), device)
    shp = SSMShape(n, *shape)
    stream = _stream(device)
    lens = host.data_ptr()
    args = (ctypes.byref(shp), lens, cu.data_ptr(), x.data_ptr(), dt.data_ptr(), a_log.data_ptr(), B.data_ptr(), _ptr(C),
            _ptr(d_skip), _ptr(dt_bias), _ptr(state_in), _ptr(out), _ptr(state_out))
    _run_with_workspace(lambda ws, nbytes: lib.gdn_ssm_scan(*args, ws, nbytes, stream), lib.gdn_ssm_workspace_size, shp,
                        lens, device, stream, workspace)
    return out, state_out


@_on_device
def ssm_step(x: torch.Tensor, dt: torch.Tensor, a_log: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
             d_skip: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None,
             state_in: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             state_out: Optional[torch.Tensor] = None):
    """``ssm_scan`` for one token per sequence (T = N).  Returns ``(y [N, H,
    head_dim], state_out)``; pass ``state_out=state_in`` to update in place."""
    lib = load_library()
    if C is None:
        raise TypeError("C must be a torch.Tensor")
    device, n, H, P, N, shape = _ssm_args(x, dt, a_log, B, C, d_skip, dt_bias, out)
    if out is None:
        out = torch.empty((n, H, P), dtype=x.dtype, device=device)
    _state(state_in, "state_in", (n, H, N, P), device)
    if state_out is None:
        state_out = torch.empty((n, H, N, P), dtype=torch.float32, device=device)
    _state(state_out, "state_out", (n, H, N, P), device)
    _check(lib.gdn_ssm_step(ctypes.byref(SSMShape(n, *shape)), x.data_ptr(), dt.data_ptr(), a_log.data_ptr(), B.data_ptr(),
                            C.data_ptr(), _ptr(d_skip), _ptr(dt_bias), _ptr(state_in), out.data_ptr(),
                            state_out.data_ptr(), _stream(device)))
    return out, state_out


# ---------------------------------------------------------------- linear attention

def _linear_args(q, k, v, g, scale, out):
    device, dtype = v.device, v.dtype
    if v.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be [T, Hk, d_k] and v [T, Hv, d_v]")
    T, Hv, V = v.shape
    Hk, K = k.shape[1], k.shape[2]
    ldk, ldv = _rows(k, "k", dtype, device, (Hk, K)), _rows(v, "v", dtype, device, (Hv, V))
    ldq = ldk if q is None else _rows(q, "q", dtype, device, (Hk, K))
    ldo = Hv * V if out is None else _rows(out, "out", dtype, device, (Hv, V))
    if k.shape[0] != T or (q is not None and q.shape[0] != T) or (out is not None and out.shape[0] != T):
        raise ValueError("q, k and out must hold the same tokens as v")
    if g is None:
        raise TypeError("g must be a torch.Tensor")
    _flat(g, "g", (Hv,), device)
    return device, T, Hv, K, V, (Hk, Hv, K, V, _dtype_code(v), float(scale), ldq, ldk, ldv, ldo)


@functools.partial(_on_device, at=1)   # q may be None
def linear_attention(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, g: torch.Tensor, cu_seqlens,
                     cu_seqlens_host=None, scale: float = 1.0, state_in: Optional[torch.Tensor] = None,
                     outputs: bool = True, out: Optional[torch.Tensor] = None,
                     state_out: Optional[torch.Tensor] = None, write_state: bool = True,
                     workspace: Optional[torch.Tensor] = None):
    """Linear attention with a decay for each head, of packed sequences, on
    torch's current stream.

    Per token and value head: M = exp(g) M + k v^T, o = scale M^T q.  q, k
    [T, Hk, d_k], v [T, Hv, d_v] (bf16 or fp32, token rows may be strided; head h
    reads key head h / (Hv / Hk)), g [Hv] fp32 (log decays, <= 0), state_in
    [N, Hv, d_k, d_v] fp32 (None = zero states).  Returns ``(o [T, Hv, d_v] in
    v's dtype, state_out)``; with ``outputs=False`` only the states are computed
    (a replayed tail's; o is None, q is not read and may be None).  ``state_out``
    may be ``state_in``.  Rows of ``out`` behind the last sequence are left alone.
    """
    lib = load_library()
    if not outputs:
        if out is not None or not write_state:
            raise ValueError("outputs=False computes the states alone: out must be None and write_state true")
        q = None
    elif q is None:
        raise TypeError("q must be a torch.Tensor")
    device, T, Hv, K, V, shape = _linear_args(q, k, v, g, scale, out)
    cu, host = _offsets(cu_seqlens, cu_seqlens_host, device, T)
    n = host.numel() - 1
    if outputs and out is None:
        out = torch.empty((T, Hv, V), dtype=v.dtype, device=device)
    _state(state_in, "state_in", (n, Hv, K, V), device, "[N, Hv, d_k, d_v]")
    if write_state and state_out is None:
        state_out = torch.empty((n, Hv, K, V), dtype=torch.float32, device=device)
    _state(state_out, "state_out", (n, Hv, K, V), device, "[N, Hv, d_k, d_v]")
    shp = LinearShape(n, *shape)
    stream = _stream(device)
    lens = host.data_ptr()
    args = (ctypes.byref(shp), lens, cu.data_ptr(), _ptr(q), k.data_ptr(), v.data_ptr(), g.data_ptr(), _ptr(state_in),
            _ptr(out), _ptr(state_out))
    _run_with_workspace(lambda ws, nbytes: lib.gdn_linear_attention(*args, ws, nbytes, stream),
                        lib.gdn_linear_attention_workspace_size, shp, lens, device, stream, workspace)
    return out, state_out


@_on_device
def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, g: torch.Tensor,
                          state_in: Optional[torch.Tensor] = None, scale: float = 1.0,
                          out: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None):
    """``linear_attention`` for one token per sequence (T = N).  Returns ``(o [N,
    Hv, d_v], state_out)``; pass ``state_out=state_in`` to update in place."""
    lib = load_library()
    if q is None:
        raise TypeError("q must be a torch.Tensor")
    device, n, Hv, K, V, shape = _linear_args(q, k, v, g, scale, out)
    if out is None:
        out = torch.empty((n, Hv, V), dtype=v.dtype, device=device)
    _state(state_in, "state_in", (n, Hv, K, V), device, "[N, Hv, d_k, d_v]")
    if state_out is None:
        state_out = torch.empty((n, Hv, K, V), dtype=torch.float32, device=device)
    _state(state_out, "state_out", (n, Hv, K, V), device, "[N, Hv, d_k, d_v]")
    _check(lib.gdn_linear_attention_step(ctypes.byref(LinearShape(n, *shape)), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                         g.data_ptr(), _ptr(state_in), out.data_ptr(), state_out.data_ptr(),
                                         _stream(device)))
    return out, state_out


# ---------------------------------------------------------------- low-rank adapters

@_on_device
def lora_add(base: torch.Tensor, x: torch.Tensor, lora_a: torch.Tensor, lora_b: torch.Tensor, adapters, cu_seqlens,
             cu_seqlens_host=None, adapters_host=None, scales: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Adds each request's low-rank adapter to a shared projection's result, on
    torch's current stream: out[t] = base[t] + scales[a] (x[t] A_a^T) B_a^T with
    a the adapter of token t's sequence, out[t] = base[t] where a is -1.

    base [T, M] bf16 or fp32: the projection of x [T, K] bf16 (rows of both may
    be strided); lora_a [n, R, K] and lora_b [n, M, R] bf16, R a multiple of 8 up
    to 128 (pad smaller adapters with zeros); adapters: one int32 index per
    sequence of ``cu_seqlens``; scales [n] fp32 (None = 1).  ``out`` may be
    ``base`` (added in place).  Rows behind the last sequence are left alone.
    """
    lib = load_library()
    device = base.device
    if base.dim() != 2 or not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("base must be [T, M] and x [T, K]")
    T, M = base.shape
    K = x.shape[1]
    if x.shape[0] != T:
        raise ValueError("base and x must hold the same tokens")
    ldbase = _rows(base, "base", base.dtype, device, (M,))
    ldx = _rows(x, "x", torch.bfloat16, device, (K,))
    _need(lora_a, "lora_a", torch.bfloat16, device, 3)
    _need(lora_b, "lora_b", torch.bfloat16, device, 3)
    na, R = lora_a.shape[0], lora_a.shape[1]
    if lora_a.shape[2] != K or tuple(lora_b.shape) != (na, M, R):
        raise ValueError("lora_a must be [n, R, K] and lora_b [n, M, R]")
    _flat(scales, "scales", (na,), device)
    if out is None:
        out, ldout = torch.empty((T, M), dtype=base.dtype, device=device), M
    else:
        ldout = _rows(out, "out", base.dtype, device, (M,))
        if out.shape[0] != T:
            raise ValueError("out must hold the same tokens as base")
    cu, host = _offsets(cu_seqlens, cu_seqlens_host, device, T)
    n = host.numel() - 1
    ids, ids_host = _adapter_ids(adapters, adapters_host, n, device)
    shp = LoraShape(n, na, K, M, R, _dtype_code(base), ldx, ldbase, ldout)
    stream = _stream(device)
    lens = host.data_ptr()
    args = (ctypes.byref(shp), lens, cu.data_ptr(), ids_host.data_ptr(), ids.data_ptr(), base.data_ptr(), x.data_ptr(),
            lora_a.data_ptr(), lora_b.data_ptr(), _ptr(scales), out.data_ptr())
    _run_with_workspace(lambda ws, nbytes: lib.gdn_lora_add(*args, ws, nbytes, stream), lib.gdn_lora_workspace_size, shp,
                        lens, device, stream, workspace)
    return out
