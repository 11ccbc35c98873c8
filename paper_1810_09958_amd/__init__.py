"""MI355X (gfx950) hot path of ISA Mapper (arXiv 1810.09958): GEMM, separable depthwise
convolution and GRU forward, and the operators of a gated recurrent language-model block with
their gradients, as hand-written HIP kernels behind the C ABI in ``include/isam.h``.

This module is argument marshalling only: it checks torch tensors (device, dtype,
contiguity), sizes and allocates the workspace, and calls the C ABI on torch's current
stream.  Every arithmetic step runs in the library's kernels.  If ``libisam.so`` is
missing the calls raise; there is no fallback.  No call is recorded by torch's autograd,
whatever its inputs require: gradients come from the ``*_backward`` calls.
"""
from __future__ import annotations

import ctypes
import os

import torch

from ._lib import (ISAM_BF16, ISAM_F32, IsamError, lib, lib_path)

__all__ = ["gemm", "conv1d", "dwsep_conv", "gru_forward", "gru_forward_noalloc", "gemm_workspace_size",
           "dwsep_conv_workspace_size", "gru_forward_workspace_size", "IsamError",
           "linear_gru", "linear_gru_backward", "linear_gru_states_shape", "linear_gru_workspace_size",
           "linear_gru_backward_workspace_size", "norm_residual", "norm_residual_backward",
           "norm_residual_backward_workspace_size", "gated_ffn", "gated_ffn_backward", "gated_ffn_workspace_size",
           "gated_ffn_backward_workspace_size",
           "selective_scan", "selective_scan_backward", "selective_scan_states_shape", "selective_scan_workspace_size",
           "selective_scan_backward_workspace_size", "causal_conv", "causal_conv_backward",
           "causal_conv_backward_workspace_size", "beam_step", "beam_step_workspace_size", "beam_reorder", "linear", "linear_backward", "linear_workspace_size",
           "linear_backward_workspace_size", "lib", "lib_path", "ISAM_F32", "ISAM_BF16", "version"]

_DT = {torch.float32: ISAM_F32, torch.bfloat16: ISAM_BF16}


def _dt(t: torch.Tensor) -> int:
    try:
        return _DT[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16") from None


def _ptr(t):
    # plain ints: the ctypes signatures convert them (no per-call c_void_p objects)
    return None if t is None else t.data_ptr()


try:
    _raw_stream = torch._C._cuda_getCurrentRawStream  # current stream handle, no Stream object
except AttributeError:  # pragma: no cover - older torch
    _raw_stream = None


def _stream(device=None):
    """The current stream of the current GPU (`device`, where the caller has asked for it already)."""
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device() if device is None else device)
    return torch.cuda.current_stream().cuda_stream


def _check_dev(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("tensors must be on the GPU")


def _call(rc, name):
    if rc != 0:
        L = lib()
        raise IsamError(rc, f"{name}: {L.isam_status_string(rc).decode()}: {L.isam_last_error().decode()}")


def version() -> int:
    return lib().isam_version()


def conv1d(A: torch.Tensor, B: torch.Tensor, out: torch.Tensor | None = None, *, accumulate=False,
           out_dtype=None):
    """1D convolution (valid, stride 1): C[i][x][ko] (+)= sum_{d,ki} A[i][x+d][ki] * B[d][ki][ko].
    A is [batch][L][Ki], B is [D][Ki][Ko], both contiguous and of one dtype; returns C
    ([batch][L-D+1][Ko], float32 unless out_dtype / out say otherwise)."""
    _check_dev(A, B, out)
    if A.dim() != 3 or B.dim() != 3:
        raise ValueError("A must be [batch][L][Ki] and B [D][Ki][Ko]")
    if not A.is_contiguous() or not B.is_contiguous():
        raise ValueError("A and B must be contiguous")
    if A.dtype != B.dtype:
        raise TypeError("A and B must share a dtype")
    nb, L, Ki = A.shape
    D, Ki2, Ko = B.shape
    if Ki2 != Ki:
        raise ValueError(f"channel counts differ: {Ki} vs {Ki2}")
    X = max(L - D + 1, 0)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((nb, X, Ko), device=A.device, dtype=out_dtype or torch.float32)
    elif tuple(out.shape) != (nb, X, Ko) or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous [{nb}][{X}][{Ko}] tensor")
    rc = lib().isam_conv1d(nb, L, Ki, D, Ko, _dt(A), _ptr(A), _ptr(B), int(accumulate), _dt(out), _ptr(out),
                           _stream())
    _call(rc, "isam_conv1d")
    return out


def gemm_workspace_size(M, N, K, ab_type, c_type, trans_a=0, trans_b=0) -> int:
    return lib().isam_gemm_workspace_size(trans_a, trans_b, M, N, K, ab_type, c_type)


def gemm(A: torch.Tensor, B: torch.Tensor, out: torch.Tensor | None = None, *, trans_a=False,
         trans_b=False, accumulate=False, out_dtype=None, workspace: torch.Tensor | None = None):
    """C (+)= op(A) op(B).  A is [M][K] ([K][M] with trans_a); B is [K][N] ([N][K] with
    trans_b).  Row strides may exceed the row length (leading dimensions); the inner stride
    must be 1.  Returns C ([M][N], float32 unless out_dtype / out say otherwise)."""
    _check_dev(A, B, out, workspace)
    if A.dim() != 2 or B.dim() != 2:
        raise ValueError("A and B must be 2-D")
    if A.stride(1) != 1 or B.stride(1) != 1:
        raise ValueError("A and B need unit inner stride")
    M, K = (A.shape[1], A.shape[0]) if trans_a else (A.shape[0], A.shape[1])
    KB, N = (B.shape[1], B.shape[0]) if trans_b else (B.shape[0], B.shape[1])
    if KB != K:
        raise ValueError(f"inner sizes differ: {K} vs {KB}")
    if A.dtype != B.dtype:
        raise TypeError("A and B must share a dtype")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((M, N), device=A.device, dtype=out_dtype or torch.float32)
    if out.shape != (M, N) or (N > 0 and out.stride(1) != 1):
        raise ValueError("out must be [M][N] with unit inner stride")
    ab, ct = _dt(A), _dt(out)
    if workspace is None:
        need = gemm_workspace_size(M, N, K, ab, ct, int(trans_a), int(trans_b))
        workspace = torch.empty(max(need, 1), device=A.device, dtype=torch.uint8)
    rc = lib().isam_gemm(int(trans_a), int(trans_b), M, N, K, ab, _ptr(A), max(A.stride(0), 1),
                         _ptr(B), max(B.stride(0), 1), int(accumulate), ct, _ptr(out),
                         max(out.stride(0), 1), _ptr(workspace), workspace.numel(), _stream())
    _call(rc, "isam_gemm")
    return out


def dwsep_conv_workspace_size(batch, H, W, C_in, depth_mult, kh, kw, stride, pad, C_out,
                              in_type, out_type) -> int:
    return lib().isam_dwsep_conv_workspace_size(batch, H, W, C_in, depth_mult, kh, kw, stride,
                                                pad, C_out, in_type, out_type)


def dwsep_conv(x: torch.Tensor, dw_filter: torch.Tensor, pw_weight: torch.Tensor, *, stride=1,
               pad=1, out: torch.Tensor | None = None, out_dtype=None,
               workspace: torch.Tensor | None = None):
    """Separable depthwise convolution (depthwise kh x kw, then pointwise 1x1), NHWC.
    x [b][H][W][C_in], dw_filter [kh][kw][C_in][c], pw_weight [C_in*c][C_out]."""
    _check_dev(x, dw_filter, pw_weight, out, workspace)
    for t in (x, dw_filter, pw_weight):
        if not t.is_contiguous():
            raise ValueError("inputs must be contiguous")
    if not (x.dtype == dw_filter.dtype == pw_weight.dtype):
        raise TypeError("x, dw_filter and pw_weight must share a dtype")
    b, H, W, C = x.shape
    kh, kw, C2, cm = dw_filter.shape
    Cm, Co = pw_weight.shape
    if C2 != C or Cm != C * cm:
        raise ValueError("filter shapes do not match x")
    Ho = (H + 2 * pad - kh) // stride + 1
    Wo = (W + 2 * pad - kw) // stride + 1
    if out is None:
        out = torch.empty((b, Ho, Wo, Co), device=x.device, dtype=out_dtype or torch.float32)
    if not out.is_contiguous() or tuple(out.shape) != (b, Ho, Wo, Co):
        raise ValueError("out must be contiguous [b][Ho][Wo][C_out]")
    it, ot = _dt(x), _dt(out)
    if workspace is None:
        need = dwsep_conv_workspace_size(b, H, W, C, cm, kh, kw, stride, pad, Co, it, ot)
        workspace = torch.empty(max(need, 1), device=x.device, dtype=torch.uint8)
    rc = lib().isam_dwsep_conv(b, H, W, C, cm, kh, kw, stride, pad, Co, it, _ptr(x),
                               _ptr(dw_filter), _ptr(pw_weight), ot, _ptr(out), _ptr(workspace),
                               workspace.numel(), _stream())
    _call(rc, "isam_dwsep_conv")
    return out


def gru_forward_workspace_size(T, batch, input_size, hidden, w_type) -> int:
    return lib().isam_gru_forward_workspace_size(T, batch, input_size, hidden, w_type)


def gru_forward(x: torch.Tensor, W: torch.Tensor, U: torch.Tensor, *, bias=None, bias_hn=None,
                h0=None, return_sequence=True, h_seq=None, h_T=None,
                workspace: torch.Tensor | None = None):
    """GRU forward.  x [T][batch][I], W [3H][I], U [3H][H] (gate rows r, z, n; float32 or
    bfloat16), bias [3H], bias_hn [H], h0 [batch][H] float32 or None.  Returns (h_seq, h_T)."""
    _check_dev(x, W, U, bias, bias_hn, h0, h_seq, h_T, workspace)
    for t in (x, W, U, bias, bias_hn, h0):
        if t is not None and not t.is_contiguous():
            raise ValueError("inputs must be contiguous")
    if not (x.dtype == W.dtype == U.dtype):
        raise TypeError("x, W, U must share a dtype")
    for t in (bias, bias_hn, h0):
        if t is not None and t.dtype != torch.float32:
            raise TypeError("bias, bias_hn and h0 are float32")
    T, B, I = x.shape
    H = U.shape[1]
    if tuple(W.shape) != (3 * H, I) or tuple(U.shape) != (3 * H, H):
        raise ValueError("W must be [3H][I] and U [3H][H]")
    dev = x.device
    if h_seq is None and return_sequence:
        h_seq = torch.empty((T, B, H), device=dev, dtype=torch.float32)
    if h_T is None:
        h_T = torch.empty((B, H), device=dev, dtype=torch.float32)
    wt = _dt(W)
    if workspace is None:
        need = gru_forward_workspace_size(T, B, I, H, wt)
        workspace = torch.empty(max(need, 1), device=dev, dtype=torch.uint8)
    rc = lib().isam_gru_forward(T, B, I, H, wt, _ptr(x), _ptr(h0), _ptr(W), _ptr(U), _ptr(bias),
                                _ptr(bias_hn), _ptr(h_seq), _ptr(h_T), _ptr(workspace),
                                workspace.numel(), _stream())
    _call(rc, "isam_gru_forward")
    return h_seq, h_T


def gru_forward_noalloc(x: torch.Tensor, W: torch.Tensor, U: torch.Tensor, h_seq: torch.Tensor,
                        h_T: torch.Tensor, *, bias=None, bias_hn=None, h0=None):
    """GRU forward through isam_gru_forward_noalloc: the library's static device scratch
    serves as workspace and nothing is allocated (h_seq and h_T are caller-provided; either
    may be None, not both).  Calls that overlap in time on one device race."""
    _check_dev(x, W, U, bias, bias_hn, h0, h_seq, h_T)
    for t in (x, W, U, bias, bias_hn, h0, h_seq, h_T):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensors must be contiguous")
    if not (x.dtype == W.dtype == U.dtype):
        raise TypeError("x, W, U must share a dtype")
    T, B, I = x.shape
    H = U.shape[1]
    rc = lib().isam_gru_forward_noalloc(T, B, I, H, _dt(W), _ptr(x), _ptr(h0), _ptr(W), _ptr(U), _ptr(bias),
                                        _ptr(bias_hn), _ptr(h_seq), _ptr(h_T), _stream())
    _call(rc, "isam_gru_forward_noalloc")
    return h_seq, h_T


# ---------------------------------------------------------------------------------------
# Linear GRU
# ---------------------------------------------------------------------------------------
_CANDIDATES = {"linear": 0, "tanh": 1}


def _code(table, name, what):
    try:
        return table[name]
    except (KeyError, TypeError):
        raise ValueError(f"{what} must be one of {', '.join(sorted(table))}") from None


def _want(t, name, shape, dtype=torch.float32):
    """Checks a contiguous tensor argument (None passes)."""
    if t is None:
        return
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} tensor")


def _rows(t, name, shape, dtype):
    """Strides of the rows of a [T][batch][width] tensor with unit inner stride (None: zeros)."""
    if t is None:
        return 0, 0
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    st = t.stride()
    if len(st) == 3 and st[2] != 1 and shape[2] > 1:
        raise ValueError(f"{name} needs unit inner stride")
    return st[0], st[1]


def _on(first, *ts):
    """Checks that every tensor given is on the current GPU, whose stream the call runs on; its number."""
    at = first.get_device()
    if at < 0:
        raise ValueError("tensors must be on the GPU")
    if at != torch.cuda.current_device():
        raise ValueError("tensors must be on the current GPU (torch.cuda.set_device)")
    for t in ts:
        if t is not None and t.get_device() != at:
            raise ValueError("tensors must be on one GPU")
    return at


def _room(nbytes, dev):
    return torch.empty(max(nbytes, 1), device=dev, dtype=torch.uint8)


def _bytes(t):
    return t.numel() * t.element_size()


def linear_gru_workspace_size(T, batch, hidden, dtype) -> int:
    return lib().isam_linear_gru_workspace_size(T, batch, hidden, dtype)


def linear_gru_backward_workspace_size(T, batch, hidden, dtype) -> int:
    return lib().isam_linear_gru_backward_workspace_size(T, batch, hidden, dtype)


def linear_gru_states_shape(T, batch, hidden):
    """Shape of the ``states`` tensor: the state before steps 0, 128, 256, ..."""
    return (T + 127) // 128, batch, hidden


def _linear_gru_args(gx, bias, reset):
    if gx.dim() != 3 or gx.shape[2] % 2:
        raise ValueError("gx must be [T][batch][2 * hidden]")
    T, B, H2 = gx.shape
    _want(bias, "bias", (H2,))
    gs = _rows(gx, "gx", (T, B, H2), gx.dtype)
    if reset is not None and reset.dtype not in (torch.bool, torch.uint8):
        raise TypeError("reset must be bool or uint8")
    rs = (0, 0) if reset is None else _rows(reset, "reset", (T, B), reset.dtype)
    return T, B, H2 // 2, _dt(gx), gs, rs


def linear_gru(gx: torch.Tensor, *, bias=None, h0=None, reset=None, candidate="tanh", return_sequence=True, h_seq=None,
               h_T=None, states=None, workspace: torch.Tensor | None = None):
    """Linear GRU (gates that do not see the state): h_t = z_t h_{t-1} + (1 - z_t) n_t with z =
    sigmoid(gz + b_z) and n = tanh(gn + b_n), or gn + b_n for candidate="linear".
    gx [T][batch][2H] (blocks z, n; float32 or bfloat16; any strides of the first two
    dimensions, so batch-first tensors go in transposed), bias [2H] and h0 [batch][H] float32,
    reset [T][batch] bool (the step starts from a zero state).  states
    (``linear_gru_states_shape``, float32) receives what ``linear_gru_backward`` needs.
    Returns (h_seq in gx's dtype, h_T in float32)."""
    at = _on(gx, bias, h0, reset, h_seq, h_T, states, workspace)
    T, B, H, dt, gs, rs = _linear_gru_args(gx, bias, reset)
    cand = _code(_CANDIDATES, candidate, "candidate")
    dev = gx.device
    _want(h0, "h0", (B, H))
    _want(states, "states", linear_gru_states_shape(T, B, H))
    if h_seq is None and return_sequence:
        h_seq = torch.empty((T, B, H), device=dev, dtype=gx.dtype)
    if h_T is None:
        h_T = torch.empty((B, H), device=dev, dtype=torch.float32)
    _want(h_T, "h_T", (B, H))
    hs = _rows(h_seq, "h_seq", (T, B, H), gx.dtype)
    if workspace is None:
        workspace = _room(linear_gru_workspace_size(T, B, H, dt), dev)
    rc = lib().isam_linear_gru(T, B, H, dt, cand, _ptr(gx), *gs, _ptr(bias), _ptr(h0), _ptr(reset), *rs, _ptr(h_seq), *hs,
                               _ptr(h_T), _ptr(states), _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_linear_gru")
    return h_seq, h_T


def linear_gru_backward(gx: torch.Tensor, dh_seq: torch.Tensor | None, *, states, bias=None, reset=None, candidate="tanh",
                        dh_T=None, dgx=None, dh0=None, dbias=None, workspace: torch.Tensor | None = None):
    """Gradient of ``linear_gru``: gx, bias, reset, candidate and states as in (and from) the forward
    call, dh_seq [T][batch][H] in gx's dtype or None, dh_T [batch][H] float32 or None.  Returns
    (dgx in gx's dtype, dh0, dbias in float32; dbias is None without a bias unless given)."""
    at = _on(gx, dh_seq, states, bias, reset, dh_T, dgx, dh0, dbias, workspace)
    T, B, H, dt, gs, rs = _linear_gru_args(gx, bias, reset)
    cand = _code(_CANDIDATES, candidate, "candidate")
    dev = gx.device
    _want(states, "states", linear_gru_states_shape(T, B, H))
    _want(dh_T, "dh_T", (B, H))
    ds = _rows(dh_seq, "dh_seq", (T, B, H), gx.dtype)
    if dgx is None:
        dgx = torch.empty((T, B, 2 * H), device=dev, dtype=gx.dtype)
    if dh0 is None:
        dh0 = torch.empty((B, H), device=dev, dtype=torch.float32)
    if dbias is None and bias is not None:
        dbias = torch.empty((2 * H,), device=dev, dtype=torch.float32)
    _want(dh0, "dh0", (B, H))
    _want(dbias, "dbias", (2 * H,))
    dgs = _rows(dgx, "dgx", (T, B, 2 * H), gx.dtype)
    if workspace is None:
        workspace = _room(linear_gru_backward_workspace_size(T, B, H, dt), dev)
    rc = lib().isam_linear_gru_backward(T, B, H, dt, cand, _ptr(gx), *gs, _ptr(bias), _ptr(reset), *rs, _ptr(states),
                                        _ptr(dh_seq), *ds, _ptr(dh_T), _ptr(dgx), *dgs, _ptr(dh0), _ptr(dbias),
                                        _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_linear_gru_backward")
    return dgx, dh0, dbias


# ---------------------------------------------------------------------------------------
# Gated residual norm
# ---------------------------------------------------------------------------------------
def _matrix(t, name, shape, dtype):
    """Leading dimension of a [rows][D] tensor with unit inner stride (None: 0)."""
    if t is None:
        return 0
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    ld, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError(f"{name} needs unit inner stride")
    return ld if shape[0] > 1 else shape[1]


def _norm_args(r, gate, w_post, w_pre):
    if r.dim() != 2:
        raise ValueError("rows must be [rows][D]")
    R, D = r.shape
    if gate is not None and (gate.dim() != 2 or gate.shape[1] != D or (R and (gate.shape[0] == 0 or R % gate.shape[0]))):
        raise ValueError("gate must be [gates][D] with gates a divisor of rows")
    G = 1 if gate is None else gate.shape[0]
    _want(gate, "gate", (G, D), r.dtype)
    _want(w_post, "w_post", (D,))
    _want(w_pre, "w_pre", (D,))
    return R, D, G


def norm_residual_backward_workspace_size(rows, D, gates, dtype) -> int:
    return lib().isam_norm_residual_backward_workspace_size(rows, D, gates, dtype)


def norm_residual(x: torch.Tensor | None, r: torch.Tensor, *, w_pre, w_post=None, gate=None, scale=1.0, eps=1e-6, r_out=None,
                  y=None):
    """Gated residual norm over rows: r_out = r + scale * gate * u with u = x / rms(x) * w_post (u = x
    without w_post), y = r_out / rms(r_out) * w_pre, rms(v) = sqrt(mean(v^2) + eps).
    x, r [rows][D] (float32 or bfloat16; row strides may exceed D), gate [gates][D] in their
    dtype with gates a divisor of rows, w_post and w_pre [D] float32.  r_out may be r.
    x None: y = norm of r alone.  Returns (r_out, y); r_out is r without x."""
    at = _on(r, x, w_pre, w_post, gate, r_out, y)
    R, D, G = _norm_args(r, gate, w_post, w_pre)
    dt, dev = _dt(r), r.device
    if r_out is None and x is not None:
        r_out = torch.empty((R, D), device=dev, dtype=r.dtype)
    if y is None:
        y = torch.empty((R, D), device=dev, dtype=r.dtype)
    shape, ty = (R, D), r.dtype
    ldx, ldr = _matrix(x, "x", shape, ty), _matrix(r, "r", shape, ty)
    ldro, ldy = _matrix(r_out, "r_out", shape, ty), _matrix(y, "y", shape, ty)
    rc = lib().isam_norm_residual(R, D, G, dt, _ptr(x), ldx, _ptr(r), ldr, _ptr(gate), _ptr(w_post), _ptr(w_pre), scale, eps,
                                  _ptr(r_out), ldro, _ptr(y), ldy, _stream(at))
    _call(rc, "isam_norm_residual")
    return (r if x is None else r_out), y


def norm_residual_backward(x: torch.Tensor | None, r_out: torch.Tensor, dy: torch.Tensor, *, w_pre, w_post=None, gate=None,
                           scale=1.0, eps=1e-6, dr_out=None, dx=None, dr=None, dgate=None, dw_post=None, dw_pre=None,
                           workspace: torch.Tensor | None = None):
    """Gradient of ``norm_residual``: x, gate, w_post, w_pre, scale and eps as in the forward call, r_out
    as it left it, dy and dr_out (None for zeros) the gradients of y and r_out.  dr may be dr_out.
    Returns (dx, dr, dgate, dw_post, dw_pre), None where the forward call had no such input."""
    at = _on(r_out, x, dy, w_pre, w_post, gate, dr_out, dx, dr, dgate, dw_post, dw_pre, workspace)
    R, D, G = _norm_args(r_out, gate, w_post, w_pre)
    dt, dev, shape, ty = _dt(r_out), r_out.device, (R, D), r_out.dtype
    if dx is None and x is not None:
        dx = torch.empty(shape, device=dev, dtype=ty)
    if dr is None:
        dr = torch.empty(shape, device=dev, dtype=ty)
    if dgate is None and gate is not None:
        dgate = torch.empty((G, D), device=dev, dtype=ty)
    if dw_post is None and w_post is not None:
        dw_post = torch.empty((D,), device=dev, dtype=torch.float32)
    if dw_pre is None:
        dw_pre = torch.empty((D,), device=dev, dtype=torch.float32)
    _want(dgate, "dgate", (G, D), ty)
    _want(dw_post, "dw_post", (D,))
    _want(dw_pre, "dw_pre", (D,))
    if workspace is None:
        workspace = _room(norm_residual_backward_workspace_size(R, D, G, dt), dev)
    rc = lib().isam_norm_residual_backward(
        R, D, G, dt, _ptr(x), _matrix(x, "x", shape, ty), _ptr(r_out), _matrix(r_out, "r_out", shape, ty), _ptr(gate),
        _ptr(w_post), _ptr(w_pre), scale, eps, _ptr(dy), _matrix(dy, "dy", shape, ty), _ptr(dr_out),
        _matrix(dr_out, "dr_out", shape, ty), _ptr(dx), _matrix(dx, "dx", shape, ty), _ptr(dr), _matrix(dr, "dr", shape, ty),
        _ptr(dgate), _ptr(dw_post), _ptr(dw_pre), _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_norm_residual_backward")
    return dx, dr, dgate, dw_post, dw_pre


# ---------------------------------------------------------------------------------------
# Gated feed-forward block
# ---------------------------------------------------------------------------------------
_ACTIVATIONS = {"sigmoid": 0, "silu": 1, "gelu": 2}
_NONE = 3  # no activation


def gated_ffn_workspace_size(M, K, F, dtype, aligned=True) -> int:
    return lib().isam_gated_ffn_workspace_size(M, K, F, dtype, int(aligned))


def gated_ffn_backward_workspace_size(M, K, F, dtype, aligned=True) -> int:
    return lib().isam_gated_ffn_backward_workspace_size(M, K, F, dtype, int(aligned))


def _gated_args(x, W, bias):
    if x.dim() != 2 or W.dim() != 2 or W.shape[0] % 2 or W.shape[1] != x.shape[1]:
        raise ValueError("x must be [M][K] and W [2 * F][K]")
    M, K = x.shape
    F = W.shape[0] // 2
    _want(bias, "bias", (2 * F,))
    return M, K, F, _dt(x), _matrix(x, "x", (M, K), x.dtype), _matrix(W, "W", (2 * F, K), x.dtype)


def _aligned(t, ld):
    return t.data_ptr() % 16 == 0 and ld % 8 == 0


def gated_ffn(x: torch.Tensor, W: torch.Tensor, *, bias=None, activation="silu", out=None,
              workspace: torch.Tensor | None = None):
    """Gated feed-forward block: act(x Wg^T + bg) * (x Wu^T + bu), both projections, the activation
    ("sigmoid", "silu" or "gelu") and the product together.  x [M][K], W [2F][K] (gate rows, then up
    rows; float32 or bfloat16; row strides may exceed K), bias [2F] float32.  Returns out [M][F] in
    x's dtype."""
    at = _on(x, W, bias, out, workspace)
    M, K, F, dt, ldx, ldw = _gated_args(x, W, bias)
    act, dev = _code(_ACTIVATIONS, activation, "activation"), x.device
    if out is None:
        out = torch.empty((M, F), device=dev, dtype=x.dtype)
    ldo = _matrix(out, "out", (M, F), x.dtype)
    if workspace is None:
        workspace = _room(gated_ffn_workspace_size(M, K, F, dt, _aligned(x, ldx) and _aligned(W, ldw)), dev)
    rc = lib().isam_gated_ffn(M, K, F, dt, act, _ptr(x), ldx, _ptr(W), ldw, _ptr(bias), _ptr(out), ldo, _ptr(workspace),
                              _bytes(workspace), _stream(at))
    _call(rc, "isam_gated_ffn")
    return out


def gated_ffn_backward(x: torch.Tensor, W: torch.Tensor, dout: torch.Tensor, *, bias=None, activation="silu", return_dx=True,
                       return_dW=True, dx=None, dW=None, dbias=None, workspace: torch.Tensor | None = None):
    """Gradient of ``gated_ffn`` from dout [M][F]: the projections are formed again, nothing is kept
    from the forward call.  Returns (dx [M][K], dW [2F][K] in x's dtype, dbias [2F] float32 or
    None without a bias).  bfloat16 beyond 16 rows: the projections' gradients are rounded as the
    products' operands, so dx and dW carry two roundings.  return_dx or return_dW False (frozen inputs or weights): that product is
    left out, and None stands for it.  F = 0: dx is zeros."""
    at = _on(x, W, dout, bias, dx, dW, dbias, workspace)
    M, K, F, dt, ldx, ldw = _gated_args(x, W, bias)
    act, dev = _code(_ACTIVATIONS, activation, "activation"), x.device
    if dx is None and return_dx:
        dx = torch.empty((M, K), device=dev, dtype=x.dtype)
    if dW is None and return_dW:
        dW = torch.empty((2 * F, K), device=dev, dtype=x.dtype)
    if dbias is None and bias is not None:
        dbias = torch.empty((2 * F,), device=dev, dtype=torch.float32)
    _want(dbias, "dbias", (2 * F,))
    lddo, lddx = _matrix(dout, "dout", (M, F), x.dtype), _matrix(dx, "dx", (M, K), x.dtype)
    lddw = _matrix(dW, "dW", (2 * F, K), x.dtype)
    if F == 0:  # (a sum of nothing; the C entry takes no dx then)
        if dx is not None:
            dx.zero_()
        return dx, dW, dbias
    if workspace is None:
        workspace = _room(gated_ffn_backward_workspace_size(M, K, F, dt, _aligned(x, ldx) and _aligned(W, ldw)), dev)
    rc = lib().isam_gated_ffn_backward(M, K, F, dt, act, _ptr(x), ldx, _ptr(W), ldw, _ptr(bias), _ptr(dout), lddo, _ptr(dx), lddx,
                                       _ptr(dW), lddw, _ptr(dbias), _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_gated_ffn_backward")
    return dx, dW, dbias


# ---------------------------------------------------------------------------------------
# Selective scan
# ---------------------------------------------------------------------------------------
def selective_scan_workspace_size(T, batch, D, N, dtype) -> int:
    return lib().isam_selective_scan_workspace_size(T, batch, D, N, dtype)


def selective_scan_backward_workspace_size(T, batch, D, N, dtype) -> int:
    return lib().isam_selective_scan_backward_workspace_size(T, batch, D, N, dtype)


def selective_scan_states_shape(T, batch, D, N):
    """Shape of the ``states`` tensor: the state before tokens 0, 16, 32, ... (0, 8, 16, ... for N above 32)."""
    every = 8 if N > 32 else 16
    return (T + every - 1) // every, batch, D, N


def _sequence(t, name, shape, dtype):
    """Pointer and row strides of a [T][batch][width] tensor (None: no rows)."""
    if t is None:
        return None, 0, 0
    return (t.data_ptr(), *_rows(t, name, shape, dtype))


def _reset(reset, T, B):
    if reset is not None and reset.dtype not in (torch.bool, torch.uint8):
        raise TypeError("reset must be bool or uint8")
    return _sequence(reset, "reset", (T, B), None if reset is None else reset.dtype)


def _scan_args(x, dt, A, B, C, skip, z, dt_bias, reset):
    if x.dim() != 3 or A.dim() != 2:
        raise ValueError("x must be [T][batch][D] and A [D][N]")
    T, b, D = x.shape
    N, ty = A.shape[1], x.dtype
    _want(A, "A", (D, N))
    _want(skip, "skip", (D,))
    _want(dt_bias, "dt_bias", (D,))
    rows, few = (T, b, D), (T, b, N)
    return T, b, D, N, _dt(x), (*_sequence(x, "x", rows, ty), *_sequence(dt, "dt", rows, ty), A.data_ptr(), *_sequence(B, "B", few, ty),
                                *_sequence(C, "C", few, ty), _ptr(skip), *_sequence(z, "z", rows, ty), _ptr(dt_bias)), _reset(reset, T, b)


def selective_scan(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, *, skip=None, z=None,
                   dt_bias=None, h0=None, reset=None, return_sequence=True, y=None, h_T=None, states=None,
                   workspace: torch.Tensor | None = None):
    """Selective scan: h_t = exp(d_t A) h_{t-1} + d_t x_t B_t over channels and states with d_t =
    softplus(dt_t + dt_bias), y_t = (sum_n C_t h_t + skip x_t) silu(z_t).
    x, dt, z [T][batch][D] and B, C [T][batch][N] (float32 or bfloat16, one dtype; any strides of the
    first two dimensions, so batch-first tensors go in transposed and slices of wider rows as they are),
    A [D][N] (below 0 for states that decay), skip, dt_bias [D] and h0 [batch][D][N] float32, reset
    [T][batch] bool (the token starts from a zero state).  N up to 64.  states
    (``selective_scan_states_shape``, float32) receives what ``selective_scan_backward`` needs.  h_T may
    be h0 up to 8 tokens.  Returns (y in x's dtype, h_T in float32)."""
    at = _on(x, dt, A, B, C, skip, z, dt_bias, h0, reset, y, h_T, states, workspace)
    T, b, D, N, ty, seq, marks = _scan_args(x, dt, A, B, C, skip, z, dt_bias, reset)
    dev = x.device
    _want(h0, "h0", (b, D, N))
    _want(states, "states", selective_scan_states_shape(T, b, D, N))
    if y is None and return_sequence:
        y = torch.empty((T, b, D), device=dev, dtype=x.dtype)
    if h_T is None:
        h_T = torch.empty((b, D, N), device=dev, dtype=torch.float32)
    _want(h_T, "h_T", (b, D, N))
    if workspace is None:
        workspace = _room(selective_scan_workspace_size(T, b, D, N, ty), dev)
    rc = lib().isam_selective_scan(T, b, D, N, ty, *seq, _ptr(h0), *marks, *_sequence(y, "y", (T, b, D), x.dtype), _ptr(h_T), _ptr(states),
                                   _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_selective_scan")
    return y, h_T


def selective_scan_backward(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
                            dy: torch.Tensor | None, *, states, skip=None, z=None, dt_bias=None, reset=None, dh_T=None, dx=None,
                            ddt=None, dA=None, dB=None, dC=None, dskip=None, dz=None, ddt_bias=None, dh0=None,
                            workspace: torch.Tensor | None = None):
    """Gradient of ``selective_scan``: the inputs as in, and states from, the forward call; dy [T][batch][D] in
    x's dtype or None, dh_T [batch][D][N] float32 or None.  dx, ddt, dB, dC and dz may be slices of wider
    rows.  Returns (dx, ddt, dA, dB, dC, dskip, dz, ddt_bias, dh0), rows in x's dtype and the rest in
    float32, None where the forward call had no such input (dskip, dz, ddt_bias; given ones are filled)."""
    at = _on(x, dt, A, B, C, dy, states, skip, z, dt_bias, reset, dh_T, dx, ddt, dA, dB, dC, dskip, dz, ddt_bias, dh0, workspace)
    T, b, D, N, ty, seq, marks = _scan_args(x, dt, A, B, C, skip, z, dt_bias, reset)
    dev, rows, few = x.device, (T, b, D), (T, b, N)

    def made(t, shape, dtype=torch.float32):
        return torch.empty(shape, device=dev, dtype=dtype) if t is None else t

    _want(states, "states", selective_scan_states_shape(T, b, D, N))
    _want(dh_T, "dh_T", (b, D, N))
    dx, ddt, dB, dC = made(dx, rows, x.dtype), made(ddt, rows, x.dtype), made(dB, few, x.dtype), made(dC, few, x.dtype)
    if z is not None:
        dz = made(dz, rows, x.dtype)
    if skip is not None:
        dskip = made(dskip, (D,))
    if dt_bias is not None:
        ddt_bias = made(ddt_bias, (D,))
    dA, dh0 = made(dA, (D, N)), made(dh0, (b, D, N))
    _want(dA, "dA", (D, N))
    _want(dskip, "dskip", (D,))
    _want(ddt_bias, "ddt_bias", (D,))
    _want(dh0, "dh0", (b, D, N))
    if workspace is None:
        workspace = _room(selective_scan_backward_workspace_size(T, b, D, N, ty), dev)
    rc = lib().isam_selective_scan_backward(
        T, b, D, N, ty, *seq, *marks, _ptr(states), *_sequence(dy, "dy", rows, x.dtype), _ptr(dh_T),
        *_sequence(dx, "dx", rows, x.dtype), *_sequence(ddt, "ddt", rows, x.dtype), _ptr(dA), *_sequence(dB, "dB", few, x.dtype),
        *_sequence(dC, "dC", few, x.dtype), _ptr(dskip), *_sequence(dz, "dz", rows, x.dtype), _ptr(ddt_bias), _ptr(dh0),
        _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_selective_scan_backward")
    return dx, ddt, dA, dB, dC, dskip, dz, ddt_bias, dh0


# ---------------------------------------------------------------------------------------
# Causal convolution
# ---------------------------------------------------------------------------------------
_CONV_ACTIVATIONS = {"none": _NONE, "silu": 1}


def causal_conv_backward_workspace_size(T, batch, C, K, dtype) -> int:
    return lib().isam_causal_conv_backward_workspace_size(T, batch, C, K, dtype)


def _conv_args(x, w, bias, state, reset):
    if x.dim() != 3 or w.dim() != 2 or w.shape[0] == 0:
        raise ValueError("x must be [T][batch][C] and w [K][C]")
    T, b, C = x.shape
    K = w.shape[0]
    _want(w, "w", (K, C))
    _want(bias, "bias", (C,))
    _want(state, "state", (K - 1, b, C), x.dtype)
    return T, b, C, K, _dt(x), _sequence(x, "x", (T, b, C), x.dtype), (w.data_ptr(), _ptr(bias), _ptr(state), *_reset(reset, T, b))


def causal_conv(x: torch.Tensor, w: torch.Tensor, *, bias=None, state=None, reset=None, activation="silu", return_state=True,
                y=None, state_T=None):
    """Short causal convolution over time, channels independent: y_t = act(bias + sum_k w[k] x_{t-K+1+k}).
    x [T][batch][C] (float32 or bfloat16; any strides of the first two dimensions), w [K][C] (K up to 6,
    the last row for the token itself) and bias [C] float32, state [K-1][batch][C] in x's dtype (the inputs
    before the first token; zeros without), reset [T][batch] bool (the inputs before that token count as
    zeros from it on), activation "silu" or "none".  Returns (y, state_T), state_T for the next call; it may
    be state up to 8 tokens."""
    at = _on(x, w, bias, state, reset, y, state_T)
    T, b, C, K, ty, xs, rest = _conv_args(x, w, bias, state, reset)
    act = _code(_CONV_ACTIVATIONS, activation, "activation")
    if y is None:
        y = torch.empty((T, b, C), device=x.device, dtype=x.dtype)
    if state_T is None and return_state:
        state_T = torch.empty((K - 1, b, C), device=x.device, dtype=x.dtype)
    _want(state_T, "state_T", (K - 1, b, C), x.dtype)
    rc = lib().isam_causal_conv(T, b, C, K, ty, act, *xs, *rest, *_sequence(y, "y", (T, b, C), x.dtype), _ptr(state_T), _stream(at))
    _call(rc, "isam_causal_conv")
    return y, state_T


def causal_conv_backward(x: torch.Tensor, w: torch.Tensor, dy: torch.Tensor | None, *, bias=None, state=None, reset=None,
                         activation="silu", dstate_T=None, dx=None, dstate=None, dw=None, dbias=None,
                         workspace: torch.Tensor | None = None):
    """Gradient of ``causal_conv`` from dy [T][batch][C] and dstate_T [K-1][batch][C] in x's dtype (None for
    zeros); the rest as in the forward call.  Returns (dx, dstate in x's dtype, dw, dbias in float32; dbias is
    None without a bias unless given)."""
    at = _on(x, w, dy, bias, state, reset, dstate_T, dx, dstate, dw, dbias, workspace)
    T, b, C, K, ty, xs, rest = _conv_args(x, w, bias, state, reset)
    act, dev, rows, kept = _code(_CONV_ACTIVATIONS, activation, "activation"), x.device, (T, b, C), (K - 1, b, C)
    if dx is None:
        dx = torch.empty(rows, device=dev, dtype=x.dtype)
    if dstate is None:
        dstate = torch.empty(kept, device=dev, dtype=x.dtype)
    if dw is None:
        dw = torch.empty((K, C), device=dev, dtype=torch.float32)
    if dbias is None and bias is not None:
        dbias = torch.empty((C,), device=dev, dtype=torch.float32)
    _want(dstate_T, "dstate_T", kept, x.dtype)
    _want(dstate, "dstate", kept, x.dtype)
    _want(dw, "dw", (K, C))
    _want(dbias, "dbias", (C,))
    if workspace is None:
        workspace = _room(causal_conv_backward_workspace_size(T, b, C, K, ty), dev)
    rc = lib().isam_causal_conv_backward(T, b, C, K, ty, act, *xs, *rest, *_sequence(dy, "dy", rows, x.dtype), _ptr(dstate_T),
                                         *_sequence(dx, "dx", rows, x.dtype), _ptr(dstate), _ptr(dw), _ptr(dbias), _ptr(workspace),
                                         _bytes(workspace), _stream(at))
    _call(rc, "isam_causal_conv_backward")
    return dx, dstate, dw, dbias


# ---------------------------------------------------------------------------------------
# Beam search
# ---------------------------------------------------------------------------------------
def beam_step_workspace_size(batch, beams, V, width, dtype) -> int:
    return lib().isam_beam_step_workspace_size(batch, beams, V, width, dtype)


def beam_step(logits: torch.Tensor, scores: torch.Tensor, *, width=None, finished=None, end=-1, scores_out=None, parent=None,
              token=None, finished_out=None, workspace: torch.Tensor | None = None):
    """One step of beam search: of each text's candidates scores[b][i] + log_softmax(logits[b][i])[v] the best
    `width` (beams unless given), the best first and equal ones by the lowest i * V + v.
    logits [batch][beams][V] (float32 or bfloat16; any strides of the first two dimensions), scores
    [batch][beams] float32, finished [batch][beams] bool (such a beam goes on unchanged, by the token
    `end`).  beams and width up to 64.  Returns (scores [batch][width] float32, parent (the beam) and token
    int32, finished bool)."""
    at = _on(logits, scores, finished, scores_out, parent, token, finished_out, workspace)
    if logits.dim() != 3:
        raise ValueError("logits must be [batch][beams][V]")
    b, n, V = logits.shape
    w, ty, dev = n if width is None else width, _dt(logits), logits.device
    _want(scores, "scores", (b, n))
    if finished is not None and finished.dtype not in (torch.bool, torch.uint8):
        raise TypeError("finished must be bool or uint8")
    _want(finished, "finished", (b, n), None if finished is None else finished.dtype)
    if scores_out is None:
        scores_out = torch.empty((b, w), device=dev, dtype=torch.float32)
    if parent is None:
        parent = torch.empty((b, w), device=dev, dtype=torch.int32)
    if token is None:
        token = torch.empty((b, w), device=dev, dtype=torch.int32)
    if finished_out is None:
        finished_out = torch.empty((b, w), device=dev, dtype=torch.bool)
    _want(scores_out, "scores_out", (b, w))
    _want(parent, "parent", (b, w), torch.int32)
    _want(token, "token", (b, w), torch.int32)
    _want(finished_out, "finished_out", (b, w), torch.bool)
    if workspace is None:
        workspace = _room(beam_step_workspace_size(b, n, V, w, ty), dev)
    rc = lib().isam_beam_step(b, n, V, w, ty, *_sequence(logits, "logits", (b, n, V), logits.dtype), _ptr(scores), _ptr(finished), end,
                              _ptr(scores_out), _ptr(parent), _ptr(token), _ptr(finished_out), _ptr(workspace), _bytes(workspace),
                              _stream(at))
    _call(rc, "isam_beam_step")
    return scores_out, parent, token, finished_out


def beam_reorder(state: torch.Tensor, parent: torch.Tensor, *, dim=0, out=None):
    """The rows of the beams that go on: along `dim`, of size batch * beams, row b * beams + parent[b][k] becomes row
    b * width + k.  state contiguous, of any dtype; parent [batch][width] int32 as ``beam_step`` gives it (an index
    outside leaves zeros).  Returns out (not state itself)."""
    at = _on(state, parent, out)
    if parent.dim() != 2:
        raise ValueError("parent must be [batch][width]")
    b, w = parent.shape
    _want(parent, "parent", (b, w), torch.int32)
    shape = list(state.shape)
    if not -len(shape) <= dim < len(shape):
        raise ValueError(f"state has no dimension {dim}")
    dim %= len(shape)
    if not state.is_contiguous() or w == 0 or (shape[dim] % b or shape[dim] == 0 if b else shape[dim]):
        raise ValueError("state must be contiguous, with batch * beams rows along dim")
    beams, outer, inner = shape[dim] // b if b else 1, 1, state.element_size()
    for i, n in enumerate(shape):
        if i < dim:
            outer *= n
        elif i > dim:
            inner *= n
    shape[dim] = b * w
    if out is None:
        out = torch.empty(shape, device=state.device, dtype=state.dtype)
    _want(out, "out", tuple(shape), state.dtype)
    rc = lib().isam_beam_reorder(outer, b, beams, w, inner, _ptr(state), _ptr(parent), _ptr(out), _stream(at))
    _call(rc, "isam_beam_reorder")
    return out


# ---------------------------------------------------------------------------------------
# Projection with its epilogue
# ---------------------------------------------------------------------------------------
_LINEAR_ACTIVATIONS = {**_ACTIVATIONS, "none": _NONE}


def linear_workspace_size(M, K, N, dtype, aligned=True) -> int:
    return lib().isam_linear_workspace_size(M, K, N, dtype, int(aligned))


def linear_backward_workspace_size(M, K, N, dtype, aligned=True) -> int:
    return lib().isam_linear_backward_workspace_size(M, K, N, dtype, int(aligned))


def _linear_args(x, W, bias):
    if x.dim() != 2 or W.dim() != 2 or W.shape[1] != x.shape[1]:
        raise ValueError("x must be [M][K] and W [N][K]")
    M, K = x.shape
    N = W.shape[0]
    _want(bias, "bias", (N,))
    return M, K, N, _dt(x), _matrix(x, "x", (M, K), x.dtype), _matrix(W, "W", (N, K), x.dtype)


def linear(x: torch.Tensor, W: torch.Tensor, *, bias=None, activation="none", residual=None, out=None,
           workspace: torch.Tensor | None = None):
    """Projection with its epilogue: act(x W^T + bias) + residual.  x [M][K], W [N][K], residual and out [M][N]
    (float32 or bfloat16, one dtype; row strides may exceed the row), bias [N] float32, activation "none",
    "sigmoid", "silu" or "gelu".  residual may be out.  Returns out."""
    at = _on(x, W, bias, residual, out, workspace)
    M, K, N, dt, ldx, ldw = _linear_args(x, W, bias)
    act, dev = _code(_LINEAR_ACTIVATIONS, activation, "activation"), x.device
    if out is None:
        out = torch.empty((M, N), device=dev, dtype=x.dtype)
    ldr, ldo = _matrix(residual, "residual", (M, N), x.dtype), _matrix(out, "out", (M, N), x.dtype)
    if workspace is None:
        workspace = _room(linear_workspace_size(M, K, N, dt, _aligned(x, ldx) and _aligned(W, ldw)), dev)
    rc = lib().isam_linear(M, K, N, dt, act, _ptr(x), ldx, _ptr(W), ldw, _ptr(bias), _ptr(residual), ldr, _ptr(out), ldo, _ptr(workspace),
                           _bytes(workspace), _stream(at))
    _call(rc, "isam_linear")
    return out


def linear_backward(x: torch.Tensor, W: torch.Tensor, dout: torch.Tensor, *, bias=None, activation="none", return_dx=True,
                    return_dW=True, dx=None, dW=None, dbias=None, workspace: torch.Tensor | None = None):
    """Gradient of ``linear`` from dout [M][N] (which is also the residual's).  Returns (dx [M][K], dW [N][K] in x's
    dtype, dbias [N] float32 or None without a bias); with an activation the product is formed again, nothing is
    kept from the forward call (bfloat16 beyond 16 rows: its gradient is rounded as the products' operand, so dx and dW carry
    two roundings).  return_dx or return_dW False: that product is left out, and None stands for it.  N = 0: dx
    is zeros."""
    at = _on(x, W, dout, bias, dx, dW, dbias, workspace)
    M, K, N, dt, ldx, ldw = _linear_args(x, W, bias)
    act, dev = _code(_LINEAR_ACTIVATIONS, activation, "activation"), x.device
    if dx is None and return_dx:
        dx = torch.empty((M, K), device=dev, dtype=x.dtype)
    if dW is None and return_dW:
        dW = torch.empty((N, K), device=dev, dtype=x.dtype)
    if dbias is None and bias is not None:
        dbias = torch.empty((N,), device=dev, dtype=torch.float32)
    _want(dbias, "dbias", (N,))
    lddo, lddx, lddw = _matrix(dout, "dout", (M, N), x.dtype), _matrix(dx, "dx", (M, K), x.dtype), _matrix(dW, "dW", (N, K), x.dtype)
    if N == 0:  # (a sum of nothing; the C entry takes no dx then)
        if dx is not None:
            dx.zero_()
        return dx, dW, dbias
    if workspace is None:
        workspace = _room(linear_backward_workspace_size(M, K, N, dt, _aligned(x, ldx) and _aligned(W, ldw) and _aligned(dout, lddo)), dev)
    rc = lib().isam_linear_backward(M, K, N, dt, act, _ptr(x), ldx, _ptr(W), ldw, _ptr(bias), _ptr(dout), lddo, _ptr(dx), lddx, _ptr(dW),
                                    lddw, _ptr(dbias), _ptr(workspace), _bytes(workspace), _stream(at))
    _call(rc, "isam_linear_backward")
    return dx, dW, dbias
