"""Python binding of the operators around the aggregation (``include/mp_layers.h``): group norm with
an activation, dropout, the softmax router and microscaled 4-bit floating point.

As in the package's root, ``mp_*`` functions carry the names of the C ABI and take tensors or None for
pointers; the others size and allocate outputs and workspaces with torch.  The root re-exports all of
them.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math

import torch

from . import (MP_F32, _bytes, _check, _dtype_code, _itype_code, _ptr, _rows_ptr, _stream, _workspace,
               lib as _root_lib)

__all__ = ["MP_ACT", "mp_group_norm_workspace", "mp_group_norm", "mp_group_norm_backward",
           "group_norm", "group_norm_backward", "mp_dropout", "dropout", "dropout_backward", "mp_route_workspace", "mp_route",
           "mp_route_backward", "route", "route_backward", "mp_mx_quantize", "mp_mx_dequantize",
           "mp_mx_segment_matmul_workspace", "mp_mx_segment_matmul", "mx_quantize", "mx_dequantize",
           "mx_segment_matmul"]

MP_ACT = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

_lib = None


def _layers():
    """The library with this header's functions declared."""
    global _lib
    if _lib is None:
        L = _root_lib()
        i32, i64, p, u64 = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_uint64
        L.mp_dropout.argtypes = [p, i32, i64, i64, i64, p, i64, p, i32, ctypes.c_double, u64, u64, p,
                                 p, i64, p]
        psz, sz, f32 = ctypes.POINTER(ctypes.c_size_t), ctypes.c_size_t, ctypes.c_float
        L.mp_group_norm_workspace.argtypes = [i64, i64, i64, i64, i32, i32, psz]
        L.mp_group_norm.argtypes = [p, i32, p, i32, i64, i64, i64, i64, i64, p, p, f32, i32, p, i32,
                                    p, p, p, sz, p]
        L.mp_group_norm_backward.argtypes = [p, i32, p, i32, p, i64, i64, i64, i64, i64, p, p, p, p,
                                             i32, p, i32, p, p, p, sz, p]
        L.mp_route_workspace.argtypes = [i64, i64, psz]
        L.mp_route.argtypes = [p, i32, i64, i64, i64, i64, p, i32, p, p, p, p, p, sz, p]
        L.mp_route_backward.argtypes = [p, i32, i64, i64, i64, i64, p, i32, p, p, p, p, p, p, p]
        L.mp_mx_quantize.argtypes = [p, i32, i64, i64, i64, p, p, p, p]
        L.mp_mx_dequantize.argtypes = [p, p, i64, i64, p, i32, p]
        L.mp_mx_segment_matmul_workspace.argtypes = [i64, i64, i64, i64, psz]
        L.mp_mx_segment_matmul.argtypes = [p, i32, i64, p, i32, i64, i64, i64, p, p, i64, p, i32, p, sz,
                                           p]
        for name in ("mp_mx_quantize", "mp_mx_dequantize", "mp_mx_segment_matmul_workspace",
                     "mp_mx_segment_matmul", "mp_group_norm_workspace", "mp_group_norm", "mp_group_norm_backward",
                     "mp_dropout", "mp_route_workspace", "mp_route", "mp_route_backward"):
            getattr(L, name).restype = i32
        _lib = L
    return _lib


_NO_CONTEXT = contextlib.nullcontext()


def _on(stream):
    """What the wrappers allocate and free while they enqueue on `stream` belongs to that stream, so
    that memory is not given away while its kernels run."""
    if stream is None:
        return _NO_CONTEXT
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream))
    return torch.cuda.stream(stream)


def _on_gpu(*tensors):
    """Kernels run on the current GPU: an operand elsewhere is refused."""
    for t in tensors:
        if t is not None and (not t.is_cuda or t.get_device() != torch.cuda.current_device()):
            raise ValueError(f"operands must be on the current GPU, got one on {t.device}")


@functools.lru_cache(maxsize=4096)
def _sized(query, *sizes):
    """Workspace bytes, a function of the sizes alone."""
    return query(*sizes)


def _table(t):
    """_rows_ptr, also for one value a row ([N] as a table of one column)."""
    return _rows_ptr(t[:, None] if t.dim() == 1 else t)


def _like(t, ref, name):
    if t is not None and (t.shape != ref.shape or t.dtype != ref.dtype):
        raise ValueError(f"{name} must have the shape and dtype of x")
    return t


def _vector(t, n, dtype, name):
    """Checks a small contiguous operand of n values."""
    if t is not None and (t.numel() != n or t.dtype != dtype):
        raise ValueError(f"{name} must hold {n} values of {dtype}")
    return t


# ---- group norm ---------------------------------------------------------------------------

def mp_group_norm_workspace(N, S, F, G, x_dtype, backward) -> int:
    _layers()
    return _bytes("mp_group_norm_workspace", N, S, F, G, x_dtype, int(backward))


def mp_group_norm(ptr, ptr_itype, x, x_dtype, N, S, F, ldx, G, gamma, beta, eps, act, out, out_dtype,
                  mean, rstd, ws, ws_bytes, stream=None):
    """x: a tensor (rows may be strided) or a raw address."""
    xp = _rows_ptr(x)[0] if isinstance(x, torch.Tensor) else x
    _check("mp_group_norm", _layers().mp_group_norm(
        _ptr(ptr), ptr_itype, xp, x_dtype, N, S, F, ldx, G, _ptr(gamma), _ptr(beta), eps, act,
        _ptr(out), out_dtype, _ptr(mean), _ptr(rstd), _ptr(ws), ws_bytes, _stream(stream)))


def mp_group_norm_backward(ptr, ptr_itype, x, x_dtype, dout, N, S, F, ldx, G, gamma, beta, mean, rstd,
                           act, dx, dx_dtype, dgamma, dbeta, ws, ws_bytes, stream=None):
    xp = _rows_ptr(x)[0] if isinstance(x, torch.Tensor) else x
    _check("mp_group_norm_backward", _layers().mp_group_norm_backward(
        _ptr(ptr), ptr_itype, xp, x_dtype, _ptr(dout), N, S, F, ldx, G, _ptr(gamma), _ptr(beta),
        _ptr(mean), _ptr(rstd), act, _ptr(dx), dx_dtype, _ptr(dgamma), _ptr(dbeta), _ptr(ws),
        ws_bytes, _stream(stream)))


def _act(act):
    if act not in MP_ACT:
        raise ValueError(f"act must be one of {', '.join(MP_ACT)}")
    return MP_ACT[act]


def group_norm(ptr, x, groups, *, weight=None, bias=None, eps=1e-5, act="none", out_dtype=None,
               out=None, stream=None):
    """act(group norm of x [N, F]) over the segments of consecutive rows that ptr [S + 1] gives (the
    graphs of a batch) and `groups` groups of consecutive channels; weight and bias [F] fp32.

    Returns (out [N, F] of out_dtype (default x's), mean [S, groups], rstd [S, groups]); the latter two
    go to group_norm_backward."""
    N, F = int(x.shape[0]), int(x.shape[1])
    S, G = int(ptr.numel()) - 1, int(groups)
    a = _act(act)
    _vector(weight, F, torch.float32, "weight")
    _vector(bias, F, torch.float32, "bias")
    if out is not None and out.shape != x.shape:
        raise ValueError("out must have the shape of x")
    _on_gpu(ptr, x, weight, bias, out)
    dt, it = _dtype_code(x.dtype), _itype_code(ptr.dtype)
    xp, ldx = _rows_ptr(x)
    nb = _sized(mp_group_norm_workspace, N, S, F, G, dt, 0)
    dev = x.device
    with _on(stream):
        if out is None:
            out = torch.empty(N, F, dtype=out_dtype or x.dtype, device=dev)
        mean = torch.empty(S, G, dtype=torch.float32, device=dev)
        rstd = torch.empty(S, G, dtype=torch.float32, device=dev)
        ws = _workspace(nb, dev) if nb else None
        mp_group_norm(ptr, it, xp, dt, N, S, F, ldx, G, weight, bias, eps, a, out,
                      _dtype_code(out.dtype), mean, rstd, ws, nb, stream)
    return out, mean, rstd


def group_norm_backward(ptr, x, dout, groups, mean, rstd, *, weight=None, bias=None, act="none",
                        dx_dtype=None, want_dx=True, want_dw=True, stream=None):
    """Gradients of group_norm given dout [N, F] (dtype of x): (dx [N, F] of dx_dtype (default x's) or
    None, dweight [F] fp32 or None, dbias [F] fp32 or None)."""
    N, F = int(x.shape[0]), int(x.shape[1])
    S, G = int(ptr.numel()) - 1, int(groups)
    a = _act(act)
    _like(dout, x, "dout")
    _vector(mean, S * G, torch.float32, "mean")
    _vector(rstd, S * G, torch.float32, "rstd")
    _vector(weight, F, torch.float32, "weight")
    _vector(bias, F, torch.float32, "bias")
    _on_gpu(ptr, x, dout, mean, rstd, weight, bias)
    dt, it = _dtype_code(x.dtype), _itype_code(ptr.dtype)
    xp, ldx = _rows_ptr(x)
    nb = _sized(mp_group_norm_workspace, N, S, F, G, dt, 1)
    dev = x.device
    with _on(stream):
        dx = torch.empty(N, F, dtype=dx_dtype or x.dtype, device=dev) if want_dx else None
        dw = torch.empty(F, dtype=torch.float32, device=dev) if want_dw else None
        db = torch.empty(F, dtype=torch.float32, device=dev) if want_dw else None
        ws = _workspace(nb, dev) if nb else None
        mp_group_norm_backward(ptr, it, xp, dt, dout, N, S, F, ldx, G, weight, bias, mean, rstd, a, dx,
                               _dtype_code(dx.dtype) if want_dx else MP_F32, dw, db, ws, nb, stream)
    return dx, dw, db


# ---- dropout ------------------------------------------------------------------------------

def mp_dropout(x, dtype, N, F, ldx, residual, ldr, ids, whole_rows, p, seed, offset, step, out, ldo,
               stream=None):
    """x, residual and out: tensors (rows may be strided) or raw addresses."""
    xp, rp, op = (_table(t)[0] if isinstance(t, torch.Tensor) else t for t in (x, residual, out))
    _check("mp_dropout", _layers().mp_dropout(
        xp, dtype, N, F, ldx, rp, ldr, _ptr(ids), whole_rows, p, seed, offset, _ptr(step), op, ldo,
        _stream(stream)))


def dropout(x, p, seed, *, offset=0, step=None, ids=None, rows=False, residual=None, out=None,
            stream=None):
    """x [N, F] or [N] with each element (rows: each row) dropped with probability p and the others
    scaled by 1 / (1 - p), plus residual.

    The mask is a function of seed, offset + step (step: an int64 tensor on the device) and the
    element's number ids[r] * F + f (ids: int32 [N], default r; rows: ids[r]), and is stored nowhere:
    dropout_backward draws it again."""
    N, F = int(x.shape[0]), int(x.shape[1]) if x.dim() == 2 else 1
    _like(residual, x, "residual")
    _vector(ids, N, torch.int32, "ids")
    _vector(step, 1, torch.int64, "step")
    _like(out, x, "out")
    _on_gpu(x, residual, ids, step, out)
    if out is None:
        with _on(stream):
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    xp, ldx = _table(x)
    rp, ldr = _table(residual) if residual is not None else (None, F)
    op, ldo = _table(out)
    mp_dropout(xp, _dtype_code(x.dtype), N, F, ldx, rp, ldr, ids, int(rows), p, seed, offset, step, op,
               ldo, stream)
    return out


def dropout_backward(dout, p, seed, *, offset=0, step=None, ids=None, rows=False, out=None,
                     stream=None):
    """dL/dx of dropout given dL/dout: the same mask and scale (the residual's gradient is dout)."""
    return dropout(dout, p, seed, offset=offset, step=step, ids=ids, rows=rows, out=out, stream=stream)


# ---- router -------------------------------------------------------------------------------

def mp_route_workspace(N, E) -> int:
    _layers()
    return _bytes("mp_route_workspace", N, E)


def mp_route(logits, dtype, N, E, ldl, k, mask, renorm, idx, weight, counts, loss, ws, ws_bytes,
             stream=None):
    """logits: a tensor (rows may be strided) or a raw address."""
    lp = _rows_ptr(logits)[0] if isinstance(logits, torch.Tensor) else logits
    _check("mp_route", _layers().mp_route(
        lp, dtype, N, E, ldl, k, _ptr(mask), renorm, _ptr(idx), _ptr(weight), _ptr(counts),
        _ptr(loss), _ptr(ws), ws_bytes, _stream(stream)))


def mp_route_backward(logits, dtype, N, E, ldl, k, mask, renorm, idx, weight, counts, dweight, dloss,
                      dlogits, stream=None):
    lp = _rows_ptr(logits)[0] if isinstance(logits, torch.Tensor) else logits
    _check("mp_route_backward", _layers().mp_route_backward(
        lp, dtype, N, E, ldl, k, _ptr(mask), renorm, _ptr(idx), _ptr(weight), _ptr(counts),
        _ptr(dweight), _ptr(dloss), _ptr(dlogits), _stream(stream)))


def _mask(mask, N):
    if mask is None:
        return None
    if mask.numel() != N or mask.dtype not in (torch.bool, torch.uint8):
        raise ValueError(f"mask must hold {N} truth values")
    return mask


def route(logits, k, *, mask=None, renorm=True, stream=None):
    """The k experts of every row of logits [N, E] and what the batch makes of them:
    (idx [N, k] int32, weight [N, k] fp32, counts [E + 1] int32: choices of each expert and the rows
    that took part, loss [2] fp32: balance and z).

    Rows whose mask ([N] bool) is false, or whose logits are all -inf, take no part: idx -1, weight 0.
    renorm: the weights of a row add up to 1 (else they are softmax probabilities over all experts)."""
    N, E = int(logits.shape[0]), int(logits.shape[1])
    k = int(k)
    _mask(mask, N)
    _on_gpu(logits, mask)
    dev = logits.device
    dt = _dtype_code(logits.dtype)
    lp, ldl = _rows_ptr(logits)
    nb = _sized(mp_route_workspace, N, E)
    with _on(stream):
        idx = torch.empty(N, max(k, 0), dtype=torch.int32, device=dev)
        weight = torch.empty(N, max(k, 0), dtype=torch.float32, device=dev)
        counts = torch.empty(E + 1, dtype=torch.int32, device=dev)
        loss = torch.empty(2, dtype=torch.float32, device=dev)
        ws = _workspace(nb, dev) if nb else None
        mp_route(lp, dt, N, E, ldl, k, mask, int(renorm), idx, weight, counts, loss, ws, nb, stream)
    return idx, weight, counts, loss


def route_backward(logits, idx, weight, counts, *, dweight=None, dloss=None, mask=None, renorm=True,
                   out=None, stream=None):
    """dL/dlogits [N, E] (dtype of logits) given dweight = dL/dweight [N, k] fp32 and dloss = dL/dloss
    [2] fp32 on the GPU (None: 0), and what route returned."""
    N, E = int(logits.shape[0]), int(logits.shape[1])
    k = int(idx.shape[1])
    _mask(mask, N)
    _vector(idx, N * k, torch.int32, "idx")
    _vector(weight, N * k, torch.float32, "weight")
    _vector(counts, E + 1, torch.int32, "counts")
    _vector(dweight, N * k, torch.float32, "dweight")
    _vector(dloss, 2, torch.float32, "dloss")
    _like(out, logits, "out")
    _on_gpu(logits, idx, weight, counts, dweight, dloss, mask, out)
    lp, ldl = _rows_ptr(logits)
    if out is None:
        with _on(stream):
            out = torch.empty(N, E, dtype=logits.dtype, device=logits.device)
    mp_route_backward(lp, _dtype_code(logits.dtype), N, E, ldl, k, mask, int(renorm), idx, weight,
                      counts, dweight, dloss, out, stream)
    return out


# ---- microscaled 4-bit floating point --------------------------------------------------------

def mp_mx_quantize(x, dtype, N, K, ldx, codes, scales, values, stream=None):
    """x: a tensor (rows may be strided) or a raw address."""
    xp = _rows_ptr(x)[0] if isinstance(x, torch.Tensor) else x
    _check("mp_mx_quantize", _layers().mp_mx_quantize(
        xp, dtype, N, K, ldx, _ptr(codes), _ptr(scales), _ptr(values), _stream(stream)))


def mp_mx_dequantize(codes, scales, N, K, out, dtype, stream=None):
    _check("mp_mx_dequantize", _layers().mp_mx_dequantize(
        _ptr(codes), _ptr(scales), N, K, _ptr(out), dtype, _stream(stream)))


def mp_mx_segment_matmul_workspace(T, N, K, Fo) -> int:
    _layers()
    return _bytes("mp_mx_segment_matmul_workspace", T, N, K, Fo)


def mp_mx_segment_matmul(seg, seg_itype, T, x, x_dtype, N, K, ldx, w_codes, w_scales, Fo, out,
                         out_dtype, ws, ws_bytes, stream=None):
    xp = _rows_ptr(x)[0] if isinstance(x, torch.Tensor) else x
    _check("mp_mx_segment_matmul", _layers().mp_mx_segment_matmul(
        _ptr(seg), seg_itype, T, xp, x_dtype, N, K, ldx, _ptr(w_codes), _ptr(w_scales), Fo, _ptr(out),
        out_dtype, _ptr(ws), ws_bytes, _stream(stream)))


def _blocks(K):
    return -(-int(K) // 32)


def mx_quantize(x, *, want_values=False, stream=None):
    """x [..., K] in 4 bits: (codes [..., 16 KB] uint8, scales [..., KB] uint8), KB = ceil(K / 32), and
    with want_values also the values that they stand for, in x's shape and dtype (training with
    quantised values: use them in the forward pass and hand their gradient to x unchanged).

    The weights of mx_segment_matmul are mx_quantize(W.transpose(1, 2)) of segment_matmul's W; one type's
    may come as a table, W.t().  Views of other strides than a table's are copied."""
    K = int(x.shape[-1])
    _on_gpu(x)
    lead, kb = tuple(x.shape[:-1]), _blocks(K)
    with _on(stream):
        # (of a table the rows may be strided; other views are made contiguous, by and for the stream)
        table = x.dim() == 2 and x.stride(1) == 1 and x.stride(0) >= K
        rows = x if table else x.contiguous().view(math.prod(lead), K)
        N = int(rows.shape[0])
        xp, ldx = _rows_ptr(rows)
        codes = torch.empty(*lead, 16 * kb, dtype=torch.uint8, device=x.device)
        scales = torch.empty(*lead, kb, dtype=torch.uint8, device=x.device)
        values = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_values else None
        mp_mx_quantize(xp, _dtype_code(x.dtype), N, K, ldx, codes, scales, values, stream)
    return (codes, scales, values) if want_values else (codes, scales)


def _mx(codes, scales, K):
    kb = _blocks(K)
    if (codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.shape[-1] != 16 * kb
            or scales.shape[-1] != kb or codes.shape[:-1] != scales.shape[:-1]):
        raise ValueError(f"codes [..., {16 * kb}] and scales [..., {kb}] of uint8 expected for K = {K}")


def mx_dequantize(codes, scales, K, *, dtype=torch.float32, stream=None):
    """The values [..., K] that codes and scales stand for."""
    _mx(codes, scales, K)
    _on_gpu(codes, scales)
    lead = tuple(codes.shape[:-1])
    kb = _blocks(K)
    with _on(stream):
        out = torch.empty(*lead, int(K), dtype=dtype, device=codes.device)
        mp_mx_dequantize(codes, scales, scales.numel() // kb, int(K), out, _dtype_code(dtype), stream)
    return out


def mx_segment_matmul(seg, x, codes, scales, *, out_dtype=torch.float32, out=None, stream=None):
    """out[r] = q(x[r]) @ W[t]^T for the rows r of segment t: x [N, K] is quantised on the way, W is
    given in 4 bits as codes [T, Fo, 16 KB] and scales [T, Fo, KB] (mx_quantize of [T, Fo, K]).

    seg [T + 1] (int32 or int64) lies on the GPU, as the rowptr of a dispatch does; rows of no segment
    are not written."""
    N, K = int(x.shape[0]), int(x.shape[1])
    _mx(codes, scales, K)
    if codes.dim() != 3 or int(seg.numel()) != codes.shape[0] + 1:
        raise ValueError("codes [T, Fo, ...] and seg [T + 1] expected")
    T, Fo = int(codes.shape[0]), int(codes.shape[1])
    if out is not None and tuple(out.shape) != (N, Fo):
        raise ValueError("out must be [N, Fo]")
    _on_gpu(seg, x, codes, scales, out)
    dt, it = _dtype_code(x.dtype), _itype_code(seg.dtype)
    xp, ldx = _rows_ptr(x)
    nb = _sized(mp_mx_segment_matmul_workspace, T, N, K, Fo)
    with _on(stream):
        if out is None:
            out = torch.empty(N, Fo, dtype=out_dtype, device=x.device)
        ws = _workspace(nb, x.device)
        mp_mx_segment_matmul(seg, it, T, xp, dt, N, K, ldx, codes, scales, Fo, out,
                             _dtype_code(out.dtype), ws, nb, stream)
    return out
