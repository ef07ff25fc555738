"""Python binding of the operators around the aggregation (``include/mp_layers.h``): group norm with
an activation, dropout, the softmax router, microscaled 4-bit floating point, embeddings,
root-mean-square norm and the experts of few rows.

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
           "mx_segment_matmul", "mp_embed", "mp_embed_backward_workspace", "mp_embed_backward", "embed",
           "embed_backward", "mp_rms_norm", "mp_rms_norm_mx8", "mp_rms_norm_backward_workspace",
           "mp_rms_norm_backward", "mp_mx8_dequantize", "rms_norm", "rms_norm_mx8", "rms_norm_backward",
           "mx8_dequantize", "mp_expert_mlp_workspace", "mp_expert_mlp", "expert_mlp"]

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
        L.mp_embed.argtypes = [p, i32, i64, p, i32, i64, i64, i64, i64, f32, p, i32, p]
        L.mp_embed_backward_workspace.argtypes = [i64, i64, i64, psz]
        L.mp_embed_backward.argtypes = [p, i32, i64, p, i32, i64, i64, i64, i64, f32, p, i32, p, sz, p]
        L.mp_rms_norm.argtypes = [p, i32, i64, i64, i64, p, i64, p, f32, p, p, i32, p, p]
        L.mp_rms_norm_mx8.argtypes = [p, i32, i64, i64, i64, p, i64, p, f32, p, p, p, p, p, p]
        L.mp_mx8_dequantize.argtypes = [p, p, i64, i64, p, i32, p]
        L.mp_rms_norm_backward_workspace.argtypes = [i64, i64, i32, psz]
        L.mp_rms_norm_backward.argtypes = [p, i32, i64, i64, i64, p, p, p, p, p, i32, p, p, sz, p]
        L.mp_expert_mlp_workspace.argtypes = [i64, i64, i64, i64, i64, i32, psz]
        L.mp_expert_mlp.argtypes = [p, i32, p, i64, i64, i64, p, p, i64, i64, i64, i64, p, p, p, p, i32, i32,
                                    p, i64, p, i32, p, sz, p]
        for name in ("mp_expert_mlp_workspace", "mp_expert_mlp", "mp_embed", "mp_embed_backward_workspace", "mp_embed_backward", "mp_rms_norm",
                     "mp_rms_norm_mx8", "mp_mx8_dequantize", "mp_rms_norm_backward_workspace",
                     "mp_rms_norm_backward", "mp_mx_quantize", "mp_mx_dequantize", "mp_mx_segment_matmul_workspace",
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
    here = -1
    for t in tensors:
        if t is None:
            continue
        at = t.get_device()  # (-1: not on a GPU)
        if here < 0 <= at:
            here = torch.cuda.current_device()
        if at < 0 or at != here:
            raise ValueError(f"operands must be on the current GPU, got one on {t.device}")


@functools.lru_cache(maxsize=4096)
def _sized(query, *sizes):
    """Workspace bytes, a function of the sizes alone."""
    return query(*sizes)


def _table(t):
    """_rows_ptr, also for one value a row ([N] as a table of one column)."""
    return _rows_ptr(t[:, None] if t.dim() == 1 else t)


def _rows(t):
    """Address of a table whose rows may be strided; what is no tensor is an address."""
    return _rows_ptr(t)[0] if isinstance(t, torch.Tensor) else t


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


# ---- embeddings ------------------------------------------------------------------------------

def mp_embed(ids, ids_itype, N, table, dtype, V, F, ldt, padding, scale, out, out_dtype, stream=None):
    """table: a tensor (rows may be strided) or a raw address."""
    tp = _rows_ptr(table)[0] if isinstance(table, torch.Tensor) else table
    _check("mp_embed", _layers().mp_embed(
        _ptr(ids), ids_itype, N, tp, dtype, V, F, ldt, padding, scale, _ptr(out), out_dtype,
        _stream(stream)))


def mp_embed_backward_workspace(N, V, F) -> int:
    _layers()
    return _bytes("mp_embed_backward_workspace", N, V, F)


def mp_embed_backward(ids, ids_itype, N, dout, dtype, V, F, ldd, padding, scale, dtable, dtable_dtype,
                      ws, ws_bytes, stream=None):
    """dout: a tensor (rows may be strided) or a raw address."""
    dp = _rows_ptr(dout)[0] if isinstance(dout, torch.Tensor) else dout
    _check("mp_embed_backward", _layers().mp_embed_backward(
        _ptr(ids), ids_itype, N, dp, dtype, V, F, ldd, padding, scale, _ptr(dtable), dtable_dtype,
        _ptr(ws), ws_bytes, _stream(stream)))


def _padding(padding):
    if padding is not None and padding < 0:
        raise ValueError("padding must be an id of the table (ids outside it are padding anyway)")
    return -1 if padding is None else int(padding)


def embed(ids, table, *, scale=1.0, padding=None, out_dtype=None, out=None, stream=None):
    """scale * table[ids], [N, F] of out_dtype (default the table's): ids [N] int32 or int64, table
    [V, F].  Ids outside [0, V), and the id `padding`, give rows of zeros."""
    V, F = int(table.shape[0]), int(table.shape[1])
    if ids.dim() != 1:
        raise ValueError("ids [N] expected")
    N = int(ids.shape[0])
    if out is not None and tuple(out.shape) != (N, F):
        raise ValueError("out must be [N, F]")
    pad = _padding(padding)
    _on_gpu(ids, table, out)
    dt, it = _dtype_code(table.dtype), _itype_code(ids.dtype)
    tp, ldt = _rows_ptr(table)
    if out is None:
        with _on(stream):
            out = torch.empty(N, F, dtype=out_dtype or table.dtype, device=table.device)
    mp_embed(ids, it, N, tp, dt, V, F, ldt, pad, scale, out, _dtype_code(out.dtype), stream)
    return out


def embed_backward(ids, dout, V, *, scale=1.0, padding=None, out_dtype=None, out=None, stream=None):
    """dL/dtable [V, F] of out_dtype (default dout's) of embed given dout = dL/dout [N, F], in full: 0 for
    ids of no row.  Sums are in fp32 and in a fixed order (ids and sizes alone set it), so the same bits
    every time."""
    V, N, F = int(V), int(dout.shape[0]), int(dout.shape[1])
    if ids.dim() != 1 or int(ids.shape[0]) != N:
        raise ValueError("ids [N] and dout [N, F] expected")
    if out is not None and tuple(out.shape) != (V, F):
        raise ValueError("out must be [V, F]")
    pad = _padding(padding)
    _on_gpu(ids, dout, out)
    dt, it = _dtype_code(dout.dtype), _itype_code(ids.dtype)
    dp, ldd = _rows_ptr(dout)
    nb = _sized(mp_embed_backward_workspace, N, V, F)
    with _on(stream):
        if out is None:
            out = torch.empty(V, F, dtype=out_dtype or dout.dtype, device=dout.device)
        ws = _workspace(nb, dout.device)
        mp_embed_backward(ids, it, N, dp, dt, V, F, ldd, pad, scale, out, _dtype_code(out.dtype), ws, nb,
                          stream)
    return out


# ---- root-mean-square norm ---------------------------------------------------------------------

def mp_rms_norm(x, dtype, N, F, ldx, residual, ldr, weight, eps, total, out, out_dtype, rstd,
                stream=None):
    """x and residual: tensors (rows may be strided) or raw addresses."""
    _check("mp_rms_norm", _layers().mp_rms_norm(
        _rows(x), dtype, N, F, ldx, _rows(residual), ldr, _ptr(weight), eps, _ptr(total), _ptr(out),
        out_dtype, _ptr(rstd), _stream(stream)))


def mp_rms_norm_mx8(x, dtype, N, F, ldx, residual, ldr, weight, eps, total, codes, scales, values, rstd,
                    stream=None):
    _check("mp_rms_norm_mx8", _layers().mp_rms_norm_mx8(
        _rows(x), dtype, N, F, ldx, _rows(residual), ldr, _ptr(weight), eps, _ptr(total), _ptr(codes),
        _ptr(scales), _ptr(values), _ptr(rstd), _stream(stream)))


def mp_mx8_dequantize(codes, scales, N, K, out, dtype, stream=None):
    _check("mp_mx8_dequantize", _layers().mp_mx8_dequantize(
        _ptr(codes), _ptr(scales), N, K, _ptr(out), dtype, _stream(stream)))


def mp_rms_norm_backward_workspace(N, F, dtype) -> int:
    _layers()
    return _bytes("mp_rms_norm_backward_workspace", N, F, dtype)


def mp_rms_norm_backward(total, dtype, N, F, ldt, dout, rstd, weight, dtotal, dx, dx_dtype, dweight, ws,
                         ws_bytes, stream=None):
    tp = _rows_ptr(total)[0] if isinstance(total, torch.Tensor) else total
    _check("mp_rms_norm_backward", _layers().mp_rms_norm_backward(
        tp, dtype, N, F, ldt, _ptr(dout), _ptr(rstd), _ptr(weight), _ptr(dtotal), _ptr(dx), dx_dtype,
        _ptr(dweight), _ptr(ws), ws_bytes, _stream(stream)))


def _rms_operands(x, weight, residual, total):
    N, F = int(x.shape[0]), int(x.shape[1])
    _vector(weight, F, torch.float32, "weight")
    _like(residual, x, "residual")
    _like(total, x, "total")
    _on_gpu(x, weight, residual, total)
    xp, ldx = _rows_ptr(x)
    rp, ldr = _rows_ptr(residual) if residual is not None else (None, F)
    return N, F, _dtype_code(x.dtype), xp, ldx, rp, ldr


def rms_norm(x, weight=None, *, residual=None, eps=1e-5, out_dtype=None, out=None, total=None,
             stream=None):
    """Root-mean-square norm of the rows of x [N, F], or of x + residual: (out [N, F] of out_dtype
    (default x's), total [N, F]: the sum as it is stored (x itself without a residual), rstd [N] fp32);
    the latter two go to rms_norm_backward.  weight [F] fp32.  total may be given, as x or residual
    itself to be overwritten."""
    N, F, dt, xp, ldx, rp, ldr = _rms_operands(x, weight, residual, total)
    if out is not None and out.shape != x.shape:
        raise ValueError("out must have the shape of x")
    _on_gpu(out)
    dev = x.device
    with _on(stream):
        if out is None:
            out = torch.empty(N, F, dtype=out_dtype or x.dtype, device=dev)
        rstd = torch.empty(N, dtype=torch.float32, device=dev)
        if residual is not None and total is None:
            total = torch.empty_like(x)
        mp_rms_norm(xp, dt, N, F, ldx, rp, ldr, weight, eps, total, out, _dtype_code(out.dtype), rstd,
                    stream)
    return out, x if total is None else total, rstd


def rms_norm_mx8(x, weight=None, *, residual=None, eps=1e-5, want_values=False, total=None, stream=None):
    """rms_norm in microscaled 8 bits: (codes [N, 32 KB] uint8, scales [N, KB] uint8, values, total),
    KB = ceil(F / 32).  values: what they stand for, [N, F] of x's dtype, or None without want_values;
    total as rms_norm's.  (codes, scales) are rows of expert_mlp.  The gradient is rms_norm_backward's, with
    the rstd that rms_norm gives of the same rows (mp_rms_norm_mx8 writes it too)."""
    N, F, dt, xp, ldx, rp, ldr = _rms_operands(x, weight, residual, total)
    dev, kb = x.device, _blocks(F)
    with _on(stream):
        codes = torch.empty(N, 32 * kb, dtype=torch.uint8, device=dev)
        scales = torch.empty(N, kb, dtype=torch.uint8, device=dev)
        values = torch.empty_like(x) if want_values else None
        if residual is not None and total is None:
            total = torch.empty_like(x)
        mp_rms_norm_mx8(xp, dt, N, F, ldx, rp, ldr, weight, eps, total, codes, scales, values, None,
                        stream)
    return codes, scales, values, x if total is None else total


def _mx8(codes, scales, K):
    kb = _blocks(K)
    if (codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2
            or codes.shape[1] != 32 * kb or tuple(scales.shape) != (codes.shape[0], kb)):
        raise ValueError(f"codes [N, {32 * kb}] and scales [N, {kb}] of uint8 expected for K = {K}")


def mx8_dequantize(codes, scales, K, *, dtype=torch.float32, stream=None):
    """The values [N, K] that 8-bit codes and scales stand for."""
    _mx8(codes, scales, K)
    _on_gpu(codes, scales)
    with _on(stream):
        out = torch.empty(codes.shape[0], int(K), dtype=dtype, device=codes.device)
        mp_mx8_dequantize(codes, scales, int(codes.shape[0]), int(K), out, _dtype_code(dtype), stream)
    return out


def rms_norm_backward(total, dout, rstd, weight=None, *, dtotal=None, dx_dtype=None, want_dx=True,
                      want_dw=True, stream=None):
    """Gradients of rms_norm given dout [N, F] (dtype of x), its total and rstd, and dtotal (the gradient
    that reaches total by itself): (dx [N, F] of dx_dtype (default x's), of x and of residual alike, or
    None; dweight [F] fp32 or None)."""
    N, F = int(total.shape[0]), int(total.shape[1])
    _like(dout, total, "dout")
    _like(dtotal, total, "dtotal")
    _vector(rstd, N, torch.float32, "rstd")
    _vector(weight, F, torch.float32, "weight")
    _on_gpu(total, dout, rstd, weight, dtotal)
    dt = _dtype_code(total.dtype)
    tp, ldt = _rows_ptr(total)
    nb = _sized(mp_rms_norm_backward_workspace, N, F, dt) if want_dw else 0
    dev = total.device
    with _on(stream):
        dx = torch.empty(N, F, dtype=dx_dtype or total.dtype, device=dev) if want_dx else None
        dw = torch.empty(F, dtype=torch.float32, device=dev) if want_dw else None
        ws = _workspace(nb, dev) if nb else None
        mp_rms_norm_backward(tp, dt, N, F, ldt, dout, rstd, weight, dtotal, dx,
                             _dtype_code(dx.dtype) if want_dx else MP_F32, dw, ws, nb, stream)
    return dx, dw


# ---- the experts of few rows ---------------------------------------------------------------------

def mp_expert_mlp_workspace(N, k, E, H, Fo, out_dtype) -> int:
    _layers()
    return _bytes("mp_expert_mlp_workspace", N, k, E, H, Fo, out_dtype)


def mp_expert_mlp(x, x_dtype, x_scales, N, K, ldx, idx, weight, k, E, H, Fo, w1, w1_scales, w2, w2_scales,
                  act, gated, residual, ldr, out, out_dtype, ws, ws_bytes, stream=None):
    """x and residual: tensors (rows may be strided) or raw addresses."""
    _check("mp_expert_mlp", _layers().mp_expert_mlp(
        _rows(x), x_dtype, _ptr(x_scales), N, K, ldx, _ptr(idx), _ptr(weight), k, E, H, Fo, _ptr(w1),
        _ptr(w1_scales), _ptr(w2), _ptr(w2_scales), act, gated, _rows(residual), ldr,
        _ptr(out), out_dtype, _ptr(ws), ws_bytes, _stream(stream)))


def _expert_weights(w, cols, name):
    """codes (or bf16 weights) [E, rows, ...] and scales or None, for rows of `cols` values."""
    if isinstance(w, torch.Tensor):
        if w.dim() != 3 or w.dtype != torch.bfloat16 or w.shape[2] != cols:
            raise ValueError(f"{name}: [E, rows, {cols}] bf16, or codes and scales of mx_quantize expected")
        return w, None
    codes, scales = w
    _mx(codes, scales, cols)
    if codes.dim() != 3:
        raise ValueError(f"{name}: codes [E, rows, ...] expected")
    return codes, scales


def expert_mlp(x, idx, weight, w1, w2, *, act="silu", gated=True, residual=None, out_dtype=None, out=None,
               stream=None):
    """What the chosen experts make of few rows (at most 64): [N, Fo] of out_dtype,
    out[r] = residual[r] + sum_j weight[r, j] * w2[e] h with e = idx[r, j] and h = act(w1[e] x[r]), or
    with gated act(g) * u, where g and u are the two halves of w1[e] x[r].

    x: [N, K] fp32 or bf16, or (codes, scales) of rms_norm_mx8.  idx [N, k] int32 and weight [N, k] fp32
    are route's (idx -1: no choice).  w1 [E, (2 if gated else 1) * H, K] and w2 [E, Fo, H]: bf16 both, or
    both as (codes, scales) of mx_quantize.  out_dtype: default x's, bf16 for rows in 8 bits.

    For the many rows of a batch sort them by expert (coo_to_csr) and take mx_segment_matmul, or segment_matmul
    (rows and W.transpose(1, 2) in bf16).  The former takes the rows in 4 bits, which this call does not, so
    that its results differ by that rounding."""
    a = _act(act)
    if isinstance(x, torch.Tensor):
        xs, K, dt = None, int(x.shape[1]), _dtype_code(x.dtype)
        N = int(x.shape[0])
        default = x.dtype
    else:
        x, xs = x
        _mx8(x, xs, x.shape[1])
        N, K, dt, default = int(x.shape[0]), int(x.shape[1]), MP_F32, torch.bfloat16
    if xs is not None:
        # blocks are whole: places past K hold zeros
        K = int(w1.shape[2]) if isinstance(w1, torch.Tensor) else K
        if _blocks(K) != xs.shape[1]:
            raise ValueError("rows in 8 bits must have the blocks of w1's columns")
    if isinstance(w1, torch.Tensor) != isinstance(w2, torch.Tensor):
        raise ValueError("w1 and w2 must both be bf16 or both in 4 bits")
    c1, s1 = _expert_weights(w1, K, "w1")
    E, rows = int(c1.shape[0]), int(c1.shape[1])
    if gated and rows % 2:
        raise ValueError("w1 of gated experts has 2 H rows")
    H = rows // 2 if gated else rows
    c2, s2 = _expert_weights(w2, H, "w2")
    Fo = int(c2.shape[1])
    if int(c2.shape[0]) != E:
        raise ValueError("w1 and w2 must be of as many experts")
    if idx.dim() != 2 or int(idx.shape[0]) != N:
        raise ValueError("idx [N, k] expected")
    k = int(idx.shape[1])
    _vector(idx, N * k, torch.int32, "idx")
    _vector(weight, N * k, torch.float32, "weight")
    if weight.shape != idx.shape:
        raise ValueError("weight must have the shape of idx")
    if out is not None and tuple(out.shape) != (N, Fo):
        raise ValueError("out must be [N, Fo]")
    kind = out.dtype if out is not None else out_dtype or default
    if residual is not None and (tuple(residual.shape) != (N, Fo) or residual.dtype != kind):
        raise ValueError("residual must have the shape and dtype of out")
    _on_gpu(x, xs, idx, weight, c1, s1, c2, s2, residual, out)
    xp, ldx = _rows_ptr(x) if xs is None else (_ptr(x), K)
    rp, ldr = _rows_ptr(residual) if residual is not None else (None, Fo)
    od = _dtype_code(kind)
    nb = _sized(mp_expert_mlp_workspace, N, k, E, H, Fo, od)
    with _on(stream):
        if out is None:
            out = torch.empty(N, Fo, dtype=kind, device=x.device)
        ws = _workspace(nb, x.device)
        mp_expert_mlp(xp, dt, xs, N, K, ldx, idx, weight, k, E, H, Fo, c1, s1, c2, s2, a, int(bool(gated)), rp,
                      ldr, out, od, ws, nb, stream)
    return out
