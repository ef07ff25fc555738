"""The operators around the aggregation in 64 bits, in numpy, written from their definitions
(include/mp_layers.h) without the package's code."""
from __future__ import annotations

import math

import numpy as np
import torch


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- dropout ------------------------------------------------------------------------------

def philox(counter, key):
    """Philox4x32-10: counter [n, 4] and key (2 values) of 32 bits -> [n, 4]."""
    c = [np.asarray(counter[:, i], np.uint64) for i in range(4)]
    low = np.uint64(0xFFFFFFFF)
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, 1)


def words(e, seed, t):
    """The 16-bit word of every element number."""
    e = np.asarray(e, np.uint64).reshape(-1)
    b = e // np.uint64(8)
    c = np.stack([b % np.uint64(2 ** 32), b // np.uint64(2 ** 32),
                  np.full_like(b, t % 2 ** 32), np.full_like(b, t // 2 ** 32)], 1)
    w = philox(c, (seed % 2 ** 32, seed // 2 ** 32))
    h = np.stack([w & np.uint64(65535), w >> np.uint64(16)], 2).reshape(-1, 8)
    return h[np.arange(len(e)), (e % np.uint64(8)).astype(np.int64)]


def dropout(x, p, seed, t=0, ids=None, rows=False, residual=None):
    """x [N, F] float64 -> (out, keep [N, F])."""
    n, f = x.shape
    who = np.arange(n, dtype=np.uint64) if ids is None else ids.astype(np.uint64)
    e = who[:, None] if rows else who[:, None] * np.uint64(f) + np.arange(f, dtype=np.uint64)
    limit = math.floor(65536 * p + 0.5)
    keep = np.broadcast_to((words(e, seed, t) >= limit).reshape(e.shape), (n, f))
    out = np.where(keep, x * (65536 / max(1, 65536 - limit)), 0.0)
    return out if residual is None else out + residual, keep


# ---- router -------------------------------------------------------------------------------

def choose(l, k, mask=None):
    """idx [N, k] of logits l [N, E] float64 (equal logits: lower number first; -inf never), and which
    rows take part."""
    n, e = l.shape
    part = np.ones(n, bool) if mask is None else mask.astype(bool)
    part = part & (np.where(part[:, None], l, -np.inf) > -np.inf).any(1)
    idx = np.full((n, k), -1, np.int64)
    for r in np.nonzero(part)[0]:
        order = sorted(range(e), key=lambda i: (-l[r, i], i))
        for j in range(k):
            if l[r, order[j]] > -np.inf:
                idx[r, j] = order[j]
    return idx, part


def route(l, idx, part, renorm=True):
    """weight, counts, loss [balance, z], and what the gradient needs, for given choices."""
    n, e = l.shape
    safe = np.where(part[:, None], l, 0.0)
    big = safe.max(1, keepdims=True)
    p = np.where(part[:, None], np.exp(safe - big), 0.0)
    tot = np.where(part, p.sum(1), 1.0)
    p = p / tot[:, None]
    real = idx >= 0
    w = np.where(real, np.take_along_axis(p, np.maximum(idx, 0), 1), 0.0)
    if renorm:
        w = w / np.where(part, w.sum(1), 1.0)[:, None]
    counts = np.bincount(idx[real], minlength=e)
    rows = int(part.sum())
    lse = np.where(part, np.log(tot) + big[:, 0], 0.0)
    balance = e * float((counts / max(1, counts.sum()) * p.sum(0) / max(1, rows)).sum())
    return w, counts, rows, np.array([balance, float((lse ** 2).sum()) / max(1, rows)]), p, lse


def route_backward(l, idx, part, dweight, dloss, renorm=True):
    """dL/dl and, element by element, the size of the terms that make it up."""
    n, e = l.shape
    w, counts, rows, _, p, lse = route(l, idx, part, renorm)
    real = idx >= 0
    dw = np.where(real, dweight, 0.0)
    S = (w * dw).sum(1, keepdims=True)
    d = dloss[0] * e * counts / max(1, counts.sum()) / max(1, rows)
    z = 2 * dloss[1] * lse[:, None] / max(1, rows)
    pd = (p * d).sum(1, keepdims=True)
    g = p * (d - pd + z - (0 if renorm else S))
    size = p * (np.abs(d) + np.abs(pd) + np.abs(z) + (0 if renorm else np.abs(w * dw).sum(1, keepdims=True)))
    for r in range(n):
        for j in range(idx.shape[1]):
            if real[r, j]:
                g[r, idx[r, j]] += w[r, j] * (dw[r, j] - (S[r, 0] if renorm else 0))
                size[r, idx[r, j]] += w[r, j] * (abs(dw[r, j]) + np.abs(w[r] * dw[r]).sum())
    return np.where(part[:, None], g, 0.0), size


# ---- group norm ---------------------------------------------------------------------------

def _erf(v):
    return torch.erf(torch.from_numpy(np.ascontiguousarray(v))).numpy()


def act(z, name):
    """act(z) and its derivative."""
    if name == "relu":
        return np.maximum(z, 0), (z > 0).astype(np.float64)
    if name == "silu":
        g = 1 / (1 + np.exp(-z))
        return z * g, g + z * g * (1 - g)
    if name == "gelu":
        g = 0.5 * (1 + _erf(z / math.sqrt(2)))
        return z * g, g + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, np.ones_like(z)


def group_norm(ptr, x, groups, weight, bias, eps, name):
    """A dict of out, mean, rstd, xhat and z for x [N, F] float64."""
    n, f = x.shape
    s, w = len(ptr) - 1, f // groups
    mean, rstd = np.zeros((s, groups)), np.zeros((s, groups))
    xhat = np.zeros((n, groups, w))
    for i in range(s):
        v = x[ptr[i]:ptr[i + 1]].reshape(-1, groups, w)
        if not v.shape[0]:
            continue
        mean[i] = v.mean((0, 2))
        rstd[i] = 1 / np.sqrt(((v - mean[i][:, None]) ** 2).mean((0, 2)) + eps)
        xhat[ptr[i]:ptr[i + 1]] = (v - mean[i][:, None]) * rstd[i][:, None]
    xhat = xhat.reshape(n, f)
    z = xhat * weight + bias
    return dict(out=act(z, name)[0], mean=mean, rstd=rstd, xhat=xhat, z=z)


def group_norm_backward(ptr, r, dout, groups, weight, name):
    """dx, dweight, dbias from what group_norm returned."""
    n, f = dout.shape
    w = f // groups
    da = dout * act(r["z"], name)[1]
    dweight, dbias = (da * r["xhat"]).sum(0), da.sum(0)
    g = (da * weight).reshape(n, groups, w)
    xh = r["xhat"].reshape(n, groups, w)
    dx = np.zeros((n, groups, w))
    for i in range(len(ptr) - 1):
        a, b = ptr[i], ptr[i + 1]
        if a == b:
            continue
        m1, m2 = g[a:b].mean((0, 2))[:, None], (g[a:b] * xh[a:b]).mean((0, 2))[:, None]
        dx[a:b] = r["rstd"][i][:, None] * (g[a:b] - m1 - xh[a:b] * m2)
    return dx.reshape(n, f), dweight, dbias


# ---- microscaled 4-bit floating point --------------------------------------------------------

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx_quantize(x):
    """x [N, K] float64 (values of fp32 or bf16) -> codes [N, KB, 32], scale bytes [N, KB], values
    [N, K]."""
    n, k = x.shape
    kb = -(-k // 32)
    v = np.zeros((n, kb * 32))
    v[:, :k] = x
    v = v.reshape(n, kb, 32)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(2)
        bad = ~np.isfinite(v).all(2)
        e = np.frexp(np.where(bad | (top == 0), 1.0, top))[1] - 1  # floor(log2)
        s = np.clip(e - 2 + 127, 0, 254)
        s = np.where(top == 0, 0, s)
        s = np.where(bad, 255, s)
        a = np.abs(np.where(bad[..., None], 0.0, v)) / np.exp2(np.where(bad, 127, s) - 127.0)[..., None]
    # nearest of the eight magnitudes; halfway, the one with the even code
    dist = np.abs(a[..., None] - E2M1)
    near = dist.min(-1, keepdims=True)
    cand = dist == near
    code = np.where(cand[..., 0::2].any(-1) & (cand.sum(-1) > 1), 2 * cand[..., 0::2].argmax(-1),
                    cand.argmax(-1))
    code = code + 8 * np.signbit(v)
    value = mx_values(code, s).reshape(n, -1)[:, :k]
    return code, s, value


def mx_values(code, s):
    sign = np.where(code >= 8, -1.0, 1.0)
    v = sign * E2M1[code & 7] * np.exp2(np.where(s == 255, 127, s) - 127.0)[..., None]
    return np.where((s == 255)[..., None], np.nan, v)


def mx_pack(code):
    """[..., KB, 32] codes -> [..., KB * 16] bytes."""
    b = code[..., 0::2] | (code[..., 1::2] << 4)
    return b.reshape(*code.shape[:-2], -1).astype(np.uint8)
