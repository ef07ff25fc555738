"""Embeddings, root-mean-square norm, 8-bit values and the experts of rows in 64 bits, in numpy, written
from their definitions (include/mp_layers.h) without the package's code."""
from __future__ import annotations

import math

import numpy as np
import torch

import layer_refs

U = 2.0 ** -24  # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- embeddings ---------------------------------------------------------------------------

def inside(ids, V, padding=None):
    ok = (ids >= 0) & (ids < V)
    return ok if padding is None else ok & (ids != padding)


def embed(ids, table, scale, padding=None):
    ok = inside(ids, len(table), padding)
    return np.where(ok[:, None], table[np.where(ok, ids, 0)] * float(np.float32(scale)), 0.0)


def embed_backward(ids, dout, V, scale, padding=None):
    """dtable, the sums of magnitudes and the rows of each id."""
    ok = inside(ids, V, padding)
    d, size, count = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V)
    np.add.at(d, ids[ok], dout[ok])
    np.add.at(size, ids[ok], np.abs(dout[ok]))
    np.add.at(count, ids[ok], 1)
    s = float(np.float32(scale))
    return d * s, size * abs(s), count


# ---- root-mean-square norm -------------------------------------------------------------------

def rms_norm(total, weight, eps):
    rstd = 1 / np.sqrt((total ** 2).mean(1) + float(np.float32(eps)))
    xhat = total * rstd[:, None]
    return xhat * weight, rstd, xhat


def rms_norm_backward(total, dout, weight, eps, dtotal=None):
    """dx and the size of its terms, dweight and the size of its terms."""
    _, rstd, xhat = rms_norm(total, weight, eps)
    g = dout * weight
    c = (g * xhat).mean(1, keepdims=True)
    r = rstd[:, None]
    dx = r * (g - xhat * c)
    size = np.abs(r) * (np.abs(g) + np.abs(xhat) * np.abs(g * xhat).mean(1, keepdims=True))
    if dtotal is not None:
        dx, size = dx + dtotal, size + np.abs(dtotal)
    return dx, size, (dout * xhat).sum(0), np.abs(dout * xhat).sum(0)


# ---- microscaled 8-bit floating point ----------------------------------------------------------

E4M3 = np.array([m / 512 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])
E4M3[127] = np.nan


def mx8_quantize(v):
    """v [N, K] (fp32 values as float64) -> codes [N, KB, 32], scale bytes [N, KB]."""
    n, k = v.shape
    kb = -(-k // 32)
    a = np.zeros((n, kb * 32))
    a[:, :k] = v
    a = a.reshape(n, kb, 32)
    bad = ~np.isfinite(a).all(2)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(a), a, 0)).max(2))
    e = np.frexp(np.where(top == 0, 1.0, top))[1] - 1
    s = np.clip(e - 8 + 127, 0, 254)
    s = np.where(top == 0, 0, s)
    q = np.abs(np.where(bad[..., None], 0.0, a)) / np.exp2(s - 127.0)[..., None]
    s = np.where(bad, 255, s)
    lower = np.clip(np.searchsorted(E4M3[:127], q, side="right") - 1, 0, 125)
    down, up = E4M3[lower], E4M3[lower + 1]
    near = np.where(q - down == up - q, lower + lower % 2, np.where(q - down < up - q, lower, lower + 1))
    code = near + 128 * np.signbit(np.where(bad[..., None], 0.0, a))
    return code.astype(np.int64), s.astype(np.int64)


def mx8_values(code, s):
    """[N, KB, 32] codes and [N, KB] scales -> [N, KB * 32] values."""
    v = np.where(code >= 128, -1.0, 1.0) * E4M3[code & 127] * np.exp2(np.where(s == 255, 0, s) - 127.0)[..., None]
    return np.where((s == 255)[..., None], np.nan, v).reshape(code.shape[0], -1)


# ---- the experts of rows -------------------------------------------------------------------------

def expert_mlp(x, idx, weight, w1, w2, act, gated):
    """out and, element by element, a bound on what the rounding of h's factors and sums can make of it
    relative to one rounding: sum_j |w_j| |w2| |h|size."""
    n, h = x.shape[0], w2.shape[2]
    out, size = np.zeros((n, w2.shape[1])), np.zeros((n, w2.shape[1]))
    for r in range(n):
        for j in range(idx.shape[1]):
            e = idx[r, j]
            if e < 0 or e >= w1.shape[0]:
                continue
            z, zs = w1[e] @ x[r], np.abs(w1[e]) @ np.abs(x[r])
            a, slope = layer_refs.act(z[:h], act)
            # an error of z[:h] reaches a by the slope, at most 1.13 for these functions
            hs = np.abs(a) + 1.13 * zs[:h]
            if gated:
                hs = hs * np.abs(z[h:]) + np.abs(a) * zs[h:]
                a = a * z[h:]
            out[r] += weight[r, j] * (w2[e] @ a)
            size[r] += abs(weight[r, j]) * (np.abs(w2[e]) @ hs)
    return out, size
