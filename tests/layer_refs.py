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
