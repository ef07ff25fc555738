"""Group norm where segments are many: on either side of 4,096 segments, from which on a unit takes up to
128 KB of one by itself, and past the two levels of a search by 64 offsets a step.  The definition in 64
bits and the bounds are those of test_gpu_norm.py (C u = 64 2^-24 times the terms' sizes)."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
CU = 64 * 2.0 ** -24
EPS = 1e-5


def segments(s, mean_rows, long_rows, seed):
    """Offsets of s segments: none to twice mean_rows rows, a fifth of them empty, runs of 70 empty ones
    at both ends, and one of long_rows rows a third of the way."""
    r = np.random.default_rng(seed)
    n = r.integers(0, 2 * mean_rows + 1, s)
    n[r.random(s) < 0.2] = 0
    n[:70] = 0
    n[-70:] = 0
    if long_rows:
        n[s // 3] = long_rows
    return np.concatenate([[0], np.cumsum(n)])


def over(v, p, at, g, cg):
    """Sums of v [n, f] over segments and groups, [s, g]."""
    run = np.zeros((v.shape[0] + 1, g))
    np.cumsum(v.reshape(-1, g, cg).sum(2), axis=0, out=run[1:])
    return run[p[1:]] - run[p[:-1]]


def check(s, f, g, dtype, mean_rows, long_rows, seed=1):
    p = segments(s, mean_rows, long_rows, seed)
    n, cg = int(p[-1]), f // g
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, f, generator=gen) + torch.randn(f, generator=gen)).to(dtype).to(DEV)
    dout = torch.randn(n, f, generator=gen).to(dtype).to(DEV)
    weight = (1 + 0.2 * torch.randn(f, generator=gen)).to(DEV)
    bias = (0.3 * torch.randn(f, generator=gen)).to(DEV)
    ptr = torch.from_numpy(p.astype(np.int32)).to(DEV)
    out, mean, rstd = mp.group_norm(ptr, x, g, weight=weight, bias=bias, eps=EPS, act="silu")
    dx, dw, db = mp.group_norm_backward(ptr, x, dout, g, mean, rstd, weight=weight, bias=bias, act="silu")

    x64, w64, d64 = ref.f64(x), ref.f64(weight), ref.f64(dout)
    r = ref.group_norm(p, x64, g, w64, ref.f64(bias), EPS, "silu")
    dx_r, dw_r, db_r = ref.group_norm_backward(p, r, d64, g, w64, "silu")
    empty = np.diff(p) == 0
    assert np.all(ref.f64(mean)[empty] == 0) and np.all(ref.f64(rstd)[empty] == 0)
    at = np.repeat(np.arange(s), np.diff(p))
    big = np.zeros((s, g))
    np.maximum.at(big, at, np.abs(x64).reshape(n, g, cg).max(2))
    T = CU * (1 + big * r["rstd"])
    assert np.all(np.abs(ref.f64(mean) - r["mean"]) <= CU * big)
    assert np.all(np.abs(ref.f64(rstd) - r["rstd"]) <= T * r["rstd"])

    def rows(v):  # [s, g] to [n, f]
        return np.repeat(v[at], cg, axis=1)

    Tx, xh = rows(T), np.abs(r["xhat"])
    rounding = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}[dtype]
    zerr = np.abs(w64) * Tx * (1 + xh) + 2.0 ** -22 * np.abs(r["z"])
    own = 4e-7 * (1 + np.abs(r["z"]))
    assert np.all(np.abs(ref.f64(out) - r["out"]) <= 1.13 * zerr + own + rounding * np.abs(r["out"]))
    d = np.abs(d64)
    da, da_err = 1.13 * d, d * (1.2 * zerr + own) + 2.0 ** -21 * d
    term = da_err * xh + da * Tx * (1 + xh)
    assert np.all(np.abs(ref.f64(db) - db_r) <= (da_err + CU * da).sum(0))
    assert np.all(np.abs(ref.f64(dw) - dw_r) <= (term + CU * da * xh).sum(0))
    wa = np.abs(w64)
    share = 1 / (np.maximum(np.diff(p), 1) * cg)[:, None]

    def mean_of(v):
        return rows(over(v, p, at, g, cg) * share)

    m1, e1 = mean_of(wa * da), mean_of(wa * (da_err + CU * da))
    m2, e2 = mean_of(wa * da * xh), mean_of(wa * (term + CU * da * xh))
    size = wa * da + m1 + xh * m2
    err = wa * da_err + e1 + xh * e2 + Tx * (1 + xh) * m2
    bound = rows(r["rstd"]) * (err + (Tx + 2.0 ** -21) * size)
    assert np.all(np.abs(ref.f64(dx) - dx_r) <= bound + rounding * np.abs(dx_r) + 1e-12)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("s", [4095, 4096, 4097, 8192])
@pytest.mark.parametrize("f,g", [(8, 2), (12, 4)])
def test_either_side_of_the_rule(s, f, g, dtype):
    """Chunks within a group, and chunks of several; segments of a few rows."""
    check(s, f, g, dtype, 6, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("s,f,g,mean_rows,long_rows", [
    (4095, 16, 4, 4, 1500), (4096, 16, 4, 4, 1500),      # a unit's own from 4,096 on
    (4096, 16, 4, 4, 9000), (4100, 15, 5, 3, 12000),     # past 128 KB: tiles
    (5000, 3, 1, 5, 30000), (4096, 256, 8, 2, 600),
    (300000, 4, 2, 1, 0), (300000, 4, 2, 1, 20000)])     # past 64^3 segments
def test_long_ones_among_many(s, f, g, mean_rows, long_rows, dtype):
    check(s, f, g, dtype, mean_rows, long_rows)
