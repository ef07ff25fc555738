"""CPU checks of include/mp_layers.h: every function is exported, and bad arguments are refused on
the host, before anything is enqueued (the pointers are fake and never followed)."""
import os
import re

import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp
from paper_2507_16991_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000


def test_exports_every_declared_function():
    text = open(os.path.join(ROOT, "include", "mp_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\bint (mp_[a-z0-9_]+)\s*\(", text))
    assert "mp_dropout" in names
    for n in names:
        assert hasattr(mp.lib(), n), f"{n} declared but not exported"
        assert getattr(mp, n), f"{n} has no binding"


def refused(fn, base, status, **change):
    args = dict(base, **change)
    assert getattr(layers._layers(), fn)(*args.values()) == status, change


DROPOUT = dict(x=FAKE, dtype=0, N=10, F=8, ldx=8, residual=None, ldr=8, ids=None, whole_rows=0, p=0.5,
               seed=1, offset=0, step=None, out=FAKE, ldo=8, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(dtype=2)), (-2, dict(N=-1)), (-2, dict(N=2 ** 31)), (-2, dict(F=0)),
    (-2, dict(F=65537, ldx=65537, ldo=65537)), (-2, dict(ldx=7)), (-2, dict(ldo=7)),
    (-2, dict(residual=FAKE, ldr=7)), (-2, dict(p=-0.1)), (-2, dict(p=1.1)),
    (-2, dict(p=float("nan"))), (-1, dict(x=None)), (-1, dict(out=None)), (-8, dict(x=FAKE + 2)),
    (-8, dict(out=FAKE + 1)), (-8, dict(residual=FAKE + 2)), (-8, dict(ids=FAKE + 2)),
    (-8, dict(step=FAKE + 4))])
def test_dropout_refusals(status, change):
    refused("mp_dropout", DROPOUT, status, **change)


def test_nothing_to_do_is_accepted():
    assert layers._layers().mp_dropout(*dict(DROPOUT, N=0, x=None, out=None).values()) == 0


def test_operands_elsewhere_are_refused():
    with pytest.raises(ValueError):
        mp.dropout(torch.zeros(4, 4), 0.5, 1)


def test_philox_published_outputs():
    """The known answers that its authors publish for Philox4x32-10."""
    ones = 0xFFFFFFFF
    cases = [([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
             ([ones] * 4, [ones] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
             ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
              [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]
    for counter, key, out in cases:
        assert ref.philox(np.array([counter]), key).tolist() == [out]


ROUTE = dict(logits=FAKE, dtype=0, N=10, E=8, ldl=8, k=2, mask=None, renorm=1, idx=FAKE, weight=FAKE,
             counts=FAKE, loss=FAKE, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(dtype=7)), (-2, dict(N=-1)), (-2, dict(N=2 ** 31)), (-2, dict(E=0)),
    (-2, dict(E=1025, ldl=1025)), (-2, dict(ldl=7)), (-2, dict(k=0)), (-2, dict(k=9)),
    (-2, dict(N=2 ** 30, k=2)), (-2, dict(E=100, ldl=100, k=65)), (-1, dict(logits=None)),
    (-1, dict(idx=None)), (-1, dict(weight=None)), (-1, dict(counts=None)), (-1, dict(loss=None)),
    (-8, dict(logits=FAKE + 2)), (-8, dict(idx=FAKE + 2)), (-8, dict(counts=FAKE + 1)),
    (-1, dict(N=100000)), (-5, dict(N=100000, ws=FAKE, ws_bytes=64))])
def test_route_refusals(status, change):
    refused("mp_route", ROUTE, status, **change)


ROUTE_BACKWARD = dict(logits=FAKE, dtype=1, N=10, E=8, ldl=8, k=2, mask=None, renorm=1, idx=FAKE,
                      weight=FAKE, counts=FAKE, dweight=None, dloss=None, dlogits=FAKE, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(dtype=7)), (-2, dict(k=9)), (-1, dict(dlogits=None)), (-1, dict(counts=None)),
    (-8, dict(dweight=FAKE + 2)), (-8, dict(dloss=FAKE + 2)), (-8, dict(dlogits=FAKE + 1))])
def test_route_backward_refusals(status, change):
    refused("mp_route_backward", ROUTE_BACKWARD, status, **change)


def test_route_workspace():
    assert mp.mp_route_workspace(0, 64) == 0 and mp.mp_route_workspace(16, 64) == 0
    assert mp.mp_route_workspace(10 ** 6, 64) > 0
    for bad in ((-1, 8), (2 ** 31, 8), (8, 0), (8, 1025)):
        with pytest.raises(mp.MPError):
            mp.mp_route_workspace(*bad)


NORM = dict(ptr=FAKE, ptr_itype=0, x=FAKE, x_dtype=0, N=10, S=2, F=8, ldx=8, G=2, gamma=None, beta=None,
            eps=1e-5, act=0, out=FAKE, out_dtype=0, mean=FAKE, rstd=FAKE, ws=None, ws_bytes=0,
            stream=None)
NORM_BACKWARD = dict(ptr=FAKE, ptr_itype=0, x=FAKE, x_dtype=0, dout=FAKE, N=10, S=2, F=8, ldx=8, G=2,
                     gamma=None, beta=None, mean=FAKE, rstd=FAKE, act=0, dx=FAKE, dx_dtype=0,
                     dgamma=FAKE, dbeta=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
SHARED = [(-3, dict(ptr_itype=2)), (-3, dict(x_dtype=2)), (-2, dict(N=-1)), (-2, dict(S=0)),
          (-2, dict(F=0)), (-2, dict(F=65537, ldx=65537)), (-2, dict(G=0)), (-2, dict(G=3)),
          (-2, dict(G=16)), (-2, dict(ldx=7)), (-2, dict(act=4)), (-2, dict(act=-1)),
          (-1, dict(ptr=None)), (-1, dict(x=None)), (-1, dict(mean=None)), (-1, dict(rstd=None)),
          (-8, dict(ptr=FAKE + 4, ptr_itype=1)), (-8, dict(x=FAKE + 2)), (-8, dict(gamma=FAKE + 2)),
          (-8, dict(beta=FAKE + 1)), (-8, dict(mean=FAKE + 2)), (-8, dict(ws=FAKE + 8))]


@pytest.mark.parametrize("status,change", SHARED + [
    (-3, dict(out_dtype=5)), (-2, dict(eps=-1.0)), (-2, dict(eps=float("nan"))),
    (-2, dict(eps=float("inf"))), (-1, dict(out=None)), (-8, dict(out=FAKE + 2)),
    (-1, dict(N=10 ** 6)), (-5, dict(N=10 ** 6, ws=FAKE, ws_bytes=64))])
def test_group_norm_refusals(status, change):
    refused("mp_group_norm", NORM, status, **change)


@pytest.mark.parametrize("status,change", SHARED + [
    (-3, dict(dx_dtype=5)), (-1, dict(dout=None)), (-1, dict(dgamma=None)), (-1, dict(dbeta=None)),
    (-1, dict(dx=None, dgamma=None, dbeta=None)), (-8, dict(dout=FAKE + 2)), (-8, dict(dx=FAKE + 2)),
    (-1, dict(ws=None)), (-5, dict(ws_bytes=16))])
def test_group_norm_backward_refusals(status, change):
    refused("mp_group_norm_backward", NORM_BACKWARD, status, **change)


def test_group_norm_workspace():
    assert mp.mp_group_norm_workspace(100, 5, 64, 8, 0, False) == 0
    assert mp.mp_group_norm_workspace(10 ** 6, 5, 64, 8, 0, False) > 0
    assert mp.mp_group_norm_workspace(100, 5, 64, 8, 1, True) > 0
    with pytest.raises(mp.MPError):
        mp.mp_group_norm_workspace(100, 5, 64, 7, 0, False)


QUANTIZE = dict(x=FAKE, dtype=0, N=10, K=64, ldx=64, codes=FAKE, scales=FAKE, values=None, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(dtype=2)), (-2, dict(N=-1)), (-2, dict(N=2 ** 31)), (-2, dict(K=0)), (-2, dict(ldx=63)),
    (-2, dict(K=65537, ldx=65537)), (-1, dict(x=None)), (-1, dict(codes=None)), (-1, dict(scales=None)),
    (-1, dict(codes=None, scales=None)), (-8, dict(x=FAKE + 2)), (-8, dict(codes=FAKE + 8)),
    (-8, dict(values=FAKE + 2))])
def test_quantize_refusals(status, change):
    refused("mp_mx_quantize", QUANTIZE, status, **change)


DEQUANTIZE = dict(codes=FAKE, scales=FAKE, N=10, K=64, out=FAKE, dtype=0, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(dtype=2)), (-2, dict(N=-1)), (-2, dict(K=0)), (-1, dict(codes=None)),
    (-1, dict(scales=None)), (-1, dict(out=None)), (-8, dict(codes=FAKE + 4)), (-8, dict(out=FAKE + 2))])
def test_dequantize_refusals(status, change):
    refused("mp_mx_dequantize", DEQUANTIZE, status, **change)


PRODUCT = dict(seg=FAKE, seg_itype=0, T=2, x=FAKE, x_dtype=1, N=10, K=64, ldx=64, w_codes=FAKE,
               w_scales=FAKE, Fo=32, out=FAKE, out_dtype=0, ws=FAKE, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("status,change", [
    (-3, dict(seg_itype=2)), (-3, dict(x_dtype=2)), (-3, dict(out_dtype=2)), (-2, dict(T=0)),
    (-2, dict(T=4097)), (-2, dict(N=-1)), (-2, dict(K=0)), (-2, dict(ldx=63)), (-2, dict(Fo=0)),
    (-2, dict(Fo=65537)), (-1, dict(seg=None)), (-1, dict(w_codes=None)), (-1, dict(w_scales=None)),
    (-1, dict(x=None)), (-1, dict(out=None)), (-1, dict(ws=None)), (-8, dict(seg=FAKE + 4, seg_itype=1)),
    (-8, dict(x=FAKE + 1)), (-8, dict(w_codes=FAKE + 8)), (-8, dict(out=FAKE + 2)),
    (-8, dict(ws=FAKE + 8)), (-5, dict(ws_bytes=16))])
def test_product_refusals(status, change):
    refused("mp_mx_segment_matmul", PRODUCT, status, **change)


def test_product_workspace():
    assert mp.mp_mx_segment_matmul_workspace(2, 100, 64, 32) >= 100 * 34
    for bad in ((0, 100, 64, 32), (2, -1, 64, 32), (2, 100, 0, 32), (2, 100, 64, 0), (4097, 1, 1, 1)):
        with pytest.raises(mp.MPError):
            mp.mp_mx_segment_matmul_workspace(*bad)


@pytest.mark.parametrize("rows", [1, 2])
def test_tables_of_strided_columns_are_refused(rows):
    """A view of every second column, of one row as of several."""
    buf = torch.arange(32.0).view(2, 16)
    with pytest.raises(ValueError):
        mp._rows_ptr(buf[:rows, ::2])


def test_tables_of_strided_rows_are_taken():
    buf = torch.arange(32.0).view(2, 16)
    for t, ld in ((buf, 16), (buf[:, 3:8], 16), (buf[:1, 3:8], 5), (buf[:, 2:3], 16), (buf[:0, ::2], 8),
                  (buf[1:, 5:6], 1), (buf[1:, 4:10:8], 1)):
        address, stride = mp._rows_ptr(t)
        assert stride == ld and (not t.numel() or address == t.data_ptr())


def test_quantize_copies_a_view_on_the_stream_of_the_call(monkeypatch):
    """A transposed weight is made contiguous within the context of the call's stream, which orders the
    copy after its producer and before the kernel, and owns its memory."""
    inside, copies, calls = [], [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            inside.append(self.stream)

        def __exit__(self, *_):
            inside.pop()

    contiguous = torch.Tensor.contiguous

    def copy(t, *a, **k):
        copies.append(list(inside))
        return contiguous(t, *a, **k)

    monkeypatch.setattr(layers, "_on", On)
    monkeypatch.setattr(layers, "_on_gpu", lambda *_: None)
    monkeypatch.setattr(torch.Tensor, "contiguous", copy)
    monkeypatch.setattr(layers, "mp_mx_quantize", lambda *a: calls.append((a, list(inside))))
    w = torch.zeros(2, 64, 40)
    codes, scales = mp.mx_quantize(w.transpose(1, 2), stream="side")
    assert codes.shape == (2, 40, 32) and scales.shape == (2, 40, 2)
    assert copies == [["side"]] and len(calls) == 1 and calls[0][1] == ["side"]
    assert calls[0][0][2:5] == (80, 64, 64)


def test_quantize_takes_views_of_one_table(monkeypatch):
    """What reaches the library: a table of strided rows as it is, other views as contiguous copies."""
    calls = []
    monkeypatch.setattr(layers, "_on_gpu", lambda *_: None)
    monkeypatch.setattr(layers, "mp_mx_quantize", lambda *a: calls.append(a))
    w = torch.zeros(64, 40)
    for view, n, k, ld in ((w, 64, 40, 40), (w[:, 3:36], 64, 33, 40), (w.t(), 40, 64, 64),
                           (w[:, ::2], 64, 20, 20), (w[:1, ::2], 1, 20, 20), (w[:1].expand(5, 40), 5, 40, 40)):
        mp.mx_quantize(view)
        assert calls[-1][2:5] == (n, k, ld)
        assert (calls[-1][0] == view.data_ptr()) == (view.stride(1) == 1 and view.stride(0) >= k)


def test_products_of_more_tiles_than_a_launch_holds_are_refused():
    """By the host, as a size: (N / 128 + min(T, N)) * ceil(Fo / 256) tiles, 2^24 - 8 at most; products
    of few columns and little LDS have no such tiles."""
    query = mp.mp_mx_segment_matmul_workspace
    assert query(1, 2 ** 23 - 256, 32, 65536) > 0   # (2^16 - 1) * 256
    for t, n, k, fo in ((1, 2 ** 23 - 128, 32, 65536), (2, 2 ** 31 - 1, 32, 65536),
                        (1, 2 ** 31 - 1, 65536, 16), (1, 2 ** 31 - 1, 32, 257)):
        with pytest.raises(mp.MPError) as e:
            query(t, n, k, fo)
        assert e.value.status == -2
        refused("mp_mx_segment_matmul", PRODUCT, -2, T=t, N=n, K=k, ldx=k, Fo=fo,
                ws_bytes=2 ** 62)
    for t, n, k, fo in ((1, 2 ** 31 - 1, 32, 1), (4096, 2 ** 31 - 1, 64, 256), (3, 2 ** 31 - 1, 128, 128)):
        assert query(t, n, k, fo) > 0
