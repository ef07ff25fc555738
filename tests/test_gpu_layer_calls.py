"""Calls of the operators around the aggregation at the corners of what the binding accepts: views,
streams, and tables without rows."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def test_one_row_of_strided_columns_is_refused():
    """As it is for several rows; nothing is read or written beside the view."""
    buf = torch.arange(32, dtype=torch.float32, device=DEV).view(2, 16)
    row, good = buf[:1, ::2], torch.ones(1, 8, device=DEV)
    ptr = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    codes, scales = mp.mx_quantize(torch.ones(1, 4, 8, device=DEV))
    idx, weight, counts, _ = mp.route(good, 2)
    _, mean, rstd = mp.group_norm(ptr, good, 2)
    calls = [lambda: mp.group_norm(ptr, row, 2), lambda: mp.route(row, 2),
             lambda: mp.group_norm_backward(ptr, row, good, 2, mean, rstd),
             lambda: mp.route_backward(row, idx, weight, counts), lambda: mp.dropout(row, 0.5, 1),
             lambda: mp.dropout(good, 0.5, 1, out=row), lambda: mp.dropout(good, 0.5, 1, residual=row),
             lambda: mp.mx_segment_matmul(ptr, row, codes, scales),
             lambda: mp.spmm(ptr, torch.zeros(1, dtype=torch.int32, device=DEV), row, mp.MP_SUM)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    assert torch.equal(buf.view(-1).cpu(), torch.arange(32.0))
    # one value has no stride to be wrong about
    assert mp.dropout(buf[1:, 4:10:8], 0.0, 1).tolist() == [[20.0]]
