"""Sorts of few rows, whose places one tile of each names, on either side of the borders between tiles."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("ids", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 64, 257, 512, 513])
@pytest.mark.parametrize("n", [16385, 100001, 3 << 18, (3 << 18) + 1, 2 ** 20, 2 ** 20 + 1])
def test_rows_and_their_places(n, rows, ids):
    r = np.random.default_rng([n, rows])
    src = torch.from_numpy(r.integers(0, 2 ** 20, n).astype(np.int32)).to(DEV)
    late = np.zeros(n, np.int64)
    late[-3:] = rows - 1  # the last row's edges in the last tile alone
    for dst in (r.integers(0, rows, n), np.sort(r.integers(0, rows, n))[::-1].copy(), late, np.full(n, rows // 2)):
        order = torch.from_numpy(np.argsort(dst, kind="stable")).to(DEV)
        ends = np.concatenate(([0], np.cumsum(np.bincount(dst, minlength=rows))))
        rowptr, col, perm, _ = mp.coo_to_csr(src, torch.from_numpy(dst.astype(np.int32)).to(DEV), rows, want_perm=ids)
        assert np.array_equal(rowptr.cpu().numpy(), ends)
        assert torch.equal(col, src[order])
        assert perm is None or torch.equal(perm.long(), order)


def test_replayed_from_a_graph():
    """Other edges of the same places of memory; a row that had edges has none afterwards."""
    n, rows = 300001, 64
    r = np.random.default_rng(1)
    dst = torch.zeros(n, dtype=torch.int32, device=DEV)
    src = torch.arange(n, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step():
        return mp.coo_to_csr(src, dst, rows, status=status)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for some in (64, 7, 1, 30):
        new = r.integers(0, some, n) * (64 // some)
        dst.copy_(torch.from_numpy(new.astype(np.int32)))
        g.replay()
        torch.cuda.synchronize()
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and int(status) == 0
        assert np.array_equal(got[0].cpu().numpy()[1:], np.cumsum(np.bincount(new, minlength=rows)))
