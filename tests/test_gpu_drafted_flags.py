"""Bad pages under items that are cut: what a row becomes goes by the pages that its item reads in this very call, not by the cut or by a call before."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import drafted_reference as dr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("users", [1, 60])
def test_zeros_where_the_page_was_needed(dtype, users):
    """A long run whose last page is out of range: only the rows of the last tile need it, whether items are cut (one user) or not."""
    n, hq = 600, 4
    w = dr.batch([n] * users, [3000] + [0] * (users - 1), [0] * users, hq, 1, 64, dtype, seed=5, kind="run")
    g = dr.OnDevice(w)
    rows = set(range(0, 576, 53)) | {574, 575}
    want, _, _, _, tol = dr.expected(w, rows=rows)
    g.pub.page_indices[int(g.pub.page_indptr[0]) + (n - 1) // 16] = 1 << 29
    out = g.fused()
    assert spd.spd_query_device_status(g.ws) == (4, 0)
    at = torch.tensor(sorted(rows))
    dr.close(out[at.cuda()], want[at], tol[at])
    assert bool((out[592:600] == 0).all())                   # tokens 592 .. 599 lie in that page; tiles of at most 64 tokens start at 576


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_replayed_graph_judges_its_users_afresh(dtype):
    """A page that was out of range at one replay and is mended before the next leaves nothing behind."""
    w = dr.batch([6, 2], [5000, 3001], [77, 0], 4, 1, 64, dtype, seed=6)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    out, side = g.out(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g.fused(out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.fused(out=out)
    entry = int(g.priv.page_indptr[0]) + 3
    page = int(g.priv.page_indices[entry])
    for bad in (False, True, False, True, False):
        g.priv.page_indices[entry] = -7 if bad else page
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        if bad:
            assert bool((out[:6] == 0).all())
            dr.close(out[6:], want[6:], tol[6:])
        else:
            dr.close(out, want, tol)
    assert spd.spd_query_device_status(g.ws) == (4, 0)
