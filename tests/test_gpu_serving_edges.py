"""More GPU tests of the serving calls: long runs of short requests, strides and alignments, extreme and non-finite
values.  Formulas and tolerances are those of test_gpu_serving.py."""
import numpy as np
import pytest
import torch

from paper_2502_01681_b200 import dg4
from tests.test_gpu_serving import BF16, desc, edgeless, i32, make_adapters, normal, project_ref, within

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------
# projections with adapters
# ---------------------------------------------------------------------------------------------------
def project_ref_by_adapter(x, w, ad, ptr, ids, res=None):
    """project_ref with the rows of one adapter taken together: it is one formula per row, and thousands of products of a
    few rows are slow on the CPU."""
    of_row = torch.from_numpy(np.repeat(ids, np.diff(ptr)))
    y, tol = (torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64) for _ in range(2))
    for i in sorted(set(ids)):
        at = torch.nonzero(of_row == i)[:, 0]
        on = at.cuda()
        y[at], tol[at], _ = project_ref(x[on], w, ad, [0, len(at)], [i], None if res is None else res[on])
    return y, tol


@pytest.mark.parametrize("rank,residual", [(16, True), (16, False), (64, True), (64, False), (8, True)])
def test_out_projection_over_thousands_of_short_requests(rank, residual):
    """Some forty items per CTA, the adapter (or none) another at nearly every one: the next item's product runs ahead of
    this one's second product all along.  Every repetition gives the same bits."""
    rng = np.random.default_rng(11)
    count = 6000
    lens = rng.choice([1, 2, 7, 31, 32, 33, 64], size=count)
    ptr = np.concatenate([[0], np.cumsum(lens)]).tolist()
    n, ids = ptr[-1], rng.integers(-1, 8, size=count).tolist()
    g = edgeless(n)
    o, w, res, ad = normal(1, (n, 128)), normal(2, (128, 128), 0.1), normal(4, (n, 128)), make_adapters(3, 8, rank, 128)
    seg = dg4.segments(i32(ptr), i32(ids))
    first = torch.empty((n, 128), dtype=BF16, device="cuda")
    dg4.dg4_out_project_adapters(g, desc(residual=residual), o, w, ad, seg, res, first)
    y, tol = project_ref_by_adapter(o, w, ad, ptr, ids, res if residual else None)
    within(first, y, tol)
    for _ in range(30):
        again = torch.zeros_like(first)
        dg4.dg4_out_project_adapters(g, desc(residual=residual), o, w, ad, seg, res, again)
        assert torch.equal(first, again)
    assert dg4.dg4_graph_poll_status(g) == 0
