"""GPU: orthogonalize under coefficients near the ends of their range."""
import pytest
import torch

import layer_reference as ref
from test_gpu_worker import U, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("table", [[(0.0, 0.0, 0.0)], [(1e-310, 0.0, 0.0)], [(5e-324, 0.0, 0.0), (1.0, -0.5, 0.0)], [(1e-200, 0.0, 0.0), (3e38, 0.0, 0.0)], [(0.0, 0.0, 1e-300), (1.0, 1.0, 1.0)],
                                   [(1e-280, 0.0, 0.0)] * 3])
@pytest.mark.parametrize("count, rows, cols", [(2, 30, 50), (1, 60, 900), (1, 200, 300)])
def test_what_becomes_nothing_leaves_the_base(count, rows, cols, table):
    """All singular values are below 1e-150 in the end, which no type holds."""
    import paper_2605_01989_amd as dblp
    g = gen(rows)
    x, base = (torch.randn(count, rows, cols, generator=g, device="cuda") for _ in range(2))
    out = torch.empty_like(x)
    dblp.orthogonalize(x, out, torch.full((dblp.orthogonalize_workspace(count, rows, cols),), 255, dtype=torch.uint8, device="cuda"), base=base, steps=len(table), coefficients=table)
    assert torch.equal(out, base)


@pytest.mark.parametrize("rows, cols", [(30, 50), (60, 900), (200, 300)])
def test_small_coefficients_and_large_ones_after(rows, cols):
    """X times 1e-38, or 1e-80 in steps, and back: as near as after as many ordinary steps."""
    import paper_2605_01989_amd as dblp
    x = torch.randn(rows, cols, generator=gen(cols), device="cuda")
    out = torch.empty_like(x)
    ws = torch.empty(dblp.orthogonalize_workspace(1, rows, cols), dtype=torch.uint8, device="cuda")
    want = x.cpu().double() / x.cpu().double().norm()
    for table in ([(1e-38, 0.0, 0.0), (1e38, 0.0, 0.0)], [(1e-40, 0.0, 0.0), (1e-40, 0.0, 0.0), (1e38, 0.0, 0.0), (1e38, 0.0, 0.0), (1e4, 0.0, 0.0)]):
        dblp.orthogonalize(x, out, ws, steps=len(table), coefficients=table)
        # a step holds a I and X with 22 bits, and rounds coefficients and sums to fp32
        assert float((out.cpu().double() - want).norm()) <= len(table) * (3 * 2.0 ** -22 + 8 * U)
