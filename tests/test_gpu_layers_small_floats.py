"""GPU: fp32 operands near and below the normal numbers, times large ones: results are ordinary numbers, and as near as of ordinary operands.

Tolerance: k products added in any order, each within a whole step of fp32 of itself and of a partial sum: 2 (k + 4) U times the sum of the magnitudes."""
import pytest
import torch

from test_gpu_worker import U, gen

pytestmark = pytest.mark.gpu


# one token, few, tiles of 64, large tiles with rows and columns behind the last whole one, and such ones with sums of three products, whose bounds are narrow: of a row, of its gradient, of the weight's
@pytest.mark.parametrize("n, inner, outer", [(1, 64, 128), (9, 300, 70), (70, 65, 33), (1500, 130, 2200), (2100, 1030, 1300), (1500, 3, 2200), (1500, 2200, 3), (3, 1500, 2200)])
@pytest.mark.parametrize("power", [-100, -109, -112, -116, -120, -126, -132, -142])
def test_small_operands_count(power, n, inner, outer):
    import paper_2605_01989_amd as dblp
    g = gen(-power)

    def small(r, c):
        return (torch.randn(r, c, generator=g, device="cuda").double() * 2.0 ** power).float()

    def large(r, c):
        return (torch.randn(r, c, generator=g, device="cuda").double() * 2.0 ** -(power + 4)).clamp(-2.0 ** 127, 2.0 ** 127).float()

    def near(got, a, b):
        a, b = a.double(), b.double()
        off, most = (got.double() - a @ b).abs(), 2 * (a.shape[1] + 4) * U * (a.abs() @ b.abs())
        assert bool((off <= most).all()), float((off / most).max())
    ws = torch.full((dblp.linear_workspace(n, inner, outer),), 255, dtype=torch.uint8, device="cuda")
    y, dx, dw, db = (torch.empty(*s, device="cuda") for s in ((n, outer), (n, inner), (outer, inner), (outer,)))
    for first, second in ((small, large), (large, small)):
        x, w = first(n, inner), second(outer, inner)
        dblp.linear(x, w, y, ws)
        near(y, x, w.T)
        dy = first(n, outer)
        w = second(outer, inner)
        dblp.linear_grad_input(dy, w, dx, ws)
        near(dx, dy, w)
        x = second(n, inner)
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        near(dw, dy.T, x)
    # one value among ordinary ones
    x, w = torch.zeros(n, inner, device="cuda"), torch.randn(outer, inner, generator=g, device="cuda")
    x[n - 1, inner - 1] = 1.7 * 2.0 ** power
    w[:, inner - 1] *= 2.0 ** 60
    dblp.linear(x, w, y, ws)
    near(y, x, w.T)


@pytest.mark.parametrize("n, inner, outer", [(1000, 2002, 1001), (700, 1901, 2102), (1500, 203, 2203)])
def test_what_lies_behind_rows_changes_no_bit(n, inner, outer):
    """Values near and below the normal numbers between an operand's rows: results are made as with zeros there."""
    import paper_2605_01989_amd as dblp
    g = gen(n)
    ws = torch.empty(dblp.linear_workspace(n, inner, outer), dtype=torch.uint8, device="cuda")
    values = [torch.randn(*s, generator=g, device="cuda") for s in ((n, inner), (outer, inner), (n, outer))]
    got = []
    for scale in (0.0, 2.0 ** -120, 2.0 ** -140):
        x, w, dy = ((torch.randn(v.shape[0], v.shape[1] + 5, generator=g, device="cuda").double() * scale).float()[:, :v.shape[1]].copy_(v) for v in values)
        y, dx, dw, db = (torch.empty(*s, device="cuda") for s in ((n, outer), (n, inner), (outer, inner), (outer,)))
        dblp.linear(x, w, y, ws)
        dblp.linear_grad_input(dy, w, dx, ws)
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        got.append((y, dx, dw, db))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
