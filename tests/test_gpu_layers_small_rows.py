"""GPU: orthogonalize of matrices some of whose rows, or columns, are far below the rest: each is as near, by its own size, as the rest."""
import pytest
import torch

import layer_reference as ref
from test_gpu_worker import U, gen

pytestmark = pytest.mark.gpu

HELD = 2.0 ** -22                # of X, A and a + b A + c A A, in relation to each value
LEAST = 2.0 ** -50               # ... or to the largest one possible


def by_rows(g, steps, coefficients=None):
    """(X, bound of each row's error) of a matrix of at least as many columns as rows.

    The largest values possible are those of singular values at the ends that the steps take them to (|X| = 1 at first): `most` of X, most^2 of A, `high` of the polynomial.  With e_i the
    error of row x_i and |.| a row's norm: A_ij = x_i . x_j moves by e_i |x_j| + |x_i| e_j; a sum of n products, of magnitudes that add up to s, is off by 8 sqrt(n) U s; what is stored by HELD of
    itself and LEAST of the largest."""
    x = g.double()
    x = x / x.norm()
    r, n = x.shape
    size = lambda m: m.norm(dim=1)  # noqa: E731
    most, e = 1.0, HELD * size(x) + LEAST * n ** 0.5
    for i in range(steps):
        a, b, c = coefficients[i] if coefficients else ref.COEFFICIENTS
        top = torch.linspace(0, most, 4001, dtype=torch.float64)
        high = float((a + b * top ** 2 + c * top ** 4).abs().max()) * 1.01
        rows, gram = size(x), x @ x.T
        poly = b * gram + c * gram @ gram + a * torch.eye(r, dtype=torch.float64)
        both = rows[:, None] * rows[None]
        e_gram = e[:, None] * rows[None] + rows[:, None] * e[None] + (HELD + 8 * n ** 0.5 * U) * both + LEAST * most ** 2
        mag = abs(b) * gram.abs() + abs(c) * gram.abs() @ gram.abs() + abs(a) * torch.eye(r, dtype=torch.float64)
        e_poly = abs(b) * e_gram + abs(c) * (e_gram @ gram.abs() + gram.abs() @ e_gram + 8 * r ** 0.5 * U * both.diagonal().sum() * both) + (HELD + 4 * U) * mag + LEAST * high
        most = max(float((a * top + b * top ** 3 + c * top ** 5).abs().max()) * 1.01, 1e-3)
        e = poly.abs() @ e + e_poly @ rows + (HELD + 8 * r ** 0.5 * U) * (poly.abs() @ rows) + LEAST * most * n ** 0.5
        x = poly @ x
    return x, e


# small ones of one launch, long ones of few rows in pieces, tiles of 64, 128 and more, sums in parts
@pytest.mark.parametrize("count, rows, cols", [(1, 40, 64), (3, 90, 128), (2, 50, 1500), (300, 60, 200), (1, 100, 400), (1, 130, 200), (3, 300, 500), (1, 700, 900)])
@pytest.mark.parametrize("tall", [False, True])
def test_rows_far_below_the_rest(count, rows, cols, tall):
    import paper_2605_01989_amd as dblp
    g = gen(rows + cols)
    x = torch.randn(count, rows, cols, generator=g, device="cuda")
    x[:, ::3] *= 2.0 ** -24
    x[:, 1::3] *= 2.0 ** -12
    given = x.transpose(1, 2).contiguous() if tall else x
    out = torch.empty_like(given)
    ws = torch.full((dblp.orthogonalize_workspace(*given.shape),), 255, dtype=torch.uint8, device="cuda")
    for steps, table in ((0, None), (1, None), (3, [(1.5, -0.5, 0.0)] * 3)):
        dblp.orthogonalize(given, out, ws, steps=steps, coefficients=table)
        for i in {0, count - 1}:
            want, e = by_rows(x[i].cpu(), steps, table)
            got = (out[i].T if tall else out[i]).cpu().double()
            off = (got - want).norm(dim=1)
            assert bool((off <= e + 2 * U * want.norm(dim=1)).all()), (steps, i, float((off / e).max()), float((off / want.norm(dim=1)).max()))
            # the bounds say something: of each row and from far below its own size
            assert float((e / want.norm(dim=1)).max()) < 2.0 ** -10
