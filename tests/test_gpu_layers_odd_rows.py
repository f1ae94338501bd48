"""GPU: products of operands whose rows lie at odd places.  Operands are whole numbers of at most 8, so that products and sums are exact in fp32 (4097 x 64 < 2^24) in
any order: results have to be equal to the definition's in 64 bits, with no tolerance."""
import pytest
import torch

from test_gpu_worker import gen

pytestmark = pytest.mark.gpu


def whole(g, rows, cols, t, stride, shift):
    """Whole numbers, rows `stride` apart from `shift` elements past a 16-byte border, NaN around them."""
    buf = torch.full((shift + rows * stride + 8,), float("nan"), dtype=t, device="cuda")
    m = buf[shift:].as_strided((rows, cols), (stride, 1))
    return m.copy_(torch.randint(-8, 9, (rows, cols), generator=g, device="cuda"))


# sums of whole stages (64 k) and of one k less and more; of one part and of several; one row, few, more than a tile; widths whose rows are even and odd
SIZES = [(n, inner, outer) for n in (1, 2, 300) for inner in (256, 131) for outer in (1, 63, 64, 65, 128, 320, 1024, 4096)] + [(8192, 768, 1024), (8192, 1024, 4096), (8191, 768, 1023), (40, 64, 4096)]


@pytest.mark.parametrize("n, inner, outer", SIZES)
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_every_term_counts(t, n, inner, outer):
    import paper_2605_01989_amd as dblp
    g = gen(n + inner + outer)
    ws = torch.full((dblp.linear_workspace(n, inner, outer),), 255, dtype=torch.uint8, device="cuda")
    odd, even = outer + 1 + outer % 2, outer + outer % 2
    w_even, w_odd = inner + inner % 2, inner + 1 + inner % 2
    for stride, shift in ((odd, 0), (even, 1), (odd, 1), (odd, 3), (even, 0)):
        dy = whole(g, n, outer, t, stride, shift)
        for w_stride, w_shift in ((w_even, 0), (w_even, 1), (w_odd, 0)):
            w = whole(g, outer, inner, t, w_stride, w_shift)
            want = dy.double() @ w.double()
            dx = torch.full((n, inner), 5.0, device="cuda")
            dblp.linear_grad_input(dy, w, dx, ws)
            assert torch.equal(dx.double(), want), (stride, shift, w_stride, w_shift, (dx.double() != want).nonzero()[:4].tolist())
            base = torch.randint(-8, 9, (n, inner), generator=g, device="cuda").float()
            dblp.linear_grad_input(dy, w, dx, ws, base=base)
            assert torch.equal(dx.double(), want + base.double())
            narrow = torch.empty(n, inner, dtype=t, device="cuda")
            dblp.linear_grad_input(dy, w, narrow, ws)
            assert torch.equal(narrow, want.float().to(t))


@pytest.mark.parametrize("n, inner, outer", [(1, 64, 70), (5, 1024, 65), (16, 4096, 300), (300, 64, 131), (300, 65, 256), (1024, 320, 129), (64, 300, 131), (4096, 64, 67), (1023, 768, 1025), (2048, 1025, 640)])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
def test_every_term_of_the_other_products_counts(t, n, inner, outer):
    """Forward, and the weight's and the bias' gradients, whose sums are over the input's width and over the tokens."""
    import paper_2605_01989_amd as dblp
    g = gen(n + inner + outer)
    ws = torch.full((dblp.linear_workspace(n, inner, outer),), 255, dtype=torch.uint8, device="cuda")
    for shift, pad in ((0, 0), (1, 1), (1, 0), (2, 2), (3, 1), (0, 5)):
        x, w, dy = (whole(g, r, c, t, c + pad, shift) for r, c in ((n, inner), (outer, inner), (n, outer)))
        y, dw, db = (torch.full(s, 5.0, device="cuda") for s in ((n, outer), (outer, inner), (outer,)))
        dblp.linear(x, w, y, ws)
        assert torch.equal(y.double(), x.double() @ w.double().T), (shift, pad)
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        assert torch.equal(dw.double(), dy.double().T @ x.double()) and torch.equal(db.double(), dy.double().sum(0)), (shift, pad)
