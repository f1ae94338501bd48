"""GPU: the layers' operators against their definitions in 64 bits.

Tolerances.  U = half a step of fp32, 2^-24; a result's own rounding to its type is `close`'s.
  a product        k products added in any order, an addition off by at most a whole step (2 U) of a partial sum, whatever way it is rounded:
                   2 (k + 4) U times the sum of the magnitudes (bias and base among them)
  an activation    moves by at most 1.2 times its argument's error (the largest slope of any of them is 1.13); its own: an exponential of w (or erfc, whose logarithm
                   moves by w times its argument's relative error) by 3 min(w, 104) U, past which it is zero, and ten roundings
  a slope          the same of the sum of its two terms' magnitudes
  orthogonalize    a bound carried through the steps (layer_reference.orthogonal)"""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_worker import TYPES, U, close, gen, matrix, same, untouched

pytestmark = pytest.mark.gpu

ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]


def space(n):
    return torch.randint(0, 256, (max(n, 1),), dtype=torch.uint8, device="cuda")


def d(t):
    return None if t is None else t.cpu().double()


def act_slack(y, w, p):
    """Of results of magnitude y whose gate is p: a gate below fp32's normal numbers, 2^-126 (2^-125 with its own error), may be taken as zero, and what it
    is a factor of is lost with it."""
    return torch.where(p.abs() < 2.0 ** -125, y.abs(), (10 + 3 * w.clamp(max=104.0)) * U * y.abs())


# tokens, in, out, padding of the rows, shift: none of one, one of each, odd ones, whole tiles and one more, many k
SHAPES = [(0, 5, 7, 0, 0), (3, 0, 5, 0, 0), (4, 6, 0, 0, 0), (1, 1, 1, 0, 0), (1, 64, 128, 0, 0), (1, 333, 70, 0, 0), (2, 7, 3, 0, 1), (5, 8, 64, 8, 0), (16, 256, 48, 0, 0),
          (17, 40, 129, 3, 2), (33, 130, 65, 0, 0), (64, 64, 64, 0, 0), (100, 333, 61, 1, 1), (129, 200, 257, 0, 0), (300, 1000, 40, 0, 0), (257, 65, 260, 7, 3),
          (100, 66, 130, 2, 2), (70, 70, 68, 0, 2), (90, 129, 67, 4, 1), (20, 190, 30, 2, 6)]


@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("t", TYPES)
def test_linear(t, out):
    import paper_2605_01989_amd as dblp
    if t == out:
        return
    t = TYPES[t]
    o = t if out == "same" else torch.float32
    for k, (n, inner, outer, pad, shift) in enumerate(SHAPES):
        for act in ACTS if k % 3 == 0 else [ACTS[k % 5]]:
            g = gen(100 * k)
            x, w = matrix(g, n, inner, t, inner + pad, shift)[1], matrix(g, outer, inner, t, inner + 2 * pad, shift)[1]
            bias = torch.randn(outer, generator=g, device="cuda").to((torch.float32, t)[k % 2]) if k % 4 else None
            r = matrix(g, n, outer, o, outer + pad, shift)[1] if k % 3 else None
            by, y = matrix(g, n, outer, o, outer + pad, shift, fill=5.0)
            bz, z = matrix(g, n, outer, o, outer, shift, fill=5.0)
            keep = k % 2 == 0
            dblp.linear(x, w, y, space(dblp.linear_workspace(n, inner, outer)), bias=bias, activation=act, residual=r, pre=z if keep else None)
            want, mag = d(x) @ d(w).T, d(x).abs() @ d(w).abs().T
            if bias is not None:
                want, mag = want + d(bias), mag + d(bias).abs()
            slack = 2 * (inner + 4) * U * mag
            if keep:
                close(z, want, slack, o)
            a, p, _, size = ref.parts(act, want)
            total = a + d(r) if r is not None else a
            close(y, total, 1.2 * slack + act_slack(a, size, p) + U * total.abs(), o)
            assert untouched(by, y) and untouched(bz, z)


@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("t", TYPES)
def test_linear_grad_input(t, out):
    import paper_2605_01989_amd as dblp
    if t == out:
        return
    t = TYPES[t]
    o = t if out == "same" else torch.float32
    for k, (n, inner, outer, pad, shift) in enumerate(SHAPES):
        act = ACTS[k % 5]
        g = gen(200 * k)
        dy, w = matrix(g, n, outer, t, outer + pad, shift)[1], matrix(g, outer, inner, t, inner + 2 * pad, shift)[1]
        z = matrix(g, n, inner, o, inner + pad, shift)[1] if act or k % 2 else None
        base = matrix(g, n, inner, o, inner, 0)[1] if k % 3 else None
        buf, dx = matrix(g, n, inner, o, inner + pad, shift, fill=5.0)
        dblp.linear_grad_input(dy, w, dx, space(dblp.linear_workspace(n, inner, outer)), pre=z, activation=act, base=base)
        want, mag = d(dy) @ d(w), d(dy).abs() @ d(w).abs()
        slack = 2 * (outer + 4) * U * mag
        if z is not None:
            _, p, q, size = ref.parts(act, d(z))
            slack = 1.2 * slack + act_slack(want * (p.abs() + q.abs()), size, p)
            want = want * (p + q)
        if base is not None:
            want = want + d(base)
        close(dx, want, slack + U * want.abs(), o)
        assert untouched(buf, dx)


@pytest.mark.parametrize("t", TYPES)
def test_linear_grad_weight(t):
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    for k, (outer, inner, n, pad, shift) in enumerate(SHAPES + [(40, 24, 3000, 0, 0), (64, 128, 10000, 0, 0), (33, 65, 5003, 1, 1)]):
        g = gen(300 * k)
        dy, x = matrix(g, n, outer, t, outer + pad, shift)[1], matrix(g, n, inner, t, inner + 2 * pad, shift)[1]
        base = matrix(g, outer, inner, torch.float32, inner + pad, 0)[1] if k % 2 else None
        buf, dw = matrix(g, outer, inner, torch.float32, inner + pad, shift, fill=5.0)
        db = torch.full((outer,), 5.0, device="cuda") if k % 3 else None
        bias_base = torch.randn(outer, generator=g, device="cuda") if k % 6 == 1 else None
        dblp.linear_grad_weight(dy, x, dw, space(dblp.linear_workspace(n, inner, outer)), base=base, bias_grad=db, bias_base=bias_base)
        want, mag = d(dy).T @ d(x), d(dy).abs().T @ d(x).abs()
        if base is not None:
            want, mag = want + d(base), mag + d(base).abs()
        close(dw, want, 2 * (n + 4) * U * mag, torch.float32)
        if db is not None:
            want, mag = d(dy).sum(0), d(dy).abs().sum(0)
            if bias_base is not None:
                want, mag = want + d(bias_base), mag + d(bias_base).abs()
            close(db, want, 2 * (n + 4) * U * mag, torch.float32)
        assert untouched(buf, dw)


def big(t):
    return t.double()


# tokens, in, out, padding: whole large tiles, ragged ones on aligned rows, odd rows, sums in many parts, sums that end inside a chunk
LARGE = [(4096, 128, 4096, 0), (3333, 200, 4600, 0), (4000, 77, 4099, 3), (4099, 65, 4000, 0), (700, 5000, 800, 0), (129, 9001, 130, 7), (2050, 100, 9000, 1), (260, 3000, 50257, 0),
         (1, 4096, 4096, 0), (1, 20000, 70, 0), (7, 9001, 50, 5), (16, 1000, 5003, 0), (17, 3001, 900, 0), (32, 512, 4097, 3), (33, 16384, 33, 0), (64, 2049, 1030, 1), (65, 2049, 1030, 1)]


@pytest.mark.parametrize("n, inner, outer, pad", LARGE)
@pytest.mark.parametrize("t", TYPES)
def test_large_products(t, n, inner, outer, pad):
    """The same bounds, the definition computed on the GPU in 64 bits.  Fp32 sums of `depth` products in any order."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    g = gen(n + inner)

    def near(got, want, mag, depth, o):
        got, half = big(got), torch.finfo(o).eps / 2
        tol = half * want.abs() * (1 + half) + 2 * (depth + 4) * U * mag + 2.0 ** -25 * (o == torch.float16)
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])
    rand = lambda r, c, to=t: torch.randn(r, c + pad, generator=g, device="cuda").to(to)[:, :c]  # noqa: E731
    x, w, dy = rand(n, inner), rand(outer, inner), rand(n, outer)
    ws = space(dblp.linear_workspace(n, inner, outer))
    bias, r = torch.randn(outer, generator=g, device="cuda"), rand(n, outer)
    y, z = torch.empty(n, outer, dtype=t, device="cuda"), torch.empty(n, outer, dtype=t, device="cuda")
    dblp.linear(x, w, y, ws, bias=bias, activation="relu", residual=r, pre=z)
    want, mag = big(x) @ big(w).T + big(bias), big(x).abs() @ big(w).abs().T + big(bias).abs()
    near(z, want, mag, inner, t)
    near(y, want.clamp(min=0) + big(r), mag + big(r).abs(), inner, t)
    dx, base, pre = torch.empty(n, inner, dtype=t, device="cuda"), rand(n, inner), rand(n, inner)
    dblp.linear_grad_input(dy, w, dx, ws, pre=pre, activation="relu", base=base)
    on = (pre > 0).double()
    near(dx, (big(dy) @ big(w)) * on + big(base), (big(dy).abs() @ big(w).abs()) * on + big(base).abs(), outer, t)
    dw, db = torch.empty(outer, inner, device="cuda"), torch.empty(outer, device="cuda")
    dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
    near(dw, big(dy).T @ big(x), big(dy).abs().T @ big(x).abs(), n, torch.float32)
    near(db, big(dy).sum(0), big(dy).abs().sum(0), n, torch.float32)
    again, again_b = torch.empty_like(dw), torch.empty_like(db)
    ws.fill_(255)
    dblp.linear_grad_weight(dy, x, again, ws, bias_grad=again_b)
    assert torch.equal(again, dw) and torch.equal(again_b, db)


def test_a_weight_without_columns_has_a_bias():
    import paper_2605_01989_amd as dblp
    dy = torch.randn(300, 70, generator=gen(1), device="cuda")
    db, ws = torch.empty(70, device="cuda"), space(dblp.linear_workspace(300, 0, 70))
    dblp.linear_grad_weight(dy, torch.empty(300, 0, device="cuda"), torch.empty(70, 0, device="cuda"), ws, bias_grad=db)
    close(db, d(dy).sum(0), 2 * 304 * U * d(dy).abs().sum(0), torch.float32)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t", TYPES)
def test_activation_grad(t, act):
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    for k, (rows, cols, pad, shift) in enumerate([(0, 8, 0, 0), (3, 0, 0, 0), (1, 1, 0, 0), (3, 7, 0, 1), (5, 8, 0, 0), (4, 13, 3, 2), (70, 257, 0, 0), (33, 768, 0, 0), (9, 1000, 8, 0)]):
        g = gen(17 * k)
        dy, z = matrix(g, rows, cols, t, cols + pad, shift)[1], matrix(g, rows, cols, t, cols + 2 * pad, shift)[1]
        z.mul_(4)
        if rows * cols > 20:
            z[0, 0], z[1, 1], z[2, 2], z[0, 1], z[1, 2] = 60.0, -60.0, 1e4, -1e4, 0.0
            if t != torch.float16:
                z[2, 0], z[2, 1] = 1e25, -1e25
        buf, dz = matrix(g, rows, cols, t, cols + 2 * pad, shift, fill=5.0)
        dblp.activation_grad(dy, z, dz, act)
        _, p, q, size = ref.parts(act, d(z))
        close(dz, d(dy) * (p + q), act_slack(d(dy) * (p.abs() + q.abs()), size, p), t)
        assert untouched(buf, dz)
        for over in (dy, z):                       # in place
            before = over.clone()
            dblp.activation_grad(dy, z, over, act)
            assert same(over, dz)
            over.copy_(before)


def test_activations_at_their_ends():
    """Far from zero an activation is its argument or zero and its slope one or zero; NaN stays NaN."""
    import paper_2605_01989_amd as dblp
    z = torch.tensor([[1e30, 200.0, -200.0, -1e30, float("nan"), 0.0, 3e38, -3e38]], device="cuda")
    one, y, ws = torch.eye(8, device="cuda"), torch.empty(1, 8, device="cuda"), space(dblp.linear_workspace(1, 8, 8))
    ones = torch.ones_like(z)
    for act in ACTS[1:]:
        # through the bias, the other operand being zeros: a product with NaN is NaN everywhere
        dblp.linear(torch.zeros(1, 8, device="cuda"), one, y, ws, bias=z[0], activation=act)
        want = torch.where(z > 0, z, 0.0)
        assert same(y, torch.where(torch.isnan(z), z, want)), (act, y)
        dblp.activation_grad(ones, z, y, act)
        slope = torch.where(z > 0, 1.0, 0.0)
        slope[0, 5] = 0.0 if act == "relu" else 0.5
        assert same(y, slope if act == "relu" else torch.where(torch.isnan(z), z, slope)), (act, y)


def test_infinities_stay_in_their_row():
    """A value that is not finite reaches the results that are made of it and no others, in partial tiles too."""
    import paper_2605_01989_amd as dblp
    for n, inner, outer in ((5, 37, 19), (70, 100, 130)):
        for t in TYPES.values():
            g = gen(n)
            x, w = torch.randn(n, inner, generator=g, device="cuda").to(t), torch.randn(outer, inner, generator=g, device="cuda").to(t)
            ws = space(dblp.linear_workspace(n, inner, outer))
            y = torch.empty(n, outer, dtype=t, device="cuda")
            clean = torch.empty_like(y)
            dblp.linear(x, w, clean, ws)
            x[2, inner - 1], w[3, 0] = float("nan"), float("inf")
            dblp.linear(x, w, y, ws)
            hit = torch.zeros(n, outer, dtype=torch.bool, device="cuda")
            hit[2], hit[:, 3] = True, True
            assert torch.equal(y[~hit], clean[~hit]) and not torch.isfinite(y[hit]).any()


@pytest.mark.parametrize("n,inner,outer", [(40, 30, 61), (300, 70, 200), (9000, 100, 130), (1000, 2000, 1001), (700, 1900, 2100), (2500, 4000, 4003)])
def test_what_is_not_finite_stays_in_its_sum(n, inner, outer):
    """A bias' gradient is of its own column: not of its neighbours', and not of what lies behind a row's end."""
    import paper_2605_01989_amd as dblp
    for t in TYPES.values():
        g = gen(outer)
        buf = torch.full((n, outer + 13), float("nan"), dtype=t, device="cuda")
        dy, x = buf[:, :outer], torch.randn(n, inner, generator=g, device="cuda").to(t)
        dy.copy_(torch.randn(n, outer, generator=g, device="cuda"))
        clean = torch.zeros(n, outer + 13, dtype=t, device="cuda")[:, :outer]
        clean.copy_(dy)
        ws = space(dblp.linear_workspace(n, inner, outer))
        dw, want = torch.empty(outer, inner, device="cuda"), torch.empty(outer, inner, device="cuda")
        db, sums = torch.empty(outer, device="cuda"), torch.empty(outer, device="cuda")
        dblp.linear_grad_weight(clean, x, want, ws, bias_grad=sums)
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        assert torch.equal(db, sums) and torch.equal(dw, want)
        off = (d(db) - d(dy).sum(0)).abs()
        assert bool((off <= 2 * (n + 4) * U * d(dy).abs().sum(0)).all())
        dy[n // 2, 17], dy[n - 1, outer - 2] = float("inf"), float("nan")
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        rest = torch.ones(outer, dtype=torch.bool, device="cuda")
        rest[17] = rest[outer - 2] = False
        assert torch.equal(db[rest], sums[rest]) and float(db[17]) == math.inf and math.isnan(float(db[outer - 2]))
        if t != torch.float32:
            assert torch.equal(dw[rest], want[rest])
        else:                                      # a large tile of floats that holds such a value is made by other instructions: as near, not the same bits
            keep = rest.cpu()
            mine, other = d(dy).T[keep], d(x)
            assert bool(((d(dw)[keep] - mine @ other).abs() <= 2 * (n + 4) * U * (mine.abs() @ other.abs())).all())


def test_in_place():
    import paper_2605_01989_amd as dblp
    g = gen(5)
    n, inner, outer = 70, 90, 101
    for t in TYPES.values():
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
        x, w, r, dy, z = rand(n, inner), rand(outer, inner), rand(n, outer), rand(n, outer), rand(n, inner)
        ws = space(dblp.linear_workspace(n, inner, outer))
        y, over = torch.empty_like(r), r.clone()
        dblp.linear(x, w, y, ws, activation="gelu", residual=r)
        dblp.linear(x, w, over, ws, activation="gelu", residual=over)
        assert torch.equal(y, over)
        dx, base = torch.empty_like(x), rand(n, inner)
        dblp.linear_grad_input(dy, w, dx, ws, pre=z, activation="silu", base=base)
        over_z, over_b = z.clone(), base.clone()
        dblp.linear_grad_input(dy, w, over_z, ws, pre=over_z, activation="silu", base=base)
        dblp.linear_grad_input(dy, w, over_b, ws, pre=z, activation="silu", base=over_b)
        assert torch.equal(dx, over_z) and torch.equal(dx, over_b)
        dw, db = torch.randn(outer, inner, generator=g, device="cuda"), torch.randn(outer, generator=g, device="cuda")
        want, want_b = torch.empty_like(dw), torch.empty_like(db)
        dblp.linear_grad_weight(dy, x, want, ws, base=dw, bias_grad=want_b, bias_base=db)
        dblp.linear_grad_weight(dy, x, dw, ws, base=dw, bias_grad=db, bias_base=db)
        assert torch.equal(dw, want) and torch.equal(db, want_b)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_two_layers(act):
    """y = act(x W1' + b1) W2' + b2 + x: the operators' way back in fp32 against autograd in 64 bits and against differences of the operators' own loss."""
    import paper_2605_01989_amd as dblp
    n, dim, wide = 21, 30, 70
    g = gen(8)
    x, w1, w2 = (torch.randn(*s, generator=g, device="cuda") * 0.5 for s in ((n, dim), (wide, dim), (dim, wide)))
    b1, b2, dy = torch.randn(wide, generator=g, device="cuda"), torch.randn(dim, generator=g, device="cuda"), torch.randn(n, dim, generator=g, device="cuda")
    ws = space(dblp.linear_workspace(n, dim, wide))

    def forward(x, w1, b1, w2, b2):
        z, h, y = torch.empty(n, wide, device="cuda"), torch.empty(n, wide, device="cuda"), torch.empty(n, dim, device="cuda")
        dblp.linear(x, w1, h, ws, bias=b1, activation=act, pre=z)
        dblp.linear(h, w2, y, ws, bias=b2, residual=x)
        return z, h, y
    z, h, y = forward(x, w1, b1, w2, b2)
    dz, dx = torch.empty_like(z), torch.empty_like(x)
    dw1, dw2, db1, db2 = (torch.empty_like(v) for v in (w1, w2, b1, b2))
    dblp.linear_grad_weight(dy, h, dw2, ws, bias_grad=db2)
    dblp.linear_grad_input(dy, w2, dz, ws, pre=z, activation=act)
    dblp.linear_grad_weight(dz, x, dw1, ws, bias_grad=db1)
    dblp.linear_grad_input(dz, w1, dx, ws, base=dy)
    p = [d(v).requires_grad_(True) for v in (x, w1, b1, w2, b2)]
    yy = ref.parts(act, p[0] @ p[1].T + p[2])[0] @ p[3].T + p[4] + p[0]
    (yy * d(dy)).sum().backward()
    for got, v in zip((dx, dw1, db1, dw2, db2), p):
        # eight products in a row at most, of up to `wide` terms of magnitudes below 64 times the largest gradient
        assert float((d(got) - v.grad).abs().max()) <= 8 * 2 * (wide + 4) * U * 64 * float(v.grad.abs().max())
    if act != "relu":                            # (whose slope jumps)
        for i, got in enumerate((dx, dw1, db1, dw2, db2)):
            args = [x, w1, b1, w2, b2]
            way = torch.randn(args[i].shape, generator=g, device="cuda")
            way, step = way / way.norm(), 2.0 ** -4
            ends = []
            for sign in (1, -1):
                moved = list(args)
                moved[i] = args[i] + sign * step * way
                ends.append((d(forward(*moved)[2]) * d(dy)).sum())
            slope, want = float((ends[0] - ends[1]) / (2 * step)), float((d(got) * d(way)).sum())
            # an activation's third derivative is below one: step^2 / 6 times the cube of what z moves by, weighed by its gradient; roundings: of the
            # loss' terms, each a product of a product, and of the moved argument, over the step
            moves = (lambda: d(way) @ d(w1).T, lambda: d(x) @ d(way).T, lambda: d(way).expand(n, wide), lambda: torch.zeros(1), lambda: torch.zeros(1))[i]()
            mag = float((((d(h).abs() @ d(w2).abs().T) + d(b2).abs() + d(x).abs()) * d(dy).abs()).sum())
            curve = step ** 2 / 6 * float((d(dy) @ d(w2)).abs().max()) * float((moves.abs() ** 3).sum())
            assert abs(slope - want) <= curve + (2 * 2 * (wide + dim + 8) * U * mag) / step


ORTHOGONAL = [(1, 1, 1), (1, 1, 5), (1, 7, 1), (2, 3, 4), (1, 16, 16), (3, 17, 40), (2, 40, 17), (1, 64, 64), (1, 128, 128), (2, 100, 128), (1, 130, 65), (1, 65, 300), (2, 129, 257), (1, 300, 200), (3, 64, 6016), (2, 4100, 70), (1, 10, 20001), (1, 600, 513)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("out", TYPES)
def test_orthogonalize(t, out):
    import paper_2605_01989_amd as dblp
    t, o = TYPES[t], TYPES[out]
    for k, (count, rows, cols) in enumerate(ORTHOGONAL):
        g = gen(400 * k)
        stack = torch.randn(count, rows, cols + k % 3, generator=g, device="cuda").mul_(10.0 ** (k % 5 - 2)).to(t)[:, :, :cols]
        if k % 2:                                  # a steep spectrum
            stack = (stack.float() * torch.logspace(0, -3, cols, device="cuda")).to(t)
        base = torch.randn(count, rows, cols, generator=g, device="cuda").to(o) if k % 3 else None
        buf = torch.full((count, rows, cols + 5), -77.0, dtype=o, device="cuda")
        got = buf[:, :, :cols]
        steps = (5, 1, 3, 0, 5)[k % 5]
        dblp.orthogonalize(stack, got, space(dblp.orthogonalize_workspace(count, rows, cols)), scale=-0.5, base=base, base_scale=0.75, steps=steps)
        for i in range(count):
            x, e = ref.orthogonal(d(stack[i]), steps)
            want = -0.5 * x + (0.75 * d(base[i]) if base is not None else 0.0)
            off = d(got[i]) - want
            # the error of X, two more fp32 roundings, the type's
            most = 0.5 * e + 4 * U * float(want.norm() + x.norm()) + torch.finfo(o).eps / 2 * float(want.norm())
            assert bool(torch.isfinite(off).all()) and float(off.norm()) <= most, (count, rows, cols, float(off.norm()), most)
        assert bool((buf[:, :, cols:] == -77.0).all())


def test_orthogonalize_makes_singular_values_alike():
    """From a spread of 100 the library's steps take all to 0.68 to 1.21: the polynomial's values there, an error below the carried bound apart."""
    import paper_2605_01989_amd as dblp
    g = gen(6)
    for rows, cols in ((128, 128), (96, 400), (250, 90)):
        r = min(rows, cols)
        u, v = (torch.linalg.qr(torch.randn(m, r, generator=g, device="cuda"))[0] for m in (rows, cols))
        spectrum = torch.linspace(1, 0.3, r, device="cuda")
        got = torch.empty(rows, cols, device="cuda")
        dblp.orthogonalize((u * spectrum) @ v.T, got, space(dblp.orthogonalize_workspace(1, rows, cols)))
        s = torch.linalg.svdvals(d(got))
        assert 0.67 < float(s.min()) and float(s.max()) < 1.22
        assert float((d(u).T @ d(got) @ d(v) - torch.eye(r, dtype=torch.float64)).abs().max()) < 0.34


def test_orthogonalize_of_many_matrices():
    """More of them than a grid's third dimension holds, small ones of one launch and others."""
    import paper_2605_01989_amd as dblp
    g = gen(13)
    for count, rows, cols in ((70000, 3, 4), (33000, 2, 129)):
        x = torch.randn(count, rows, cols, generator=g, device="cuda")
        out = torch.empty_like(x)
        dblp.orthogonalize(x, out, space(dblp.orthogonalize_workspace(count, rows, cols)))
        for i in (0, 1, 32767, 32768, count - 1):
            want, e = ref.orthogonal(d(x[i]), 5)
            assert float((d(out[i]) - want).norm()) <= e + 4 * U * float(want.norm()), (count, i)
        assert bool(torch.isfinite(out).all())


def test_orthogonalize_of_zeros_and_what_is_not_finite():
    import paper_2605_01989_amd as dblp
    g = gen(2)
    x = torch.randn(5, 70, 90, generator=g, device="cuda")
    x[1] = 0.0
    x[2, 3, 4] = float("inf")
    x[3, 0, 0] = float("nan")
    x[4] *= 1e-38                                  # its squares leave fp32, some of its values the normal numbers
    base = torch.randn(5, 70, 90, generator=g, device="cuda")
    out = torch.empty_like(x)
    for steps in (0, 2, 5):
        dblp.orthogonalize(x, out, space(dblp.orthogonalize_workspace(5, 70, 90)), base=base, base_scale=2.0, steps=steps)
        assert torch.equal(out[1], 2.0 * base[1])
        assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all()
        for i in (0, 4):
            want, e = ref.orthogonal(d(x[i]), steps)
            assert float((d(out[i]) - want - 2.0 * d(base[i])).norm()) <= e + 4 * U * float(2 * base[i].norm() + want.norm())


@pytest.mark.parametrize("n,inner,outer", [(1100, 1301, 1203), (2200, 333, 1601), (4099, 65, 2051), (90, 4001, 903)])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_odd_rows_give_what_even_ones_give(t, n, inner, outer):
    """Values at odd addresses and strides, NaN all around them and in the workspace, bit for bit as from rows at multiples of 16 bytes (the input's
    gradient, whose sum begins one k earlier in odd rows, where dy's are even)."""
    import paper_2605_01989_amd as dblp
    g = gen(n)

    def both(rows, cols):
        values = torch.randn(rows, cols, generator=g, device="cuda").to(t)
        got = []
        for stride, shift in ((cols + cols % 2 + 1, 1), ((cols + 7) // 8 * 8, 0)):
            buf = torch.full((rows * stride + 8 + shift,), float("nan"), dtype=t, device="cuda")
            got.append(buf[shift:shift + rows * stride].view(rows, stride)[:, :cols])
            got[-1].copy_(values)
        return got

    x, w, dy = both(n, inner), both(outer, inner), both(n, outer)
    bias = torch.randn(outer, generator=g, device="cuda")
    ws = torch.full((dblp.linear_workspace(n, inner, outer),), 255, dtype=torch.uint8, device="cuda")
    got = []
    for k in (0, 1):
        y, dx, dw, db = (torch.full(size, -77.0, device="cuda") for size in ((n, outer), (n, inner), (outer, inner), (outer,)))
        dblp.linear(x[k], w[k], y, ws, bias=bias, activation="relu")
        dblp.linear_grad_input(dy[1], w[k], dx, ws)
        dblp.linear_grad_weight(dy[k], x[k], dw, ws, bias_grad=db)
        again = torch.empty_like(dw)
        ws.fill_(7 * k)
        dblp.linear_grad_weight(dy[k], x[1 - k], again, ws)
        got.append((y, dx, dw, db))
        assert torch.equal(again, dw)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    for k in (0, 1):
        dx = torch.empty(n, inner, device="cuda")
        dblp.linear_grad_input(dy[0], w[k], dx, ws)
        off = (d(dx) - d(dy[1]) @ d(w[1])).abs()
        assert bool((off <= 2 * (outer + 4) * U * (d(dy[1]).abs() @ d(w[1]).abs())).all())
    want = (d(dy[1]).T @ d(x[1]))
    off = (d(got[0][2]) - want).abs()
    assert bool((off <= 2 * (n + 4) * U * (d(dy[1]).abs().T @ d(x[1]).abs())).all())


@pytest.mark.parametrize("count,rows,cols", [(1, 90, 511), (4, 300, 128), (270, 9, 300), (270, 400, 100), (90, 65, 700), (1, 64, 8200), (40, 1100, 33)])
def test_orthogonalize_of_long_ones(count, rows, cols):
    """Blocks of one piece and of some, of odd sizes and padded rows, with matrices of zeros and others that are not finite beside them, in place and not."""
    import paper_2605_01989_amd as dblp
    g = gen(rows)
    x = torch.randn(count, rows, cols, generator=g, device="cuda")
    bad = count > 2
    if bad:
        x[0] = 0.0
        x[1, rows - 1, cols - 1] = float("nan")
    ws = space(dblp.orthogonalize_workspace(count, rows, cols))
    for t in TYPES.values():
        buf = torch.full((count, rows, cols + 3), -77.0, dtype=t, device="cuda")
        stack, base = buf[:, :, :cols], torch.randn(count, rows, cols, generator=g, device="cuda")
        stack.copy_(x)
        start = stack.clone()
        got = torch.empty(count, rows, cols, device="cuda")
        dblp.orthogonalize(stack, got, ws, scale=-0.5, base=base, base_scale=0.75, steps=3)
        if bad:
            assert torch.equal(got[0], 0.75 * base[0]) and bool(torch.isnan(got[1]).all())
        for i in {0, 2 * bad, count // 2, count - 1} - {0, 1} if bad else range(count):
            o, e = ref.orthogonal(d(start[i]), 3)
            want = -0.5 * o + 0.75 * d(base[i])
            assert float((d(got[i]) - want).norm()) <= 0.5 * e + 4 * U * float(want.norm() + o.norm()), i
        apart = torch.empty(count, rows, cols, dtype=t, device="cuda")
        dblp.orthogonalize(stack, apart, ws, scale=0.3, base=start, steps=2)
        dblp.orthogonalize(stack, stack, ws, scale=0.3, base=stack, steps=2)
        assert torch.equal(torch.nan_to_num(stack, nan=5.0), torch.nan_to_num(apart, nan=5.0))
        assert bool((buf[:, :, cols:] == -77.0).all())


def test_orthogonalize_in_place_and_with_other_coefficients():
    import paper_2605_01989_amd as dblp
    g = gen(3)
    table = [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)]
    for rows, cols in ((60, 90), (90, 60), (200, 130)):
        x = torch.randn(2, rows, cols, generator=g, device="cuda")
        ws = space(dblp.orthogonalize_workspace(2, rows, cols))
        want = torch.empty_like(x)
        dblp.orthogonalize(x, want, ws, scale=0.3, base=x, base_scale=0.5, steps=3, coefficients=table)
        for i in range(2):
            o, e = ref.orthogonal(d(x[i]), 3, table)
            assert float((d(want[i]) - 0.3 * o - 0.5 * d(x[i])).norm()) <= 0.3 * e + 8 * U * float(x[i].norm())
        over = x.clone()
        dblp.orthogonalize(over, over, ws, scale=0.3, base=over, base_scale=0.5, steps=3, coefficients=table)
        assert torch.equal(over, want)
        base, twice = torch.ones_like(x), torch.ones_like(x)
        dblp.orthogonalize(x, want, ws, base=base)
        dblp.orthogonalize(x, twice, ws, base=twice, coefficients=ref.COEFFICIENTS)
        assert torch.equal(twice, want)


def test_the_same_bits_on_any_workspace_and_stream():
    import paper_2605_01989_amd as dblp
    g = gen(4)
    n, inner, outer = 1030, 130, 200
    side = torch.cuda.Stream()
    for t in TYPES.values():
        x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(t) for s in ((n, inner), (outer, inner), (n, outer)))
        m = torch.randn(2, inner, outer, generator=g, device="cuda")

        def go(fill):
            ws = torch.full((max(dblp.linear_workspace(n, inner, outer), dblp.orthogonalize_workspace(2, inner, outer)),), fill, dtype=torch.uint8, device="cuda")
            y, dx = torch.empty(n, outer, dtype=t, device="cuda"), torch.empty(n, inner, dtype=t, device="cuda")
            dw, db, o = torch.empty(outer, inner, device="cuda"), torch.empty(outer, device="cuda"), torch.empty_like(m)
            dblp.linear(x, w, y, ws, activation="gelu")
            dblp.linear_grad_input(dy, w, dx, ws)
            dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
            dblp.orthogonalize(m, o, ws)
            return y, dx, dw, db, o
        first = go(0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            second = go(255)                       # (NaN in every type)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_recorded_calls_give_what_eager_ones_give():
    """Two graphs that share one workspace, replayed in turn with eager calls between them."""
    import paper_2605_01989_amd as dblp
    g = gen(9)
    n, inner, outer = 200, 96, 136
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16) for s in ((n, inner), (outer, inner), (n, outer)))
    ws = space(max(dblp.linear_workspace(n, inner, outer), dblp.orthogonalize_workspace(1, outer, inner)))
    y, z, dx = (torch.empty(*s, dtype=torch.bfloat16, device="cuda") for s in ((n, outer), (n, outer), (n, inner)))
    dw, db, params = torch.empty(outer, inner, device="cuda"), torch.empty(outer, device="cuda"), torch.randn(outer, inner, generator=g, device="cuda")

    def forward():
        dblp.linear(x, w, y, ws, bias=db, activation="silu", pre=z)
        dblp.linear_grad_input(dy, w, dx, ws, pre=x, activation="silu")

    def back():
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        dblp.orthogonalize(dw, params, ws, scale=-0.1, base=params)
    db.zero_()
    graphs = []
    torch.cuda.synchronize()
    for f in (forward, back):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append(graph)
    start = params.clone()
    eager = []
    for i in range(3):
        x.copy_(torch.randn(n, inner, generator=gen(i), device="cuda"))
        forward(), back()
        eager.append([v.clone() for v in (y, z, dx, dw, db, params)])
    params.copy_(start)
    db.zero_()
    for i in range(3):
        x.copy_(torch.randn(n, inner, generator=gen(i), device="cuda"))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager[i], (y, z, dx, dw, db, params)))


def test_recorded_calls_of_odd_rows():
    """Two graphs with one workspace, in which each lays its operands out, replayed in turn on new values, with eager calls between them."""
    import paper_2605_01989_amd as dblp
    n, inner, outer = 1300, 1301, 1203
    g = gen(31)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(torch.float16) for s in ((n, inner), (outer, inner), (n, outer)))
    ws = space(max(dblp.linear_workspace(n, inner, outer), dblp.orthogonalize_workspace(9, 100, inner)))
    y, dx, dw, db = (torch.empty(*s, device="cuda") for s in ((n, outer), (n, inner), (outer, inner), (outer,)))
    rows = torch.empty(9, 100, inner, device="cuda")

    def forward():
        dblp.linear(x, w, y, ws, activation="gelu")
        dblp.linear_grad_input(dy, w, dx, ws)

    def back():
        dblp.linear_grad_weight(dy, x, dw, ws, bias_grad=db)
        dblp.orthogonalize(dw[:900].view(9, 100, inner), rows, ws, steps=2)
    graphs = []
    torch.cuda.synchronize()
    for f in (forward, back):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append(graph)
    for i in range(3):
        x.copy_(torch.randn(n, inner, generator=gen(i), device="cuda"))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        replayed = [v.clone() for v in (y, dx, dw, db, rows)]
        for v in (y, dx, dw, db, rows):
            v.fill_(-77.0)
        forward(), back()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (y, dx, dw, db, rows)))


def test_odd_rows_far_apart():
    import paper_2605_01989_amd as dblp
    n, inner, outer, far = 600, 701, 301, (1 << 22) + 1
    g = gen(8)
    t = torch.bfloat16
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(t) for s in ((n, inner), (outer, inner), (n, outer)))
    buf = torch.empty(n * far, dtype=t, device="cuda")
    ws = space(dblp.linear_workspace(n, inner, outer))
    y, dw, dx = (torch.empty(*s, device="cuda") for s in ((n, outer), (outer, inner), (n, inner)))
    fx = buf.as_strided((n, inner), (far, 1)).copy_(x)
    fdy = buf[4096:].as_strided((n, outer), (far, 1)).copy_(dy)
    dblp.linear(fx, w, y, ws)
    dblp.linear_grad_weight(fdy, fx, dw, ws)
    dblp.linear_grad_input(fdy, w, dx, ws)
    for got, a, b in ((y, d(x), d(w).T), (dw, d(dy).T, d(x)), (dx, d(dy), d(w))):
        assert bool(((d(got) - a @ b).abs() <= 2 * (a.shape[1] + 4) * U * (a.abs() @ b.abs())).all())


def test_offsets_past_32_bits():
    """Rows far enough apart that a row's place passes 2^32 elements."""
    import paper_2605_01989_amd as dblp
    n, inner, outer, far = 70, 40, 66, (1 << 26) + 8
    g = gen(7)
    t = torch.bfloat16
    buf = torch.empty(n * far, dtype=t, device="cuda")
    x, w = torch.randn(n, inner, generator=g, device="cuda").to(t), torch.randn(outer, inner, generator=g, device="cuda").to(t)
    dy = torch.randn(n, outer, generator=g, device="cuda").to(t)
    ws = space(dblp.linear_workspace(n, inner, outer))
    apart = lambda m, shift: buf[shift:].as_strided(m.shape, (far, 1)).copy_(m)  # noqa: E731
    fx, fdy = apart(x, 0), apart(dy, 1024)
    y, fy = torch.empty(n, outer, dtype=t, device="cuda"), apart(torch.zeros(n, outer, dtype=t, device="cuda"), 4096)
    dblp.linear(x, w, y, ws)
    dblp.linear(fx, w, fy, ws)
    assert torch.equal(fy, y)
    dw, fdw = torch.empty(outer, inner, device="cuda"), torch.empty(outer, inner, device="cuda")
    dblp.linear_grad_weight(dy, x, dw, ws)
    dblp.linear_grad_weight(fdy, fx, fdw, ws)
    assert torch.equal(dw, fdw)
    dx, fdx = torch.empty(n, inner, dtype=t, device="cuda"), torch.empty(n, inner, dtype=t, device="cuda")
    dblp.linear_grad_input(dy, w, dx, ws)
    dblp.linear_grad_input(fdy, w, fdx, ws)
    assert torch.equal(dx, fdx)


def test_rows_far_apart_within_a_tiles_reach():
    """Rows as far apart as a tile's offsets reach, where the wide kernels still take them, and one element farther, where they do not."""
    import paper_2605_01989_amd as dblp
    n, inner, outer = 600, 72, 80
    g = gen(21)
    buf = torch.empty(n * ((1 << 21) + 2), dtype=torch.bfloat16, device="cuda")
    for t, far in ((torch.bfloat16, (1 << 21) - 2), (torch.bfloat16, (1 << 21) - 1), (torch.bfloat16, 1 << 21), (torch.float32, (1 << 20) - 1), (torch.float32, 1 << 20)):
        x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(t) for s in ((n, inner), (outer, inner), (n, outer)))
        ws = space(dblp.linear_workspace(n, inner, outer))
        apart = lambda m: buf.view(t).as_strided(m.shape, (far, 1)).copy_(m)  # noqa: E731
        y, fy = torch.empty(n, outer, dtype=t, device="cuda"), torch.empty(n, outer, dtype=t, device="cuda")
        dblp.linear(x, w, y, ws)
        dblp.linear(apart(x), w, fy, ws)
        close(fy, d(x) @ d(w).T, 2 * (inner + 4) * U * (d(x).abs() @ d(w).abs().T), t)
        assert torch.equal(y, fy)
        dx, fdx = torch.empty(n, inner, dtype=t, device="cuda"), torch.empty(n, inner, dtype=t, device="cuda")
        dblp.linear_grad_input(dy, w, dx, ws)
        dblp.linear_grad_input(apart(dy), w, fdx, ws)
        for got in (dx, fdx):
            close(got, d(dy) @ d(w), 2 * (outer + 4) * U * (d(dy).abs() @ d(w).abs()), t)
        dw, fdw = torch.empty(outer, inner, device="cuda"), torch.empty(outer, inner, device="cuda")
        dblp.linear_grad_weight(dy, x, dw, ws)
        dblp.linear_grad_weight(apart(dy), x, fdw, ws)
        for got in (dw, fdw):
            close(got, d(dy).T @ d(x), 2 * (n + 4) * U * (d(dy).abs().T @ d(x).abs()), torch.float32)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_values_below_the_normal_numbers_count(t):
    """16-bit operands below their type's normal numbers are multiplied as what they are."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    tiny = torch.finfo(t).tiny
    g = gen(22)
    for n, inner, outer in ((3, 64, 32), (80, 96, 70), (70, 65, 33)):
        x = (torch.randint(-60, 60, (n, inner), generator=g, device="cuda") / 64 * tiny).to(t)
        w = (torch.randn(outer, inner, generator=g, device="cuda") * 2.0 ** (120 if t == torch.bfloat16 else 10)).to(t)
        y = torch.empty(n, outer, device="cuda")
        dblp.linear(x, w, y, space(dblp.linear_workspace(n, inner, outer)))
        assert bool((x != 0).any()) and float(x.float().abs().max()) < tiny
        close(y, d(x) @ d(w).T, 2 * (inner + 4) * U * (d(x).abs() @ d(w).abs().T), torch.float32)


def test_rows_that_are_one_row():
    """An input whose rows lie on each other (stride 0), as a broadcast one's do."""
    import paper_2605_01989_amd as dblp
    g = gen(11)
    n, inner, outer = 67, 72, 40
    for t in TYPES.values():
        x1, w = torch.randn(1, inner, generator=g, device="cuda").to(t), torch.randn(outer, inner, generator=g, device="cuda").to(t)
        dy1 = torch.randn(1, outer, generator=g, device="cuda").to(t)
        x, dy = x1.expand(n, inner), dy1.expand(n, outer)
        ws = space(dblp.linear_workspace(n, inner, outer))
        a, b = torch.empty(n, outer, dtype=t, device="cuda"), torch.empty(n, outer, dtype=t, device="cuda")
        dblp.linear(x, w, a, ws, residual=dy)
        dblp.linear(x.contiguous(), w, b, ws, residual=dy.contiguous())
        assert torch.equal(a, b)
        a, b = torch.empty(outer, inner, device="cuda"), torch.empty(outer, inner, device="cuda")
        dblp.linear_grad_weight(dy, x, a, ws)
        dblp.linear_grad_weight(dy.contiguous(), x.contiguous(), b, ws)
        assert torch.equal(a, b)
        want = n * d(dy1).T @ d(x1)
        close(a, want, 2 * (n + 4) * U * want.abs(), torch.float32)


def test_norms_are_of_the_whole_matrix():
    """steps = 0: G over the root of its sum of squares, onto the base, whatever the matrices' places."""
    import paper_2605_01989_amd as dblp
    g = gen(12)
    for rows, cols in ((1, 20000), (300, 257), (20000, 3)):
        x = torch.randn(rows, 3, cols, generator=g, device="cuda").permute(1, 0, 2)      # matrices that lie between each other's rows
        out = torch.empty(rows, 3, cols, device="cuda").permute(1, 0, 2)
        dblp.orthogonalize(x, out, space(dblp.orthogonalize_workspace(3, rows, cols)), steps=0, scale=math.pi)
        for i in range(3):
            want = torch.tensor(math.pi).item() * d(x[i]) / d(x[i]).norm()
            close(out[i], want, (2.0 ** -22 + 4 * U) * want.abs() + 2.0 ** -30, torch.float32)


def test_floats_of_every_size_and_what_is_not_finite_in_large_tiles():
    """Fp32 products of many tiles: values from far below to near the largest number, and infinities, whose tiles are made in another way."""
    import paper_2605_01989_amd as dblp
    g = gen(31)
    n, inner, outer = 1500, 400, 2200
    x, w = torch.randn(n, inner, generator=g, device="cuda"), torch.randn(outer, inner, generator=g, device="cuda")
    x *= 2.0 ** torch.randint(-60, 60, (n, 1), generator=g, device="cuda")
    w *= 2.0 ** torch.randint(-40, 40, (outer, 1), generator=g, device="cuda")
    x[5] = torch.finfo(torch.float32).max
    x[5, 1:] = 0.0
    ws = space(dblp.linear_workspace(n, inner, outer))
    y, clean = torch.empty(n, outer, device="cuda"), torch.empty(n, outer, device="cuda")
    dblp.linear(x, w, y, ws)
    want, mag = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    assert bool((((y.double() - want).abs() <= 2 * (inner + 4) * U * mag + 2.0 ** -125) | (want.abs() * (1 + U) > torch.finfo(torch.float32).max) & torch.isinf(y)).all())
    clean.copy_(y)
    x[700, 3], w[900, 7], x[1400, 0] = float("inf"), -float("inf"), float("nan")
    dblp.linear(x, w, y, ws)
    want = x.double() @ w.double().T
    hit = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y[hit & ~torch.isnan(want)].double(), want[hit & ~torch.isnan(want)])
    # (a row or column that keeps its values keeps its results, to the bits where its tile was not made again)
    assert bool((((y.double() - want).abs() <= 2 * (inner + 4) * U * mag + 2.0 ** -125) | hit | (want.abs() * (1 + U) > torch.finfo(torch.float32).max)).all())
