"""GPU: the gradient of a whole fp32 step against its definition, within a bound that is carried through the step."""
import pytest
import torch

import worker_reference as ref
from test_gpu_worker import U
from test_gpu_worker_step import by_definition

pytestmark = pytest.mark.gpu


def bounded(params, w, p_drop, step, clip, kl_coef):
    """Bounds of the errors of the three gradients, to first order, each value of the step beside the bound of its error: a sum of n products is off by (n + 1) U times the sum of
    their magnitudes and by its operands' errors; a dropped, scaled or added value by 2 U of its magnitudes."""
    table, positions, mix = (v.detach() for v in params)
    tokens, pos, targets = w.tokens.cpu(), w.pos.cpu(), w.targets.cpu()
    g1, g2 = (ref.gates(*w.h.shape, w.rank, 2 * step + k, p_drop) for k in (0, 1))

    def product(a, ea, b, eb):
        return a @ b, (a.shape[1] + 1) * U * (a.abs() @ b.abs()) + ea @ b.abs() + a.abs() @ eb
    zero = torch.zeros_like
    h, eh = (table[tokens] + positions[pos]) * g1, 4 * U * (table[tokens].abs() + positions[pos].abs()) * g1
    m, em = product(h, eh, mix.T, zero(mix.T))
    y, ey = m * g2 + h, em * g2 + eh + 4 * U * (m.abs() * g2 + h.abs())
    x, ex = product(y, ey, table.T, zero(table.T))
    # a score moves by the errors of its row's logits, at most twice the largest, and by lse's own: an exponential by (3 spread + 2) U, the sum of a row by at most a step a value
    worst = 2 * ex.max(1).values + (3 * (x.max(1).values - x.min(1).values) + 2 + x.shape[1]) * U + 2 * U * x.abs().max(1).values
    r = ref.policy(x, targets, w.advantages, w.weights, w.old, w.ref, clip, kl_coef, 1.0)
    dx = r["dlogits"]
    e_slope = r["bend"] * worst * 1.5 + 2 * U * r["slope"].abs()          # (half as much again: the slope's own curve, for errors far below one)
    edx = e_slope[:, None] * (r["hit"] + r["prob"]) + r["slope"].abs()[:, None] * r["prob"] * (2 * worst[:, None] + 6 * U) + 2 * U * dx.abs()
    head, e_head = product(dx.T, edx.T, y, ey)
    dy, edy = product(dx, edx, table, zero(table))
    dz, edz = dy * g2, edy * g2 + 2 * U * dy.abs() * g2
    g_mix, e_mix = product(dz.T, edz.T, h, eh)
    back, e_back = product(dz, edz, mix, zero(mix))
    dh, edh = dy + back, edy + e_back + 2 * U * (dy.abs() + back.abs())

    def rows(n, index, base, e_base):
        terms = torch.bincount(index, minlength=n)[:, None] + 6
        v, mag = dh * g1, dh.abs() * g1
        return base + zero(base).index_add(0, index, v), e_base + zero(base).index_add(0, index, edh * g1) + terms * U * (base.abs() + zero(base).index_add(0, index, mag))
    return [rows(len(table), tokens, head, e_head), rows(len(positions), pos, zero(positions), zero(positions)), (g_mix, e_mix)]


@pytest.mark.parametrize("vocab, seq, dim, batch", [(61, 12, 24, 10), (200, 17, 40, 33)])
def test_gradient_of_a_step_within_its_carried_bound(vocab, seq, dim, batch):
    import study_worker_step as study
    step = 5
    clip, kl_coef = tuple(torch.tensor(study.CLIP).tolist()), torch.tensor(study.KL).item()          # as the call takes them, in fp32
    p = study.Policy(vocab, seq, dim, seed=3)
    w = study.Worker(p, batch, seq, rank=2, p_drop=0.2, dtype=torch.float32)
    start = [v.clone() for v in (p.table, p.positions, p.mix)]
    p.flat.add_(0.05 * torch.randn(p.n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda"))
    w.sample(start)
    params = [v.cpu().double().requires_grad_(True) for v in (p.table, p.positions, p.mix)]
    w.advantages = torch.randn(batch * seq, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    w.ref[7::11] = -float("inf")                                       # answers that the reference masks
    masked = w.ref.clone()
    _, lp, r, on = by_definition(params, w, 0.2, step, clip, kl_coef)
    for border in (1 - clip[0], 1 + clip[1]):              # the gradient jumps where a ratio crosses a border: none is near one
        w.old[on.nonzero()[:, 0][(r.detach() - border).abs() < 1e-3].cuda()] += 0.01
    # (differentiated with a reference so far below that nothing is left of it: of -inf itself autograd makes NaN)
    w.ref = torch.where(torch.isinf(masked), -1e4, masked)
    by_definition(params, w, 0.2, step, clip, kl_coef)[0].backward()
    w.ref = masked
    got = p.views(w.gradient(step))
    for g, q, (value, bound) in zip(got, params, bounded(params, w, 0.2, step, clip, kl_coef)):
        scale = float(q.grad.abs().max())
        assert float((value - q.grad).abs().max()) <= 1e-11 * scale    # the bound's own values are autograd's
        assert bool(((g.cpu().double() - q.grad).abs() <= bound + 1e-11 * scale).all())
    assert float(w.stats[0]) == float("inf") and 0 < float(w.stats[3]) < float(w.stats[4])
