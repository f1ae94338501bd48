"""GPU: a worker's step as study_worker_step.py runs it, from tokens to the mean that the receiver returns."""
import pytest
import torch

import worker_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def by_definition(params, w, p_drop, step, clip, kl_coef):
    """The loss in 64 bits on the CPU, for autograd."""
    table, positions, mix = params
    gate = lambda draw: ref.gates(*w.h.shape, w.rank, draw, p_drop)  # noqa: E731
    tokens, pos, targets = w.tokens.cpu(), w.pos.cpu(), w.targets.cpu()
    h = (table[tokens] + positions[pos]) * gate(2 * step)
    y = (h @ mix.T) * gate(2 * step + 1) + h
    on = targets >= 0
    lp = (y @ table.T).log_softmax(1)[on].gather(1, targets[on][:, None])[:, 0]
    old, back, a, wt = (v.cpu().double()[on] for v in (w.old, w.ref, w.advantages, w.weights))
    r, d = (lp - old).exp(), back - lp
    pl = -torch.minimum(r * a, r.clamp(1 - clip[0], 1 + clip[1]) * a)
    return (wt * (pl + kl_coef * (d.exp() - d - 1))).sum(), lp, r, on


def test_gradient_of_a_step_is_that_of_its_loss():
    """In fp32.  A value of the forward or backward pass is made from at most `vocab` products at a time and the way through goes over eight of
    them, so a gradient's error is below 8 (vocab + 16) U times the sum of magnitudes that meet in it; that sum is taken as
    the gradient's largest value times 64 (its terms' spread over the batch)."""
    import study_worker_step as study
    vocab, seq, dim, batch, step = 61, 12, 24, 10, 5
    p = study.Policy(vocab, seq, dim, seed=3)
    w = study.Worker(p, batch, seq, rank=2, p_drop=0.2, dtype=torch.float32)
    start = [v.clone() for v in (p.table, p.positions, p.mix)]
    p.flat.add_(0.05 * torch.randn(p.n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda"))
    w.sample(start)
    params = [v.cpu().double().requires_grad_(True) for v in (p.table, p.positions, p.mix)]
    # rewards of both signs, whatever was sampled
    w.advantages = torch.randn(batch * seq, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    _, lp, r, on = by_definition(params, w, 0.2, step, study.CLIP, study.KL)
    # the gradient jumps where a ratio crosses a border: none is near one
    for border in (1 - study.CLIP[0], 1 + study.CLIP[1]):
        near = (r.detach() - border).abs() < 1e-3
        idx = on.nonzero()[:, 0][near]
        w.old[idx.cuda()] += 0.01
    loss, lp, r, on = by_definition(params, w, 0.2, step, study.CLIP, study.KL)
    loss.backward()
    got = p.views(w.gradient(step))
    assert abs(float(w.stats[0]) - float(loss.detach())) < 1e-4 * max(1.0, abs(float(loss.detach()))) and float(w.stats[4]) == int(on.sum())
    assert 0 < float(w.stats[3]) < float(w.stats[4])
    for g, q in zip(got, params):
        assert float((g.cpu().double() - q.grad).abs().max()) <= 8 * (vocab + 16) * U * 64 * float(q.grad.abs().max())
    again = w.grad.clone()
    w.gradient(step)
    assert torch.equal(again, w.grad)            # a step computed again is the same gradient


def test_workers_learn_through_a_receiver_that_loses_packets():
    import study_worker_step as study
    out = study.train(workers=3)
    assert out["sent_again"] > 0 and out["rounds"] == 120
    assert out["reward"][0] < 0.05 and max(out["reward"][-5:]) > 0.5, out["reward"]
