"""GPU: a worker's step and the update behind the receiver, as study_worker_step.py runs them with the library's products."""
import pytest
import torch

import layer_reference
from test_gpu_worker import U
from test_gpu_worker_gradient import bounded
from test_gpu_worker_step import by_definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab, seq, dim, batch", [(61, 12, 24, 10), (200, 17, 40, 33)])
def test_gradient_of_a_step_by_the_librarys_products(vocab, seq, dim, batch):
    """In fp32, within twice the bound that is carried through the step with sums rounded to nearest: a product's additions may be rounded in any way."""
    import study_worker_step as study
    step = 5
    clip, kl_coef = tuple(torch.tensor(study.CLIP).tolist()), torch.tensor(study.KL).item()
    p = study.Policy(vocab, seq, dim, seed=3)
    w = study.Worker(p, batch, seq, rank=2, p_drop=0.2, dtype=torch.float32, layers=True)
    start = [v.clone() for v in (p.table, p.positions, p.mix)]
    p.flat.add_(0.05 * torch.randn(p.n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda"))
    w.sample(start)
    params = [v.cpu().double().requires_grad_(True) for v in (p.table, p.positions, p.mix)]
    w.advantages = torch.randn(batch * seq, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    _, _, r, on = by_definition(params, w, 0.2, step, clip, kl_coef)
    for border in (1 - clip[0], 1 + clip[1]):              # the gradient jumps where a ratio crosses a border: none is near one
        w.old[on.nonzero()[:, 0][(r.detach() - border).abs() < 1e-3].cuda()] += 0.01
    by_definition(params, w, 0.2, step, clip, kl_coef)[0].backward()
    got = p.views(w.gradient(step))
    for g, q, (_, bound) in zip(got, params, bounded(params, w, 0.2, step, clip, kl_coef)):
        assert bool(((g.cpu().double() - q.grad).abs() <= 2 * bound + 1e-11 * float(q.grad.abs().max())).all())
    again = w.grad.clone()
    w.gradient(step)
    assert torch.equal(again, w.grad)


def test_the_update_of_a_mean_gradient():
    import study_worker_step as study
    p = study.Policy(32, 16, 48, seed=1)
    before = p.flat.clone()
    update = study.Update(p, rate=2.0, max_norm=0.5, layers=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    momentum = torch.zeros(48, 48, dtype=torch.float64)
    mix = p.mix.cpu().double()
    for _ in range(3):
        mean = torch.randn(p.n, generator=g, device="cuda")
        update(mean, float(mean.norm()))
        momentum = 0.8 * momentum + p.views(mean)[2].cpu().double()
        x, e = layer_reference.orthogonal(update.mean_mix.cpu(), 5)
        assert float((update.mean_mix.cpu().double() - momentum).norm()) <= 8 * U * float(momentum.norm())
        assert float((p.mix.cpu().double() - (mix - 0.02 * x)).norm()) <= 0.02 * e + 4 * U * float(mix.norm())
        mix = p.mix.cpu().double()
    rest = 32 * 48 + 16 * 48
    assert not torch.equal(p.flat[:rest], before[:rest])


def test_workers_train_with_the_librarys_layers():
    """It runs: tokens, products, packets and losses, the mean and its orthogonal update, in rounds."""
    import study_worker_step as study
    out = study.train(workers=2, iterations=6, layers=True)
    assert out["rounds"] == 18 and len(out["reward"]) == 6 and all(0 <= r <= 1 for r in out["reward"])
