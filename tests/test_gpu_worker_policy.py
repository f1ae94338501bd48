"""GPU: the policy loss where its terms leave the range of everyday numbers, on every way that a row can go.

Tolerances are those of test_gpu_worker.py unless a test says otherwise; U is half a step of fp32."""
import pytest
import torch

import worker_reference as ref
from test_gpu_worker import TYPES, U, check_policy, gen, lse_error

pytestmark = pytest.mark.gpu

# (rows, vocabulary): a wave a row; rows held by a block; rows read twice; long rows shared by blocks; one row
WAYS = [(9, 100), (140, 9001), (130, 200003), (3, 300001), (1, 5003)]


def case(g, n, vocab, t):
    x = (torch.randn(n, vocab, generator=g, device="cuda") * 3).to(t)
    target = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    adv, w = torch.randn(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda") + 0.1
    import paper_2605_01989_amd as dblp
    ws = torch.full((dblp.logits_workspace(n, vocab),), 0xA5, dtype=torch.uint8, device="cuda")
    return x, target, adv, w, ws


def run(x, target, adv, w, ws, **args):
    """With the gradient and without: (stats, logp, dlogits) and (stats, logp, None)."""
    import paper_2605_01989_amd as dblp
    got = []
    for d in (torch.full_like(x, 7.0), None):
        stats, logp = torch.full((5,), 9.0, device="cuda"), torch.full((x.shape[0],), 9.0, device="cuda")
        dblp.policy_loss(x, target, adv, w, stats, ws, dlogits=d, logp=logp, **args)
        got.append((stats, logp, d))
    return got


# a reference's log probability less the policy's, or a value that stands for a masked token
APART = [0.0, 1e-4, -0.2, 0.24, 0.26, -0.4, -20.0, -1e3, -3e7, ("is", -1e9), ("is", torch.finfo(torch.float32).min), ("is", -float("inf")), 30.0]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n, vocab", WAYS)
def test_references_far_below_the_policy(n, vocab, t):
    """A token that the reference masks has an endless KL term and a slope of kl_coef a weight."""
    t = TYPES[t]
    g = gen(31 + n)
    x, target, adv, w, ws = case(g, n, vocab, t)
    lp = ref.logprobs(x, target)[0]
    for first in range(0, len(APART), min(n, len(APART))):
        back = torch.empty(n)
        for i in range(n):
            a = APART[(first + i) % len(APART)]
            back[i] = a[1] if isinstance(a, tuple) else float(lp[i]) + a
        back = back.cuda()
        want = ref.policy(x, target, adv, w, None, back, (0.2, 0.3), 0.1, 1.0)
        for got in run(x, target, adv, w, ws, ref_logp=back, clip=(0.2, 0.3), kl_coef=0.1):
            check_policy(got, {k: v.clone() for k, v in want.items()}, x, t, 1.0)
            if got[2] is not None:                   # (the reference 30 above the policy is past fp16)
                assert bool(torch.isfinite(got[2].cpu()[want["dlogits"].abs() < torch.finfo(t).max / 2]).all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n, vocab", WAYS)
def test_ratios_past_fp32_whose_products_are_not(n, vocab, t):
    """exp(lp - old) of 100 and more with a weight that brings it back, for advantages below zero (which are not clipped above)."""
    t = TYPES[t]
    g = gen(32 + n)
    x, target, adv, w, ws = case(g, n, vocab, t)
    adv, w = -0.1 - 0.9 * torch.rand(n, generator=g, device="cuda"), torch.full((n,), 2.0 ** -110, device="cuda")
    lp = ref.logprobs(x, target)[0].cuda()
    for far in (100.0, 130.0, 155.0):
        old = (lp - far).float()
        want = ref.policy(x, target, adv, w, old, None, (0.2, 0.3), 0.0, 1.0)
        assert 2.0 ** -126 < float(want["slope"].abs().min()) and float(want["slope"].abs().max()) < 2.0 ** 127
        for got in run(x, target, adv, w, ws, old_logp=old, clip=(0.2, 0.3)):
            check_policy(got, {k: v.clone() for k, v in want.items()}, x, t, 1.0)
    # past fp64 too: infinite, but an advantage of zero gives zero
    for old in ((lp - 1000).float(), torch.full((n,), -float("inf"), device="cuda")):
        for stats, _, d in run(x, target, adv, w, ws, old_logp=old):
            assert float(stats[0]) == float("inf") and float(stats[3]) == 0 and (d is None or not bool(torch.isfinite(d[torch.arange(n), target]).any()))
        for stats, _, d in run(x, target, torch.zeros_like(adv), w, ws, old_logp=old):
            assert stats[:4].tolist() == [0, 0, 0, 0] and (d is None or not bool(d.any()))
