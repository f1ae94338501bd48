"""GPU: every place of a row of logits counts once, in the largest value, the sum and the gradient, whatever way the row goes.

The rows are such that the sums are exact, so one place left out or taken twice is many times what is allowed."""
import pytest
import torch

from test_gpu_worker import TYPES, U, gen, matrix

pytestmark = pytest.mark.gpu

VOCABS = [1, 7, 100, 515, 1021, 2500, 4096, 9001, 16387, 40001, 50257, 90113, 140001, 180225, 262145, 300001]


def rows_of(vocab):
    """Numbers of rows: one; rows that blocks share, in few and many shares; one block a row, at both of long rows' numbers of threads."""
    return [1, 3, 60, 127, 130, 300] + ([800] if vocab < 60000 else [])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_rows_of_one_value(vocab, t):
    """lse = c + log vocab and lp = -log vocab: the sum is a whole number, so that both are one rounding from their values (and 2^-30 for the logarithm); a
    place more or less is 1 / vocab.  The softmax is 1 / vocab in one rounding, the gradient slope of -1 another, the type's the last."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    u = torch.finfo(t).eps / 2
    log = torch.tensor(float(vocab), dtype=torch.float64).log().item()
    allowed = U * log * (1 + U) + 2.0 ** -30
    assert vocab == 1 or allowed < 0.3 / vocab
    for n in rows_of(vocab):
        for shift in (0, 1):
            g = gen(vocab + n)
            _, x = matrix(g, n, vocab, t, vocab + shift, shift)
            c = torch.randint(-8, 9, (n, 1), generator=g, device="cuda") / 2.0
            x.copy_(c.expand(n, vocab))
            target, one = torch.randint(0, vocab, (n,), generator=g, device="cuda"), torch.ones(n, device="cuda")
            ws = torch.full((dblp.logits_workspace(n, vocab),), 0xA5, dtype=torch.uint8, device="cuda")
            logp, lse, stats = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda"), torch.empty(5, device="cuda")
            dblp.token_logprobs(x, target, logp, ws, lse=lse)
            assert float((logp.double() + log).abs().max()) <= allowed, n
            want = c[:, 0].double() + log
            assert bool(((lse.double() - want).abs() <= U * want.abs() * (1 + U) + 2.0 ** -30).all()), n
            _, d = matrix(g, n, vocab, t, vocab + 3, 0, fill=7.0)
            for grad in (d, None):
                logp.fill_(9.0)
                dblp.policy_loss(x, target, one, one, stats, ws, dlogits=grad, logp=logp)
                assert float((logp.double() + log).abs().max()) <= allowed and float(stats[0]) == -n and float(stats[4]) == n, n
            p = 1.0 / vocab
            hit = d.gather(1, target[:, None]).double()
            assert float((hit - (p - 1)).abs().max()) <= (u + 3 * U) * (1 - p) * 1.01, n
            d.scatter_(1, target[:, None], p)                          # (rounded once as it is)
            assert float(d.float().max() - p) <= (u + 2 * U) * p * 1.01 + (2.0 ** -25 if t == torch.float16 else 0.0), n
            assert float(p - d.float().min()) <= (u + 2 * U) * p * 1.01 + (2.0 ** -25 if t == torch.float16 else 0.0), n


def places(g, vocab):
    """Both ends of the row, both sides of what threads, steps of them, held vectors and shares take, and some in between."""
    at = {0, 1, 2, 3, vocab // 2} | {vocab - 1 - i for i in range(20)}
    for width in (4, 8):
        for vectors in [64 * k for k in (1, 2, 4, 8, 14, 16, 18, 22, 32, 64, 128, 256, 288, 352)] + [(vocab // width + k - 1) // k * s for k in (4, 5, 6, 12, 32) for s in range(1, k)]:
            at |= {vectors * width + i for i in (-9, -8, -2, -1, 0, 1, 2, 8)}
    at |= set(torch.randint(0, vocab, (40,), generator=g, device="cuda").tolist())
    return sorted(p for p in at if 0 <= p < vocab)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("vocab", [v for v in VOCABS if v > 1])
def test_one_place_alone(vocab, t):
    """All logits but one are -inf.  Scores and gradients are exact: with a slope of -1 the gradient is 1 there and -1 at the target."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    g = gen(vocab)
    every = torch.tensor(places(g, vocab), device="cuda")
    some = every[torch.randperm(len(every), generator=g, device="cuda")[:150]]
    # (rows a call; all places by blocks that share a row or, where rows are short, have one each; some of them otherwise)
    for per_call, at in ((60, every), (150, some), (3, some[:9]), (1, some[:3]), (300, every if vocab < 60000 else every[:0])):
        for first in range(0, len(at), per_call):
            hot = at[first : first + per_call]
            hot = torch.cat([hot, hot[:1].expand(per_call - len(hot))])
            n, shift = per_call, first % 2
            _, x = matrix(g, n, vocab, t, vocab + 1, shift, fill=-float("inf"))
            x.scatter_(1, hot[:, None], 4.0)
            target, one = (hot + 1 + torch.randint(0, vocab - 1, (n,), generator=g, device="cuda")) % vocab, torch.ones(n, device="cuda")
            ws = torch.full((dblp.logits_workspace(n, vocab),), 0xA5, dtype=torch.uint8, device="cuda")
            logp, lse, stats = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda"), torch.empty(5, device="cuda")
            dblp.token_logprobs(x, hot, logp, ws, lse=lse)
            assert bool((logp == 0).all()) and bool((lse == 4).all()), (n, first)
            logp.fill_(9.0)
            dblp.policy_loss(x, hot, one, one, stats, ws, logp=logp)
            assert bool((logp == 0).all()), (n, first)
            _, d = matrix(g, n, vocab, t, vocab + 3, 0, fill=7.0)
            dblp.policy_loss(x, target, one, one, stats, ws, dlogits=d, logp=logp)
            assert bool((logp == -float("inf")).all()) and float(stats[0]) == -n, (n, first)
            want = torch.zeros(n, vocab, dtype=t, device="cuda").scatter_(1, hot[:, None], 1.0).scatter_(1, target[:, None], -1.0)
            assert torch.equal(d, want), (n, first)
