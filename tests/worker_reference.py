"""The worker's operators by their definitions in 64 bits, on the CPU, for the tests."""
import numpy as np
import torch

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=10):
    """Philox4x32 on arrays of four counter words and two key words (Salmon et al., SC 2011)."""
    a, b, c, d = (np.asarray(v, dtype=np.uint64) for v in counter)
    k0, k1 = (int(k) for k in key)
    for _ in range(rounds):
        p, q = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (q >> np.uint64(32)) ^ b ^ np.uint64(k0), q & M32, (p >> np.uint64(32)) ^ d ^ np.uint64(k1), p & M32
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return a, b, c, d


def gates(rows, cols, seed, draw, p):
    """[rows, cols] factors of a dropout mask: 0 where a value is dropped."""
    limit = int(np.rint(65536 * p))
    if limit == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    per_row = -(-cols // 8)
    g = np.arange(rows * per_row, dtype=np.uint64)
    same = np.ones_like(g)
    w = philox((g & M32, g >> np.uint64(32), same * np.uint64(draw & 0xFFFFFFFF), same * np.uint64(draw >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    fields = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], axis=1).reshape(rows, per_row * 8)[:, :cols]
    return torch.from_numpy((fields >= np.uint64(limit)) * (65536 / (65536 - limit) if limit < 65536 else 0.0))


def rows_of(table, index):
    table, index = table.cpu().double(), index.cpu()
    there = (index >= 0) & (index < table.shape[0])
    out = torch.zeros(index.numel(), table.shape[1], dtype=torch.float64)
    out[there] = table[index[there]]
    return out


def dropped(x, gate):
    return torch.where(gate == 0, torch.zeros_like(x), x * gate)


def embed_grad(tokens, dy, vocab, scale, gate, base):
    """(gradient, sum of the terms' magnitudes, number of terms of each row)."""
    tokens, dy = tokens.cpu(), dropped(dy.cpu().double(), gate)
    there = (tokens >= 0) & (tokens < vocab)
    g = torch.zeros(vocab, dy.shape[1], dtype=torch.float64) if base is None else base.cpu().double().clone()
    mag = g.abs()
    g.index_add_(0, tokens[there], scale * dy[there])
    mag.index_add_(0, tokens[there], abs(scale) * dy[there].abs())
    return g, mag, torch.bincount(tokens[there], minlength=vocab)[:, None]


def softmax_parts(logits):
    """(x - shift, shift, sum of exp(x - shift)): a shift and a logarithm are not added up before the difference is taken, since a row
    of the type's lowest value would lose the logarithm."""
    x = logits.cpu().double()
    m = x.max(1, keepdim=True).values
    at = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    return x - at, at, (x - at).exp().sum(1, keepdim=True)


def logprobs(logits, targets):
    """(lp, lse) by definition; the caller says which rows count."""
    x, at, total = softmax_parts(logits)
    lse = (at + total.log())[:, 0]
    lp = x.gather(1, targets.cpu().clamp(0, x.shape[1] - 1)[:, None])[:, 0] - total.log()[:, 0]
    return torch.where(lse == -np.inf, lse, lp), lse


def policy(logits, targets, adv, w, old, ref, clip, kl_coef, grad_scale):
    """dict of stats [5], logp, dlogits, slope (grad_scale d loss / d lp) and its derivative's magnitude `bend`."""
    V, t = logits.shape[1], targets.cpu()
    x, _, total = softmax_parts(logits)
    lp, lse = logprobs(logits, targets)
    asked = (t >= 0) & (t < V) & (w.cpu() != 0)
    on = asked & (lse != -np.inf)
    zero = torch.zeros_like(lp)
    lpc = torch.where(on, lp, zero)
    a, wt = torch.where(on, adv.cpu().double(), zero), torch.where(on, w.cpu().double(), zero)
    r = (lpc - torch.where(on, old.cpu().double(), zero)).exp() if old is not None else torch.ones_like(lp)
    lo, hi = 1 - float(np.float32(clip[0])), 1 + float(np.float32(clip[1]))
    free, held = r * a, r.clamp(lo, hi) * a
    cut = (held < free) & on
    pl = -torch.minimum(free, held)
    d = torch.where(on, ref.cpu().double(), zero) - lpc if ref is not None else zero
    kl = d.expm1() - d
    k = float(np.float32(kl_coef))
    slope = grad_scale * wt * (torch.where(cut, zero, -free) - k * d.expm1())
    bend = abs(grad_scale) * wt.abs() * (torch.where(cut, zero, free.abs()) + abs(k) * d.exp())
    prob = torch.where(on[:, None], x.exp() / total, torch.zeros_like(x))
    hit = torch.zeros_like(x)
    hit[torch.arange(len(t))[on], t[on]] = 1.0
    grad = torch.where(on[:, None], slope[:, None] * (hit - prob), torch.zeros_like(x))
    stats = torch.stack([(wt * (pl + k * kl)).sum(), (wt * pl).sum(), (wt * kl).sum(), cut.sum().double(), on.sum().double()])
    mags = torch.stack([(wt.abs() * (pl.abs() + abs(k) * kl.abs())).sum(), (wt.abs() * pl.abs()).sum(), (wt.abs() * kl.abs()).sum()])
    moves = torch.stack([(wt.abs() * (free.abs() + abs(k) * d.expm1().abs())).sum(), (wt.abs() * free.abs()).sum(), (wt.abs() * d.expm1().abs()).sum()])
    logp = torch.where(on, lp, torch.where(asked, lse, zero))
    return dict(stats=stats, mags=mags, moves=moves, logp=logp, dlogits=grad, slope=slope, bend=bend, prob=prob, hit=hit, on=on)
