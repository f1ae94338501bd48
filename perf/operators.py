"""The operators at the two ends of a worker's training step, as cases that can be timed and compared.

Five kinds of case, one for each entry point of include/dblp_worker.h:

  embed           y[t] = drop(scale * E[token t] + P[position t])
  embed_grad      G[v] = base[v] + scale * sum of drop(dy[t]) over the tokens t that are v
  dropout         y = drop(x) + residual; with another gradient in x's place its own backward pass
  token_logprobs  log probability of one given token a row of logits, and the row's log-sum-exp (rows without a token: 0)
  policy_loss     clipped policy loss with a KL term: loss, its parts, and the gradient of the logits

`run` computes them in their plain form (torch's elementary operations in 32 bits, rounded once at the end), or,
where `own` is true, by the library's entry points.

Keys of a case: T tokens (rows), V vocabulary, D width, `type` of activations and logits ("f32", "bf16", "f16"),
`table` type of the embedding tables, `pos` rows of the position table (0: none), `p` probability of dropping,
`none` share of rows without a token (padding, prompts), `base` whether a gradient is added to one that the caller
holds, `residual` whether dropout is added to another tensor, `pad` columns between the rows of the logits,
`old` and `ref` whether the old policy's and the reference's log probabilities are given.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
DRAW = 11                       # which of a seed's masks: a training loop counts it up


def listed():
    """Vocabulary 50257, width 768 and 1024 and sequences of 1024 are those of the GPT-2 tensors in this repository's
    workloads; the other sizes are generic."""
    return [
        # decoding: the row of one token, in the type of the activations; latency is all there is
        dict(name="embed_token", kind="embed", T=1, V=50257, D=768, table="f32", type="bf16", pos=1024, p=0.0, none=0.0, scale=1.0),
        # a worker's batch of eight sequences, fp32 tables as the aggregated gradient updates them, dropout on the sum
        dict(name="embed_gpt2s", kind="embed", T=8192, V=50257, D=768, table="f32", type="bf16", pos=1024, p=0.1, none=0.0, scale=1.0),
        # a large batch on a wide model with a 16-bit table and rows scaled by sqrt(D), padded at the sequences' ends
        dict(name="embed_wide", kind="embed", T=32768, V=131072, D=4096, table="bf16", type="bf16", pos=0, p=0.0, none=0.05, scale=64.0),
        # a short ragged batch on a small table, odd width, all in fp32
        dict(name="embed_grad_ragged", kind="embed_grad", T=300, V=1000, D=333, type="f32", p=0.1, none=0.1, base=False, scale=1.0),
        # tied tables: the lookup's gradient on top of the head's, the result is what the worker sends
        dict(name="embed_grad_gpt2s", kind="embed_grad", T=8192, V=50257, D=768, type="bf16", p=0.1, none=0.0, base=True, scale=1.0),
        # a large batch, the table's whole gradient written: rows without a token are zeros
        dict(name="embed_grad_gpt2m", kind="embed_grad", T=65536, V=50257, D=1024, type="bf16", p=0.1, none=0.03, base=False, scale=1.0),
        # a residual branch of the worker's batch, forward
        dict(name="dropout_residual", kind="dropout", T=8192, D=768, type="bf16", p=0.1, residual=True),
        # the backward pass of a wide activation
        dict(name="dropout_large", kind="dropout", T=16384, D=4096, type="f16", p=0.1, residual=False),
        # serving: the score of the one token just sampled
        dict(name="logprobs_token", kind="token_logprobs", T=1, V=50257, type="bf16", pad=0, none=0.0),
        # a reference model's scores of a batch
        dict(name="logprobs_batch", kind="token_logprobs", T=8192, V=50257, type="bf16", pad=0, none=0.3),
        # the tokens of one short answer, fp32 logits, first update on them (the old policy is the present one)
        dict(name="policy_answer", kind="policy_loss", T=100, V=50257, type="f32", pad=0, none=0.0, old=False, ref=True),
        # a batch with prompts masked, rows padded to a multiple of 64
        dict(name="policy_batch", kind="policy_loss", T=8192, V=50257, type="bf16", pad=47, none=0.3, old=True, ref=True),
    ]


def _grad_scale(c):
    """Of the logits' gradients: in fp16 they are held about one, so that small ones do not vanish."""
    return float(c["T"]) if c["type"] == "f16" else 1.0


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them multiples of 80, the others odd."""
    n = _log(rng, lo, hi)
    return max(80, n // 80 * 80) if rng.random() < 0.5 else n | 1


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "dropout", "token_logprobs", "policy_loss"])
    t = rng.choice(["f32", "bf16", "bf16", "f16"])
    none = rng.choice([0.0, round(rng.uniform(0.01, 0.6), 2)])
    if kind in ("embed", "embed_grad"):
        D = _width(rng, 32, 4096)
        T = min(_log(rng, 1, 65536), (1 << 26) // D)
        V = min(_log(rng, 500, 200_000), (1 << 27) // D)
        p = rng.choice([0.0, 0.1, round(rng.uniform(0.02, 0.5), 3)])
        scale = rng.choice([1.0, math.sqrt(D)])
        if kind == "embed":
            return dict(kind=kind, T=T, V=V, D=D, table=rng.choice(["f32", "f32", t]), type=t, pos=rng.choice([0, _log(rng, 128, 4096)]),
                        p=p, none=none, scale=scale)
        return dict(kind=kind, T=T, V=V, D=D, type=t, p=p, none=none, base=rng.random() < 0.5, scale=scale)
    if kind == "dropout":
        D = _width(rng, 32, 16384)
        return dict(kind=kind, T=min(_log(rng, 1, 65536), (1 << 26) // D), D=D, type=t, p=rng.choice([0.1, round(rng.uniform(0.02, 0.7), 3)]),
                    residual=rng.random() < 0.5)
    V = rng.choice([50257, 50304, _width(rng, 500, 200_000)])
    T = max(1, min(_log(rng, 1, 16384), 650_000_000 // (V * BYTES[t])))
    c = dict(kind=kind, T=T, V=V, type=t, pad=rng.choice([0, 0, rng.randint(1, 64)]), none=none)
    return c if kind == "token_logprobs" else dict(c, old=rng.random() < 0.7, ref=rng.random() < 0.7)


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _frequencies(V):
    """Of a language's tokens by rank: falling with about one over the rank."""
    f = 1.0 / (torch.arange(V, dtype=torch.float64) + 3.0)
    return f / f.sum()


def _tokens(gen, T, V, none):
    u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
    rank = torch.searchsorted(_frequencies(V).to(DEV).cumsum(0), u).clamp_(max=V - 1)
    ids = torch.randperm(V, generator=gen, device=DEV)[rank]
    return torch.where(torch.rand(T, generator=gen, device=DEV) < none, -torch.ones_like(ids), ids)


def _distinct(T, V):
    """How many rows of a table T such tokens are expected to touch."""
    return float((1 - (1 - _frequencies(V)) ** T).sum())


def _normal(gen, *shape, std=1.0, to=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEV).mul_(std).to(to)


def _logits(gen, c):
    """[T, V], rows V + pad apart: spread like a trained model's, the token that was taken often among the likely ones."""
    wide = _normal(gen, c["T"], c["V"] + c["pad"], std=2.0, to=TYPES[c["type"]])
    logits = wide[:, : c["V"]]
    target = torch.randint(0, c["V"], (c["T"],), generator=gen, device=DEV)
    up = torch.rand(c["T"], 1, generator=gen, device=DEV) * 10
    logits.scatter_add_(1, target[:, None], up.to(logits.dtype))
    return logits, target


def _true_logprobs(logits, target):
    parts = []
    for i in range(0, logits.shape[0], 1024):
        x = logits[i : i + 1024].double()
        parts.append(x.gather(1, target[i : i + 1024, None])[:, 0] - x.logsumexp(1))
    return torch.cat(parts)


def prepare(c, seed):
    gen = _generator(seed)
    kind, T = c["kind"], c["T"]
    s = dict(c=c, seed=seed * 0x9E3779B97F4A7C15 % (1 << 64))
    if kind == "embed":
        s["tokens"] = _tokens(gen, T, c["V"], c["none"])
        s["table"] = _normal(gen, c["V"], c["D"], std=0.02, to=TYPES[c["table"]])
        s["positions"] = torch.arange(T, device=DEV) % c["pos"] if c["pos"] else None
        s["pos_table"] = _normal(gen, c["pos"], c["D"], std=0.02, to=TYPES[c["table"]]) if c["pos"] else None
        s["out"] = torch.empty(T, c["D"], dtype=TYPES[c["type"]], device=DEV)
    elif kind == "embed_grad":
        s["tokens"] = _tokens(gen, T, c["V"], c["none"])
        s["dy"] = _normal(gen, T, c["D"], std=1e-3, to=TYPES[c["type"]])
        s["base"] = _normal(gen, c["V"], c["D"], std=1e-3) if c["base"] else None
        s["out"] = torch.empty(c["V"], c["D"], device=DEV)
    elif kind == "dropout":
        s["x"] = _normal(gen, T, c["D"], to=TYPES[c["type"]])
        s["residual"] = _normal(gen, T, c["D"], to=TYPES[c["type"]]) if c["residual"] else None
        s["out"] = torch.empty(T, c["D"], dtype=TYPES[c["type"]], device=DEV)
    else:
        s["logits"], target = _logits(gen, c)
        none = torch.rand(T, generator=gen, device=DEV) < c["none"]
        s["logp"] = torch.empty(T, device=DEV)
        s["targets"] = torch.where(none, -torch.ones_like(target), target)
        if kind == "token_logprobs":
            s["lse"] = torch.empty(T, device=DEV)
        else:
            now = _true_logprobs(s["logits"], target)
            change = 0.15 * torch.randn(T, generator=gen, device=DEV, dtype=torch.float64)
            # a ratio within rounding of a border of the clipping has two right gradients: none here is
            for border in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
                change = torch.where((change - border).abs() < 1e-3, change + 3e-3, change)
            s["old"] = (now - change).float() if c["old"] else None
            s["ref"] = (now + 0.1 * torch.randn(T, generator=gen, device=DEV, dtype=torch.float64)).float() if c["ref"] else None
            s["advantages"] = _normal(gen, T)
            s["weights"] = (~none).float() / max(1, int((~none).sum()))
            s["dlogits"] = torch.empty(T, c["V"], dtype=TYPES[c["type"]], device=DEV)
            s["stats"] = torch.empty(5, device=DEV)
    if own:
        import paper_2605_01989_amd as dblp
        s["drop"] = dblp.Drop(s["seed"], DRAW, c["p"]) if c.get("p") else None
        if kind == "embed_grad":
            s["workspace"] = torch.empty(dblp.embed_grad_workspace(T, c["V"], c["D"]), dtype=torch.uint8, device=DEV)
        if kind in ("token_logprobs", "policy_loss"):
            s["workspace"] = torch.empty(dblp.logits_workspace(T, c["V"]), dtype=torch.uint8, device=DEV)
    return s


def run(s):
    kind = s["c"]["kind"]
    if own:
        import paper_2605_01989_amd as dblp
        c = s["c"]
        if kind == "embed":
            dblp.embed(s["tokens"], s["table"], s["out"], scale=c["scale"], positions=s["positions"], pos_table=s["pos_table"], drop=s["drop"])
            return s["out"]
        if kind == "embed_grad":
            dblp.embed_grad(s["tokens"], s["dy"], s["out"], s["workspace"], scale=c["scale"], drop=s["drop"], base=s["base"])
            return s["out"]
        if kind == "dropout":
            dblp.dropout(s["x"], s["out"], s["drop"], residual=s["residual"])
            return s["out"]
        if kind == "token_logprobs":
            dblp.token_logprobs(s["logits"], s["targets"], s["logp"], s["workspace"], lse=s["lse"])
            return s["logp"], s["lse"]
        dblp.policy_loss(s["logits"], s["targets"], s["advantages"], s["weights"], s["stats"], s["workspace"], old_logp=s["old"],
                         ref_logp=s["ref"], dlogits=s["dlogits"], logp=s["logp"], clip=(CLIP_LOW, CLIP_HIGH), kl_coef=KL,
                         grad_scale=_grad_scale(c))
        return s["stats"], s["logp"], s["dlogits"]
    return PLAIN[kind](s)


# ---- the plain form ----

M32 = 0xFFFFFFFF


def _product(a, b):
    """(high, low) 32 bits of a * b: 64-bit integers wrap, which leaves their bits right."""
    ab = a * b
    return (ab >> 32) & M32, ab & M32


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _keep(rows, cols, seed, p):
    """Whether each value stays, and what it is multiplied by: eight 16-bit fields of Philox4x32 in ten rounds (Salmon et
    al., SC 2011) under the key `seed`, for the counter (number of the eight, DRAW), against 65536 p."""
    gates = -(-cols // 8)
    g = torch.arange(rows * gates, device=DEV)
    a, b, c, d = g & M32, g >> 32, torch.full_like(g, DRAW & M32), torch.full_like(g, DRAW >> 32)
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        h0, l0 = _product(a, 0xD2511F53)
        h1, l1 = _product(c, 0xCD9E8D57)
        a, b, c, d = h1 ^ b ^ k0, l1, h0 ^ d ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    fields = torch.stack([f for w in (a, b, c, d) for f in (w & 0xFFFF, w >> 16)], dim=-1)
    limit = round(p * 65536)
    return fields.view(rows, gates * 8)[:, :cols] >= limit, 65536 / (65536 - limit) if limit < 65536 else 0.0


def _dropped(x, s):
    """x in 32 bits, its dropped values zero whatever they are."""
    if not s["c"]["p"]:
        return x
    keep, q = _keep(x.shape[0], x.shape[1], s["seed"], s["c"]["p"])
    return torch.where(keep, x * q, torch.zeros_like(x))


def _rows(table, index):
    return torch.where((index >= 0)[:, None], table[index.clamp(min=0)].float(), 0.0)


def _plain_embed(s):
    y = _rows(s["table"], s["tokens"]) * s["c"]["scale"]
    if s["positions"] is not None:
        y = y + _rows(s["pos_table"], s["positions"])
    return _dropped(y, s).to(s["out"].dtype)


def _plain_embed_grad(s):
    c = s["c"]
    dy = _dropped(s["dy"].float(), s) * c["scale"]
    taken = s["tokens"] >= 0
    base = s["base"].clone() if s["base"] is not None else torch.zeros(c["V"], c["D"], device=DEV)
    return base.index_add_(0, s["tokens"][taken], dy[taken])


def _plain_dropout(s):
    y = _dropped(s["x"].float(), s)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["out"].dtype)


def _scores(s):
    """Log probabilities of the targets and log-sum-exp in 64 bits from sums in 32, and the softmax in 32."""
    x = s["logits"].float()
    top = x.max(1, keepdim=True).values
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    lse = top[:, 0].double() + total[:, 0].double().log()
    at = s["targets"].clamp(min=0)[:, None]
    return x.gather(1, at)[:, 0].double() - lse, lse, e / total


def _plain_token_logprobs(s):
    logp, lse, _ = _scores(s)
    there = s["targets"] >= 0
    return torch.where(there, logp, 0.0).float(), torch.where(there, lse, 0.0).float()


def _plain_policy_loss(s):
    logp, _, prob = _scores(s)
    counted = (s["targets"] >= 0) & (s["weights"] != 0)
    w, a = s["weights"].double(), s["advantages"].double()
    r = (logp - s["old"].double()).exp() if s["old"] is not None else torch.ones_like(logp)
    free, held = r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    policy, clipped = -torch.minimum(free, held), held < free
    slope = torch.where(clipped, 0.0, -free)
    kl = torch.zeros_like(logp)
    if s["ref"] is not None:
        d = s["ref"].double() - logp
        kl = d.exp() - d - 1
        slope = slope + KL * (1 - d.exp())
    zero = torch.zeros_like(w)
    w = torch.where(counted, w, zero)
    parts = [torch.where(counted, w * v, zero).sum() for v in (policy + KL * kl, policy, kl)]
    stats = torch.stack([*parts, (clipped & counted).sum().double(), counted.sum().double()]).float()
    slope = (_grad_scale(s["c"]) * torch.where(counted, w * slope, zero)).float()[:, None]
    grad = prob * -slope
    grad.scatter_add_(1, s["targets"].clamp(min=0)[:, None], slope)
    return stats, torch.where(counted, logp, zero).float(), grad.to(s["dlogits"].dtype)


PLAIN = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, dropout=_plain_dropout, token_logprobs=_plain_token_logprobs,
             policy_loss=_plain_policy_loss)


def work(c):
    kind, T = c["kind"], c["T"]
    if kind in ("embed", "embed_grad"):
        V, D = c["V"], c["D"]
        if kind == "embed":
            rows = _distinct(T * (1 - c["none"]), V) + min(T, c["pos"])
            return dict(bytes=rows * D * BYTES[c["table"]] + 8 * T * (2 if c["pos"] else 1) + T * D * BYTES[c["type"]], flops=3 * T * D)
        return dict(bytes=T * (1 - c["none"]) * D * BYTES[c["type"]] + 8 * T + V * D * 4 * (2 if c["base"] else 1), flops=3 * T * D)
    if kind == "dropout":
        return dict(bytes=T * c["D"] * BYTES[c["type"]] * (3 if c["residual"] else 2), flops=2 * T * c["D"])
    one, counted = T * c["V"] * BYTES[c["type"]], T * c["V"] * (1 - c["none"])
    if kind == "token_logprobs":
        return dict(bytes=one * (1 - c["none"]) + 16 * T, flops=4 * counted)
    return dict(bytes=one * (1 - c["none"]) + one + T * (20 + 4 * c["old"] + 4 * c["ref"]), flops=7 * counted)


# ---- the definitions in 64 bits ----


def _exact_gates(rows, cols, seed, p):
    """Factor of each value (0 where it is dropped): the 32-bit products put together from 16-bit halves."""
    def times(m, v):
        lo, hi = v % 65536, v // 65536
        mlo, mhi = m % 65536, m // 65536
        low = lo * mlo
        mid = hi * mlo + low // 65536
        mid2 = lo * mhi + mid % 65536
        return hi * mhi + mid // 65536 + mid2 // 65536, mid2 % 65536 * 65536 + low % 65536

    gates = (cols + 7) // 8
    n = torch.arange(rows * gates, device=DEV)
    x = [n % 2**32, n // 2**32, torch.full_like(n, DRAW), torch.zeros_like(n)]
    for i in range(10):
        key = [(seed % 2**32 + i * 0x9E3779B9) % 2**32, (seed // 2**32 + i * 0xBB67AE85) % 2**32]
        hi0, lo0 = times(0xD2511F53, x[0])
        hi1, lo1 = times(0xCD9E8D57, x[2])
        x = [hi1.bitwise_xor(x[1]).bitwise_xor(key[0]), lo1, hi0.bitwise_xor(x[3]).bitwise_xor(key[1]), lo0]
    halves = torch.empty(rows * gates, 8, dtype=torch.int64, device=DEV)
    for i in range(4):
        halves[:, 2 * i] = x[i] % 65536
        halves[:, 2 * i + 1] = x[i] // 65536
    limit = round(p * 65536)
    factor = (halves.reshape(rows, gates * 8)[:, :cols] >= limit).double()
    return factor.mul_(65536 / (65536 - limit)) if limit < 65536 else factor


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    gates = lambda: _exact_gates(c["T"], c["D"], s["seed"], c["p"]) if c["p"] else 1.0  # noqa: E731
    if kind == "embed":
        y = torch.zeros(c["T"], c["D"], dtype=torch.float64, device=DEV)
        there = s["tokens"].ge(0).nonzero()[:, 0]
        y[there] = s["table"].index_select(0, s["tokens"][there]).double() * c["scale"]
        if c["pos"]:
            y += s["pos_table"].index_select(0, s["positions"]).double()
        return y * gates()
    if kind == "embed_grad":
        dy = s["dy"].double() * gates() * c["scale"]
        g = torch.zeros(c["V"] + 1, c["D"], dtype=torch.float64, device=DEV)        # the last row takes what has no token
        g.index_put_((s["tokens"].remainder(c["V"] + 1),), dy, accumulate=True)
        return g[:-1] + s["base"] if c["base"] else g[:-1]
    if kind == "dropout":
        y = s["x"].double() * gates()
        return y + s["residual"] if c["residual"] else y
    there = s["targets"].ge(0)
    if kind == "token_logprobs":
        logp = torch.zeros(c["T"], dtype=torch.float64, device=DEV)
        logp[there] = _true_logprobs(s["logits"], s["targets"].clamp(min=0))[there]
        lse = torch.cat([x.double().logsumexp(1) for x in s["logits"].split(1024)])
        return logp, lse * there
    stats = torch.zeros(5, dtype=torch.float64, device=DEV)
    logps, grads = [], []
    for i in range(0, c["T"], 1024):
        part = slice(i, min(i + 1024, c["T"]))
        x, t, on = s["logits"][part].double(), s["targets"][part], there[part]
        logq = x - x.logsumexp(1, keepdim=True)
        lp = logq.gather(1, t.clamp(min=0)[:, None])[:, 0]
        w, a = s["weights"][part].double() * on, s["advantages"][part].double()
        ratio = torch.exp(lp - s["old"][part]) if c["old"] else torch.ones_like(lp)
        # the gradient stops where the ratio has gone past a border in the direction of the advantage
        past = torch.where(a > 0, ratio > 1 + CLIP_HIGH, (a < 0) & (ratio < 1 - CLIP_LOW))
        border = torch.where(a > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW).double()
        policy = -a * torch.where(past, border, ratio)
        back = torch.expm1(s["ref"][part] - lp) if c["ref"] else torch.zeros_like(lp)
        kl = back - (s["ref"][part] - lp) if c["ref"] else back
        slope = w * (torch.where(past, 0.0, -a * ratio) - KL * back)
        hit = torch.zeros_like(x)
        hit[torch.arange(x.shape[0], device=DEV)[on], t[on]] = 1.0
        grads.append(_grad_scale(c) * slope[:, None] * (hit - logq.exp()))
        logps.append(lp * on)
        sums = [(w * policy).sum(), (w * kl).sum()]
        stats += torch.stack([sums[0] + KL * sums[1], *sums, (past & on).sum().double(), on.sum().double()])
    return stats, torch.cat(logps), torch.cat(grads)
