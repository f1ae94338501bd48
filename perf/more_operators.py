"""The matrix products of a worker's layers, their gradients, and the update made of a mean gradient, as cases that can be timed and compared.

Five kinds of case, one for each entry point of include/dblp_layers.h:

  linear              z = x W^T + bias, y = act(z) + residual; z itself where the way back needs it
  linear_grad_input   dx = (dy W) act'(z) + base
  linear_grad_weight  dW = dy^T x + base, dbias = column sums of dy + base
  activation_grad     dz = dy act'(z)
  orthogonalize       O = X after `STEPS` steps X <- a X + (b A + c A A) X, A = X X^T, from X = G / |G| (Frobenius);
                      out = base_scale base + scale O

`run` computes them in their plain form (torch's elementary operations in 32 bits, rounded once at the end), or,
where `own` is true, by the library's entry points.

Keys of a case: T tokens (rows), `inner` and `outer` columns of a layer's input and output, `type` of activations and weights
("f32", "bf16", "f16"), `out` type of the result, `act` activation, `bias`, `residual`, `pre` (whether z is returned, or gates the gradient),
`base` whether a result is added to what the caller holds, `pad` columns between rows; count, rows and cols of the matrices
to orthogonalise.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
STEPS = 5
A, B, C = 3.4445, -4.7750, 2.0315       # of a step's odd polynomial: it takes singular values of 0.01 and above to about 0.7 to 1.2


def listed():
    """Widths of 768 and 1024 and their multiples, the vocabulary of 50257 and matrices of 768 x 2304 are those of the GPT-2 tensors in this
    repository's workloads, a matrix of 128 x 128 is that of its study of workers; the other sizes are generic."""
    return [
        # decoding: one token through the first half of a block; latency, and the reading of the weights
        dict(name="linear_token", kind="linear", T=1, inner=1024, outer=4096, type="bf16", out="bf16", act="gelu_tanh", bias=True, residual=False, pre=False, pad=0),
        # a short batch in fp32, odd widths, everything in the epilogue
        dict(name="linear_ragged", kind="linear", T=300, inner=333, outer=1000, type="f32", out="f32", act="silu", bias=True, residual=True, pre=False, pad=0),
        # the first half of a wide block in training: z is kept for the way back
        dict(name="linear_wide", kind="linear", T=8192, inner=4096, outer=16384, type="bf16", out="bf16", act="gelu_tanh", bias=True, residual=False, pre=True, pad=0),
        # back through the second half of a block into the first one's z
        dict(name="grad_input_gated", kind="linear_grad_input", T=8192, inner=4096, outer=1024, type="f16", out="f16", act="gelu_tanh", pre=True, base=False, pad=0),
        # from the logits' gradient, whose rows are odd, to the last activation's, with the sum that the residual branch brings
        dict(name="grad_input_logits", kind="linear_grad_input", T=8192, inner=768, outer=50257, type="bf16", out="bf16", act="none", pre=False, base=True, pad=0),
        # a square projection's gradient: few results, each of a long sum
        dict(name="grad_weight_square", kind="linear_grad_weight", T=8192, inner=768, outer=768, type="bf16", bias=True, base=False, pad=0),
        # a wide layer, onto the gradient of an earlier part of the batch
        dict(name="grad_weight_wide", kind="linear_grad_weight", T=32768, inner=4096, outer=4096, type="bf16", bias=True, base=True, pad=0),
        # a short batch, odd width
        dict(name="activation_ragged", kind="activation_grad", T=300, inner=333, type="f32", act="silu", pad=0),
        # the activation of a wide block
        dict(name="activation_wide", kind="activation_grad", T=8192, inner=16384, type="bf16", act="gelu", pad=0),
        # the one square matrix of the study's policy; latency
        dict(name="orthogonal_small", kind="orthogonalize", count=1, rows=128, cols=128, type="f32", base=True),
        # one tensor of each of twelve layers, in one call
        dict(name="orthogonal_gpt2s", kind="orthogonalize", count=12, rows=2304, cols=768, type="f32", base=True),
        # a wide matrix
        dict(name="orthogonal_wide", kind="orthogonalize", count=1, rows=4096, cols=8192, type="f32", base=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them multiples of 64, the others odd."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n | 1


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad_input", "linear_grad_weight", "activation_grad", "orthogonalize", "orthogonalize"])
    t = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind == "orthogonalize":
        rows, cols = _width(rng, 16, 4096), _width(rng, 16, 4096)
        if rng.random() < 0.2:
            cols = _width(rng, 2048, 8192)
        short, long = min(rows, cols), max(rows, cols)
        most = max(1, min(int(2e11 / (short * short * long)), (1 << 25) // (short * long), 64))
        return dict(kind=kind, count=_log(rng, 1, most), rows=rows, cols=cols, type=rng.choice(["f32", "f32", t]), base=rng.random() < 0.7)
    pad = rng.choice([0, 0, rng.randint(1, 64)])
    act = rng.choice(ACTS[1:])
    T = _log(rng, 1, 65536)
    if kind == "activation_grad":
        D = _width(rng, 32, 16384)
        return dict(kind=kind, T=max(1, min(T, (1 << 27) // D)), inner=D, type=t, act=act, pad=pad)
    inner, outer = _width(rng, 32, 16384), _width(rng, 32, 16384)
    if rng.random() < 0.1:
        outer = 50257
    inner, outer = min(inner, (1 << 27) // outer), outer
    T = max(1, min(T, int((2e10 if t == "f32" else 5e11) / (inner * outer)), (1 << 28) // max(inner, outer)))
    if kind == "linear":
        return dict(kind=kind, T=T, inner=inner, outer=outer, type=t, out=rng.choice([t, t, "f32"]), act=rng.choice(["none", act]), bias=rng.random() < 0.7,
                    residual=rng.random() < 0.4, pre=rng.random() < 0.4, pad=pad)
    if kind == "linear_grad_input":
        pre = rng.random() < 0.5
        return dict(kind=kind, T=T, inner=inner, outer=outer, type=t, out=rng.choice([t, t, "f32"]), act=act if pre else "none", pre=pre, base=rng.random() < 0.5, pad=pad)
    return dict(kind=kind, T=T, inner=inner, outer=outer, type=t, bias=rng.random() < 0.7, base=rng.random() < 0.5, pad=pad)


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(gen, rows, cols, std=1.0, to=torch.float32, pad=0):
    """[rows, cols], rows cols + pad apart."""
    return torch.randn(rows, cols + pad, generator=gen, device=DEV).mul_(std).to(to)[:, :cols]


def _gradients(gen, count, rows, cols, to):
    """Like those of a layer: a few strong directions whose strength falls off, over noise."""
    rank = min(rows, cols, 32)
    u, v = (torch.randn(count, n, rank, generator=gen, device=DEV) for n in (rows, cols))
    strength = 1.0 / (torch.arange(rank, device=DEV) + 1.0)
    g = torch.randn(count, rows, cols, generator=gen, device=DEV).mul_(0.1)
    for i in range(count):
        g[i].addmm_(u[i] * strength, v[i].T)
    return g.mul_(1e-3).to(to)


def prepare(c, seed):
    gen = _generator(seed)
    kind = c["kind"]
    t = TYPES[c["type"]]
    s = dict(c=c)
    if kind == "orthogonalize":
        shape = (c["count"], c["rows"], c["cols"])
        s["g"] = _gradients(gen, *shape, t)
        s["base"] = torch.randn(*shape, generator=gen, device=DEV).mul_(0.02) if c["base"] else None
        s["scale"], s["base_scale"] = (-0.02 * max(1.0, c["rows"] / c["cols"]) ** 0.5, 0.998) if c["base"] else (1.0, 0.0)
        s["out"] = torch.empty(*shape, device=DEV)
        if own:
            import paper_2605_01989_amd as dblp
            s["workspace"] = torch.empty(dblp.orthogonalize_workspace(*shape), dtype=torch.uint8, device=DEV)
        return s
    T, inner, pad = c["T"], c["inner"], c["pad"]
    if kind == "activation_grad":
        s["dy"] = _normal(gen, T, inner, 1e-3 if t != torch.float16 else 1.0, t, pad)
        s["pre"] = _normal(gen, T, inner, 1.5, t, pad)
        s["out"] = torch.empty(T, inner, dtype=t, device=DEV)
        return s
    outer = c["outer"]
    out = TYPES[c.get("out", "f32")]
    if kind == "linear":
        s["x"] = _normal(gen, T, inner, 1.0, t, pad)
        s["w"] = _normal(gen, outer, inner, inner ** -0.5, t)
        s["bias"] = torch.randn(outer, generator=gen, device=DEV).mul_(0.1) if c["bias"] else None
        s["residual"] = _normal(gen, T, outer, 1.0, out, pad) if c["residual"] else None
        s["out"] = torch.empty(T, outer, dtype=out, device=DEV)
        s["pre"] = torch.empty(T, outer, dtype=out, device=DEV) if c["pre"] else None
    elif kind == "linear_grad_input":
        # (fp16 gradients are held about one, so that small ones do not vanish)
        s["dy"] = _normal(gen, T, outer, 1e-3 if t != torch.float16 else 1.0, t, pad)
        s["w"] = _normal(gen, outer, inner, outer ** -0.5, t)
        s["pre"] = _normal(gen, T, inner, 1.5, out, pad) if c["pre"] else None
        s["base"] = _normal(gen, T, inner, 1e-3 if t != torch.float16 else 1.0, out, pad) if c["base"] else None
        s["out"] = torch.empty(T, inner, dtype=out, device=DEV)
    else:
        s["dy"] = _normal(gen, T, outer, 1e-3 if t != torch.float16 else 1.0, t, pad)
        s["x"] = _normal(gen, T, inner, 1.0, t, pad)
        s["base"] = _normal(gen, outer, inner, 1e-2) if c["base"] else None
        s["bias_base"] = torch.randn(outer, generator=gen, device=DEV).mul_(1e-2) if c["base"] and c["bias"] else None
        s["out"] = torch.empty(outer, inner, device=DEV)
        s["bias_grad"] = torch.empty(outer, device=DEV) if c["bias"] else None
    if own:
        import paper_2605_01989_amd as dblp
        s["workspace"] = torch.empty(dblp.linear_workspace(T, inner, outer), dtype=torch.uint8, device=DEV)
    return s


def _act_name(c):
    return None if c["act"] == "none" else c["act"]


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        import paper_2605_01989_amd as dblp
        if kind == "linear":
            dblp.linear(s["x"], s["w"], s["out"], s["workspace"], bias=s["bias"], activation=_act_name(c), residual=s["residual"], pre=s["pre"])
            return (s["out"], s["pre"]) if c["pre"] else s["out"]
        if kind == "linear_grad_input":
            dblp.linear_grad_input(s["dy"], s["w"], s["out"], s["workspace"], pre=s["pre"], activation=_act_name(c), base=s["base"])
            return s["out"]
        if kind == "linear_grad_weight":
            dblp.linear_grad_weight(s["dy"], s["x"], s["out"], s["workspace"], base=s["base"], bias_grad=s["bias_grad"], bias_base=s["bias_base"])
            return (s["out"], s["bias_grad"]) if c["bias"] else s["out"]
        if kind == "activation_grad":
            dblp.activation_grad(s["dy"], s["pre"], s["out"], _act_name(c))
            return s["out"]
        dblp.orthogonalize(s["g"], s["out"], s["workspace"], scale=s["scale"], base=s["base"], base_scale=s["base_scale"], steps=STEPS, coefficients=(A, B, C))
        return s["out"]
    return PLAIN[kind](s)


# ---- the plain form ----

ROOT_HALF, ROOT_TWO_OVER_PI = 0.5 ** 0.5, (2 / math.pi) ** 0.5


def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z / (1 + (-z).exp())
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z * ROOT_HALF)
    return z / (1 + (-2 * ROOT_TWO_OVER_PI * (z + 0.044715 * z * z * z)).exp())     # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))


def _slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).float()
    if name == "silu":
        p = 1 / (1 + (-z).exp())
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * torch.erfc(-z * ROOT_HALF) + z * (-0.5 * z * z).exp() * (0.5 * ROOT_TWO_OVER_PI)
    p = 1 / (1 + (-2 * ROOT_TWO_OVER_PI * (z + 0.044715 * z * z * z)).exp())
    return p + z * p * (1 - p) * 2 * ROOT_TWO_OVER_PI * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    c, out = s["c"], s["out"].dtype
    z = s["x"].float() @ s["w"].float().T
    if s["bias"] is not None:
        z += s["bias"]
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(out), z.to(out)) if c["pre"] else y.to(out)


def _plain_grad_input(s):
    dx = s["dy"].float() @ s["w"].float()
    if s["pre"] is not None:
        dx = dx * _slope(s["pre"].float(), s["c"]["act"])
    if s["base"] is not None:
        dx = dx + s["base"].float()
    return dx.to(s["out"].dtype)


def _plain_grad_weight(s):
    dy = s["dy"].float()
    dw = dy.T @ s["x"].float()
    if s["base"] is not None:
        dw += s["base"]
    if s["bias_grad"] is None:
        return dw
    db = dy.sum(0)
    return dw, db + s["bias_base"] if s["bias_base"] is not None else db


def _plain_activation_grad(s):
    return (s["dy"].float() * _slope(s["pre"].float(), s["c"]["act"])).to(s["out"].dtype)


def _plain_orthogonalize(s):
    g = s["g"].float()
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2).contiguous() if tall else g
    x = (x.double() / g.double().square().sum((1, 2), keepdim=True).sqrt()).float()
    for _ in range(STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.bmm(B * a + C * torch.bmm(a, a), x)
    if tall:
        x = x.transpose(1, 2)
    return s["scale"] * x if s["base"] is None else s["base_scale"] * s["base"] + s["scale"] * x


PLAIN = dict(linear=_plain_linear, linear_grad_input=_plain_grad_input, linear_grad_weight=_plain_grad_weight, activation_grad=_plain_activation_grad,
             orthogonalize=_plain_orthogonalize)


def work(c):
    kind = c["kind"]
    if kind == "orthogonalize":
        short, long = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        one = c["count"] * short * long
        # of the two symmetric products half
        return dict(bytes=one * (BYTES[c["type"]] + 4 + 4 * c["base"]), flops=STEPS * c["count"] * (short * short * long + short ** 3 + 2 * short * short * long))
    T, inner, b = c["T"], c["inner"], BYTES[c["type"]]
    if kind == "activation_grad":
        return dict(bytes=3 * T * inner * b, flops=10 * T * inner)
    outer, o = c["outer"], BYTES[c.get("out", "f32")]
    flops = 2 * T * inner * outer
    if kind == "linear":
        return dict(bytes=(T * inner + inner * outer) * b + 4 * outer * c["bias"] + T * outer * o * (1 + c["residual"] + c["pre"]), flops=flops)
    if kind == "linear_grad_input":
        return dict(bytes=(T * outer + inner * outer) * b + T * inner * o * (1 + c["pre"] + c["base"]), flops=flops)
    return dict(bytes=T * (inner + outer) * b + 4 * outer * (inner + c["bias"]) * (1 + c["base"]), flops=flops)


# ---- the definitions in 64 bits ----


def _exact_act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
    return z


def _exact_slope(z, name):
    if name == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if name == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        th = torch.tanh(k * (z + 0.044715 * z ** 3))
        return (1 + th) / 2 + z * (1 - th * th) * k * (1 + 0.134145 * z ** 2) / 2
    return torch.ones_like(z)


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "orthogonalize":
        got = []
        for i in range(c["count"]):
            x = s["g"][i].double()
            x = x / torch.linalg.matrix_norm(x)
            left = c["rows"] <= c["cols"]
            for _ in range(STEPS):                          # a X + b (X X') X + c (X X') (X X') X, from whichever side is the shorter
                gram = x @ x.T if left else x.T @ x
                cubic = gram @ x if left else x @ gram
                fifth = gram @ cubic if left else cubic @ gram
                x = A * x + B * cubic + C * fifth
            x = x * s["scale"]
            got.append(x + s["base"][i].double() * s["base_scale"] if c["base"] else x)
        return torch.stack(got)
    if kind == "activation_grad":
        return s["dy"].double() * _exact_slope(s["pre"].double(), c["act"])
    if kind == "linear":
        ys, zs = [], []
        w = s["w"].double().T.contiguous()
        for i in range(0, c["T"], 4096):
            part = slice(i, i + 4096)
            z = s["x"][part].double() @ w
            if c["bias"]:
                z = z + s["bias"].double()
            y = _exact_act(z, c["act"])
            ys.append(y + s["residual"][part].double() if c["residual"] else y)
            zs.append(z)
        return (torch.cat(ys), torch.cat(zs)) if c["pre"] else torch.cat(ys)
    if kind == "linear_grad_input":
        parts = []
        w = s["w"].double()
        for i in range(0, c["T"], 4096):
            part = slice(i, i + 4096)
            dx = s["dy"][part].double() @ w
            if c["pre"]:
                dx = dx * _exact_slope(s["pre"][part].double(), c["act"])
            parts.append(dx + s["base"][part].double() if c["base"] else dx)
        return torch.cat(parts)
    dw = torch.zeros(c["outer"], c["inner"], dtype=torch.float64, device=DEV) if not c["base"] else s["base"].double()
    db = torch.zeros(c["outer"], dtype=torch.float64, device=DEV) if not (c["base"] and c["bias"]) else s["bias_base"].double()
    for i in range(0, c["T"], 4096):
        dy = s["dy"][i : i + 4096].double()
        dw = dw + dy.T @ s["x"][i : i + 4096].double()
        db = db + dy.sum(0)
    return (dw, db) if c["bias"] else dw
