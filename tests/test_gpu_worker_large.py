"""GPU: the worker's operators where the data are so large that other kernels or several launches take them: past the memory-side cache, past what the launches of a sort
write beside it, past a grid's units.

References are the definitions in 64 bits, in pieces on the GPU where they are large, or the same rows in smaller calls, which the other tests compare with
the definitions.  Tolerances are those of test_gpu_worker.py."""
import numpy as np
import pytest
import torch

import worker_reference as ref
from test_gpu_worker import TYPES, U, gen, tokens_of

pytestmark = pytest.mark.gpu

CACHE = 256 << 20


def gates_of_rows(rows, cols, seed, draw, p):
    """worker_reference.gates for some rows of a matrix."""
    per_row, limit = -(-cols // 8), int(np.rint(65536 * p))
    g = (rows.cpu().numpy().astype(np.uint64)[:, None] * np.uint64(per_row) + np.arange(per_row, dtype=np.uint64)).ravel()
    same = np.ones_like(g)
    w = ref.philox((g & ref.M32, g >> np.uint64(32), same * np.uint64(draw & 0xFFFFFFFF), same * np.uint64(draw >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    fields = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], axis=1).reshape(len(rows), per_row * 8)[:, :cols]
    return torch.from_numpy((fields >= np.uint64(limit)) * (65536 / (65536 - limit)))


def near(got, want, mag, t):
    """close() on the GPU, for values well inside the type: half a step, and four fp32 roundings of `mag`."""
    u = torch.finfo(t).eps / 2
    tiny = 2.0 ** -24 if t == torch.float16 else 2.0 ** -125
    return bool(((got.double() - want).abs() <= u * want.abs() * (1 + u) + 4 * U * mag + tiny).all())


@pytest.mark.parametrize("t, rows, cols, residual", [("f16", 16400, 4096, False), ("bf16", 10930, 4096, True), ("f32", 5500, 4104, True), ("f32", 262200, 128, False)])
def test_dropout_past_the_cache(t, rows, cols, residual):
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    assert cols % 8 == 0 and rows * cols * t.itemsize * (3 if residual else 2) >= CACHE
    g, p, seed, draw = gen(41), 0.2, 0xFEDCBA9876543210, (3 << 33) + 7
    x, r, y = (torch.randn(rows, cols, generator=g, device="cuda").to(t) for _ in range(3))
    dblp.dropout(x, y, dblp.Drop(seed, draw, p), residual=r if residual else None)
    for part in torch.arange(rows).split(2048):
        a, b = int(part[0]), int(part[-1]) + 1
        xd = x[a:b].double() * gates_of_rows(part, cols, seed, draw, p).cuda()
        rd = r[a:b].double() if residual else torch.zeros_like(xd)
        assert near(y[a:b], xd + rd, xd.abs() + rd.abs(), t), a


@pytest.mark.parametrize("table, out, n, dim, p, positions", [("bf16", "bf16", 16400, 4096, 0.0, False), ("f32", "bf16", 16400, 4096, 0.1, True), ("f16", "f32", 8200, 4104, 0.1, False), ("f32", "f32", 262200, 136, 0.0, True)])
def test_embed_past_the_cache(table, out, n, dim, p, positions):
    import paper_2605_01989_amd as dblp
    tt, ot = TYPES[table], TYPES[out]
    assert dim % 8 == 0 and n * dim * ot.itemsize > CACHE / 2
    g, vocab, n_pos, seed, draw = gen(42), 3001, 1000, 99, 12
    tab, pos_tab = torch.randn(vocab, dim, generator=g, device="cuda").to(tt), torch.randn(n_pos, dim, generator=g, device="cuda").to(tt) if positions else None
    tok, pos = tokens_of(g, n, vocab, "bad"), tokens_of(g, n, n_pos, "bad") if positions else None
    y = torch.full((n, dim), 7.0, dtype=ot, device="cuda")
    dblp.embed(tok, tab, y, scale=2.5, positions=pos, pos_table=pos_tab, drop=dblp.Drop(seed, draw, p))

    def rows_of(m, i):
        there = (i >= 0) & (i < m.shape[0])
        return torch.where(there[:, None], m[i.where(there, 0)].double(), 0.0)
    for part in torch.arange(n).split(2048):
        a, b = int(part[0]), int(part[-1]) + 1
        e = rows_of(tab, tok[a:b]) * 2.5
        q = rows_of(pos_tab, pos[a:b]) if positions else torch.zeros_like(e)
        gate = gates_of_rows(part, dim, seed, draw, p).cuda()
        assert near(y[a:b], (e + q) * gate, (e.abs() + q.abs()) * gate, ot), a


def check_grad(tok, dy, grad, base, vocab, scale, gate):
    """Against the definition in 64 bits on the GPU (the order of its additions does not matter there)."""
    dim = dy.shape[1]
    there = (tok >= 0) & (tok < vocab)
    terms = torch.bincount(tok[there], minlength=vocab)[:, None].double()
    for c in torch.arange(dim).split(256):
        cols = slice(int(c[0]), int(c[-1]) + 1)
        v = dy[:, cols].double() * (gate[:, cols].cuda() if gate is not None else 1.0)
        want = base[:, cols].double() if base is not None else torch.zeros(vocab, len(c), dtype=torch.float64, device="cuda")
        mag = want.abs()
        want = want.index_add(0, tok[there], scale * v[there])
        mag = mag.index_add(0, tok[there], abs(scale) * v[there].abs())
        assert bool(((grad[:, cols].double() - want).abs() <= U * want.abs() * (1 + U) + (terms + 6) * U * mag + 2.0 ** -125).all()), cols


# one block's sort and a sort by tiles, rows without a token left for every one of the launches (a base, or a table of more than 176 MB, for the last ones); tables whose marks one
# block does not clear, with three digits; columns that rows begin off 16 bytes with
@pytest.mark.parametrize("n, vocab, dim, kind", [(2000, 50257, 1024, "skewed"), (8000, 50257, 1024, "bad"), (9000, 50257, 1024, "skewed"), (20000, 50257, 1024, "skewed"), (20000, 50257, 1024, "bad"),
                                                 (2000, (1 << 20) + 5, 8, "any"), (30000, (1 << 20) + 5, 64, "bad"), (20000, 70000, 1001, "skewed"), (3000, 40000, 1002, "any")])
@pytest.mark.parametrize("t, p, base", [("bf16", 0.1, False), ("f32", 0.0, True), ("f32", 0.1, False), ("f16", 0.0, True)])
def test_embed_grad_of_large_tables(n, vocab, dim, kind, t, p, base):
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    g = gen(n + dim)
    tok = tokens_of(g, n, vocab, kind)
    dy = torch.randn(n, dim, generator=g, device="cuda").to(t)
    b = torch.randn(vocab, dim, generator=g, device="cuda") if base else None
    # (rows that nobody writes show: NaN; so do places of the workspace that nobody wrote)
    grad = torch.full((vocab, dim), float("nan"), device="cuda")
    ws = torch.full((dblp.embed_grad_workspace(n, vocab, dim),), 0xA5, dtype=torch.uint8, device="cuda")
    dblp.embed_grad(tok, dy, grad, ws, scale=0.5, drop=dblp.Drop(5, 6, p), base=b)
    gate = ref.gates(n, dim, 5, 6, p) if p else None
    check_grad(tok, dy, grad, b, vocab, 0.5, gate)
    first, marks = grad.clone(), 0xFF
    grad.fill_(float("nan"))
    ws.fill_(marks)
    dblp.embed_grad(tok, dy, grad, ws, scale=0.5, drop=dblp.Drop(5, 6, p), base=b)
    assert torch.equal(first, grad)
    if base:                                                           # in place: rows without a token keep their bits
        over = b.clone()
        dblp.embed_grad(tok, dy, over, ws, scale=0.5, drop=dblp.Drop(5, 6, p), base=over)
        assert torch.equal(over, first)


def test_embed_grad_with_more_chains_than_blocks():
    """40 tokens of 32 places and 32768 columns: each chain takes 256 blocks' worth, together more than the launch has."""
    import paper_2605_01989_amd as dblp
    g, vocab, dim = gen(43), 45, 32768
    tok = torch.arange(40, device="cuda").repeat_interleave(32)[torch.randperm(1280, generator=g, device="cuda")]
    dy = torch.randn(1280, dim, generator=g, device="cuda").bfloat16()
    grad = torch.full((vocab, dim), float("nan"), device="cuda")
    ws = torch.full((dblp.embed_grad_workspace(1280, vocab, dim),), 0xA5, dtype=torch.uint8, device="cuda")
    dblp.embed_grad(tok, dy, grad, ws)
    check_grad(tok, dy, grad, None, vocab, 1.0, None)


def test_embed_grad_of_more_units_than_a_launch_has():
    """2^22 rows of 2048 columns: 2^31 units.  Rows without a token are zeros, all of them; 600 places are too many for the single launch."""
    import paper_2605_01989_amd as dblp
    g, vocab, dim = gen(44), 1 << 22, 2048
    for n in (600, 40):
        tok = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        tok[:4] = torch.tensor([0, vocab - 1, 4194302, 4194303], device="cuda")
        dy = torch.randn(n, dim, generator=g, device="cuda")
        grad = torch.full((vocab, dim), float("nan"), device="cuda")
        ws = torch.full((dblp.embed_grad_workspace(n, vocab, dim),), 0xA5, dtype=torch.uint8, device="cuda")
        dblp.embed_grad(tok, dy, grad, ws)
        rows = tok.unique()
        want = torch.zeros(len(rows), dim, dtype=torch.float64, device="cuda").index_add(0, torch.searchsorted(rows, tok), dy.double())
        assert bool(((grad[rows].double() - want).abs() <= n * 8 * U * want.abs().clamp(min=10.0)).all())
        grad[rows] = 0.0
        assert all(not bool(part.any()) for part in grad.split(1 << 16))
        del grad
    torch.cuda.empty_cache()


def test_rows_of_more_units_than_a_launch_has():
    """2^30 + 100 rows of 16 columns, two units each: dropout in place and embedding, in two launches."""
    import paper_2605_01989_amd as dblp
    g, rows, cols, seed, draw, p = gen(45), (1 << 30) + 100, 16, 5, 6, 0.25
    border = (2**31 - 1) // 2
    tok = torch.randint(0, 999, (rows,), generator=g, device="cuda")
    table = torch.randn(1000, cols, generator=g, device="cuda").bfloat16()
    x = torch.full((rows, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    dblp.embed(tok, table, x)
    for a in range(0, rows, 1 << 25):
        assert torch.equal(x[a : a + (1 << 25)], table[tok[a : a + (1 << 25)]]), a
    for drop in (True, False):                                         # the embedding under the mask, then dropout in place, of the same values
        if drop:
            dblp.embed(tok, table, x, drop=dblp.Drop(seed, draw, p))
        else:
            dblp.embed(tok, table, x)
            dblp.dropout(x, x, dblp.Drop(seed, draw, p))
        for a in (0, border - 300, rows - 300):
            part = torch.arange(a, a + 300)
            e = table[tok[a : a + 300]].double() * gates_of_rows(part, cols, seed, draw, p).cuda()
            assert near(x[a : a + 300], e, e.abs(), torch.bfloat16), (drop, a)
    del x, tok
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t, n, vocab, part", [("bf16", 2700, 50257, 900), ("f16", 54000, 2500, 9000), ("f32", 20100, 3500, 6700), ("f32", 2700, 25600, 900), ("bf16", 20100, 6800, 6700), ("bf16", 13200, 10500, 3300)])
def test_scores_past_the_cache(t, n, vocab, part):
    """The bits of smaller calls on the same rows, and the definition."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    assert n * vocab * t.itemsize > CACHE > part * vocab * t.itemsize and part >= 768
    g = gen(46)
    x = torch.randn(n, vocab, generator=g, device="cuda").mul_(3).to(t)
    target = torch.randint(-2, vocab + 2, (n,), generator=g, device="cuda")
    x[3, : vocab // 2] = -float("inf")
    x[4] = -float("inf")
    ws = torch.full((dblp.logits_workspace(n, vocab),), 0xA5, dtype=torch.uint8, device="cuda")
    logp, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dblp.token_logprobs(x, target, logp, ws, lse=lse)
    for a in range(0, n, part):
        lp, l = torch.empty(part, device="cuda"), torch.empty(part, device="cuda")
        dblp.token_logprobs(x[a : a + part], target[a : a + part], lp, ws, lse=l)
        assert torch.equal(lp, logp[a : a + part]) and torch.equal(l, lse[a : a + part]), a
        want = x[a : a + part].double().logsumexp(1)
        there = (target[a : a + part] >= 0) & (target[a : a + part] < vocab) & torch.isfinite(want)
        assert float((l.double() - want)[there].abs().max()) <= (3 * 40 + 66 + vocab / 64) * U + U * 30


@pytest.mark.parametrize("t, n, vocab, part", [("bf16", 1400, 50264, 200), ("f16", 1400, 50264, 200), ("f32", 1100, 33000, 220), ("bf16", 140000, 512, 20000), ("f32", 140000, 256, 20000), ("f32", 400, 90112, 200), ("bf16", 400, 180224, 200),
                                               ("bf16", 9000, 8192, 1800), ("f32", 800, 50260, 200), ("bf16", 960, 90112, 160)])
def test_policy_loss_past_the_cache(t, n, vocab, part):
    """Rows on multiples of 16 bytes, apart and in place: the bits of smaller calls on the same rows, and the sums of theirs."""
    import paper_2605_01989_amd as dblp
    t = TYPES[t]
    assert n * vocab * t.itemsize > CACHE / 2 > part * vocab * t.itemsize and vocab * t.itemsize % 16 == 0 and part >= 128 and n % part == 0
    g = gen(47)
    x = torch.randn(n, vocab, generator=g, device="cuda").mul_(3).to(t)
    target = torch.randint(-1, vocab, (n,), generator=g, device="cuda")
    adv, w = torch.randn(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    w[5] = 0.0
    x[6] = -float("inf")
    old, back = torch.randn(n, generator=g, device="cuda") * 0.3 - 9, torch.randn(n, generator=g, device="cuda") * 0.3 - 9
    ws = torch.full((dblp.logits_workspace(n, vocab),), 0xA5, dtype=torch.uint8, device="cuda")

    def run(s, logits, d):
        stats, logp = torch.full((5,), 9.0, device="cuda"), torch.full((len(target[s]),), 9.0, device="cuda")
        dblp.policy_loss(logits, target[s], adv[s], w[s], stats, ws, old_logp=old[s], ref_logp=back[s], dlogits=d, logp=logp, clip=(0.2, 0.3), kl_coef=0.1)
        return stats, logp
    d = torch.full_like(x, 7.0)
    stats, logp = run(slice(0, n), x, d)
    total, mags = torch.zeros(5, dtype=torch.float64, device="cuda"), torch.zeros(5, dtype=torch.float64, device="cuda")
    for a in range(0, n, part):
        s = slice(a, a + part)
        small = torch.full_like(x[s], 5.0)
        st, lp = run(s, x[s], small)
        assert torch.equal(small, d[s]) and torch.equal(lp, logp[s]), a
        total += st.double()
        mags += st.double().abs()
    assert bool(((stats.double() - total).abs() <= 3 * U * mags).all())
    over, lp = run(slice(0, n), x, x)
    assert torch.equal(x, d) and torch.equal(over, stats) and torch.equal(lp, logp)
