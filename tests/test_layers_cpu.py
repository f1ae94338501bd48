"""No-GPU checks of the layers' operators: the header and its binding agree, bad arguments are refused before the device is touched."""
import os
import re

import pytest
import torch

import paper_2605_01989_amd as dblp
from paper_2605_01989_amd import binding, layers

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dblp_layers.h")
A, B, C = 1 << 20, 1 << 21, 1 << 22            # addresses that are never read: every call here is refused
BIG = 1 << 31


def test_library_exports_what_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(dblp_[a-z_0-9]+)\s*\(", text)))
    assert sorted(layers.EXPORTS) == names and len(names) == 7
    for n in names:
        assert hasattr(dblp.lib(), n), n
    defines = dict(re.findall(r"^#define\s+DBLP_ACT_([A-Z_]+)\s+(\d+)", text, flags=re.M))
    assert {k.lower(): int(v) for k, v in defines.items()} == {k or "none": v for k, v in layers.ACTIVATIONS.items()}


def _call(name, a):
    layers._load()
    return getattr(dblp.lib(), name)(0, None, *a.values())


def _linear(**k):
    a = dict(n=4, inner=8, outer=6, x=A, xs=8, w=A, ws=8, type=0, bias=None, bt=0, act=0, r=None, rs=0, y=B, ys=6, z=None, zs=0, ot=0, space=C, bytes=1 << 40)
    return _call("dblp_linear", {**a, **k})


def _grad_input(**k):
    a = dict(n=4, inner=8, outer=6, dy=A, ds=6, w=A, ws=8, type=0, z=None, zs=0, act=0, base=None, bs=0, dx=B, xs=8, ot=0, space=C, bytes=1 << 40)
    return _call("dblp_linear_grad_input", {**a, **k})


def _grad_weight(**k):
    a = dict(n=4, inner=8, outer=6, dy=A, ds=6, x=A, xs=8, type=0, base=None, bs=0, dw=B, ws=8, bb=None, db=None, space=C, bytes=1 << 40)
    return _call("dblp_linear_grad_weight", {**a, **k})


def _activation(**k):
    a = dict(rows=4, cols=8, dy=A, ds=8, z=A, zs=8, act=1, dz=B, os=8, type=0)
    return _call("dblp_activation_grad", {**a, **k})


def _table(*v):
    import ctypes
    return (ctypes.c_double * len(v))(*v)


def _orthogonal(**k):
    a = dict(count=2, rows=4, cols=8, g=A, gs=8, gstep=32, gt=0, table=None, steps=5, scale=1.0, base=None, bs=0, bstep=0, bscale=1.0, out=B, os=8, ostep=32, ot=0, space=C, bytes=1 << 40)
    return _call("dblp_orthogonalize", {**a, **k})


NAN, INF = float("nan"), float("inf")
WORKSPACE = [dict(space=None), dict(space=C + 16), dict(bytes=0)]
REFUSED = [
    (_linear, [dict(type=3), dict(ot=-1), dict(ot=1), dict(type=1, ot=2), dict(bias=A, bt=7), dict(act=5), dict(act=-1), dict(n=BIG), dict(inner=BIG), dict(outer=BIG), dict(x=None), dict(w=None),
               dict(y=None), dict(x=A + 2), dict(w=A + 1, type=1, ot=1), dict(y=B + 2), dict(r=A + 2, rs=6), dict(z=C + 2, zs=6), dict(bias=A + 1, bt=2), dict(ys=5), dict(z=C, zs=5),
               dict(z=B, zs=6), dict(r=B, rs=7), *WORKSPACE]),
    (_grad_input, [dict(type=3), dict(ot=1), dict(type=2, ot=1), dict(act=9, z=A, zs=8), dict(act=1), dict(n=BIG), dict(inner=BIG), dict(outer=BIG), dict(dy=None), dict(w=None), dict(dx=None),
                   dict(dy=A + 2), dict(w=A + 2), dict(z=A + 1, zs=8), dict(base=A + 2, bs=8), dict(dx=B + 1), dict(xs=7), dict(z=B, zs=9), dict(base=B, bs=0), *WORKSPACE]),
    (_grad_weight, [dict(type=3), dict(n=BIG), dict(inner=BIG), dict(outer=BIG), dict(bb=A), dict(dy=None), dict(x=None), dict(dw=None), dict(dy=A + 2), dict(x=A + 1, type=1), dict(base=A + 2, bs=8),
                    dict(dw=B + 2), dict(db=A + 2), dict(bb=A + 1, db=A), dict(ws=7), dict(base=B, bs=16), *WORKSPACE]),
    (_activation, [dict(type=3), dict(act=5), dict(rows=BIG), dict(cols=BIG), dict(dy=None), dict(z=None), dict(dz=None), dict(dy=A + 2), dict(z=A + 1, type=1), dict(dz=B + 1), dict(os=7), dict(dz=A, os=9)]),
    (_orthogonal, [dict(gt=3), dict(ot=-1), dict(count=BIG), dict(rows=BIG), dict(cols=BIG), dict(count=1 << 30, rows=1 << 20, cols=1 << 20), dict(steps=17), dict(steps=1 << 31), dict(scale=NAN), dict(scale=INF),
                   dict(bscale=INF), dict(g=None), dict(out=None), dict(g=A + 2), dict(base=A + 2, bs=8, bstep=32), dict(out=B + 1, ot=1), dict(os=7), dict(ostep=31), dict(ostep=0),
                   dict(base=B, bs=9, bstep=32), dict(base=B, bs=8, bstep=40), dict(g=B, gt=1), dict(g=B, gs=9), dict(g=B, gstep=33), *WORKSPACE,
                   dict(steps=1, table=_table(40.0, 0.0, 0.0)), dict(steps=2, table=_table(20.0, 0.0, 0.0, 2.0, 0.0, 0.0)), dict(steps=1, table=_table(NAN, 0.0, 0.0)), dict(steps=1, table=_table(1.0, INF, 0.0)),
                   dict(steps=1, table=_table(1e3, -2e3, 1e3))]),
]


@pytest.mark.parametrize("call, k", [(c, k) for c, ks in REFUSED for k in ks], ids=lambda v: v.__name__ if callable(v) else "-".join(v))
def test_refusals(call, k):
    assert call(**k) == binding.EINVAL
    assert dblp.lib().dblp_worker_error().decode().split(":")[0] in ("linear", "linear_grad_input", "linear_grad_weight", "activation_grad", "orthogonalize")


def test_nothing_to_do_needs_no_device():
    assert _linear(n=0) == binding.OK and _linear(outer=0, y=None, w=None) == binding.OK
    assert _grad_input(n=0) == binding.OK and _grad_input(inner=0, dx=None) == binding.OK
    assert _grad_weight(outer=0) == binding.OK and _grad_weight(inner=0) == binding.OK
    assert _activation(rows=0) == binding.OK and _activation(cols=0, dy=None) == binding.OK
    assert _orthogonal(count=0) == binding.OK and _orthogonal(rows=0, g=None) == binding.OK and _orthogonal(cols=0) == binding.OK


def test_workspaces():
    for sizes in ((0, 1, 1), (1, 0, 0), (100, 7, 50257)):
        assert dblp.linear_workspace(*sizes) > 0 and dblp.orthogonalize_workspace(*sizes) > 0
    L = layers._load()
    for bad in ((BIG, 1, 1), (1, BIG, 1), (1, 1, BIG)):
        assert L.dblp_linear_workspace(*bad) == 0 and L.dblp_orthogonalize_workspace(*bad) == 0


def test_a_workspace_of_a_larger_call_is_large_enough():
    counts = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 512, 513, 768, 1000, 1024, 2304, 4096, 5000, 8192, 16384, 16385, 32768, 50257, 65536, 10**6]
    for f, tops in ((dblp.linear_workspace, counts), (dblp.orthogonalize_workspace, [c for c in counts if c < 70000])):
        for a in (1, 5, 64, 300, 768, 4096, 50257):
            for b in (1, 17, 128, 768, 5000):
                for sizes in ([f(n, a, b) for n in tops], [f(a, n, b) for n in tops], [f(a, b, n) for n in tops]):
                    assert sizes == sorted(sizes)


def test_binding_refuses_what_the_library_cannot_see():
    x, w, v = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(8)
    y = torch.zeros(4, 6)
    space = torch.zeros(1 << 16, dtype=torch.uint8)
    for f in (lambda: dblp.linear(x, w, y, space), lambda: dblp.linear_grad_input(y, w, x, space), lambda: dblp.linear_grad_weight(y, x, w, space),
              lambda: dblp.activation_grad(x, x, x, "silu"), lambda: dblp.orthogonalize(x, x, space), lambda: dblp.linear(v, w, y, space), lambda: dblp.linear_grad_input(v, w, x, space),
              lambda: dblp.linear_grad_weight(v, x, w, space), lambda: dblp.activation_grad(v, v, v, None), lambda: dblp.orthogonalize(v, v, space)):
        with pytest.raises(dblp.DblpError) as e:
            f()
        assert e.value.code == binding.EINVAL
    for name in ("tanh", 1, "none", ["relu"]):
        with pytest.raises(dblp.DblpError):
            layers._activation(name)
    meta = torch.empty(2, 4, 8, device="meta")
    assert layers._matrices("m", meta, meta.device, (2, 4, 8))[1:] == (8, 32) and layers._matrices("m", meta[0], meta.device, None)[1:] == (8, 0)
    for bad, shape in ((meta, (4, 8)), (torch.empty(8, device="meta"), None), (torch.empty(2, 8, 4, device="meta").transpose(1, 2), None), (meta.int(), None), (meta[None], None)):
        with pytest.raises(dblp.DblpError):
            layers._matrices("m", bad, meta.device, shape)
    with pytest.raises(dblp.DblpError):
        layers._sizes(4, 1 << 32)


def test_coefficients_are_looked_over():
    """The bound of a polynomial's values lies at a border or between: of each kind one that is taken and one that is not."""
    ok = dict(space=None)                          # (refused for the workspace alone, after the coefficients)
    for table, taken in ((_table(31.9, 0.0, 0.0), True), (_table(0.0, 0.0, -31.0), True), (_table(90.0, -90.0, 0.0), False), (_table(80.0, -80.0, 0.0), True), (_table(100.0, -190.0, 91.0), True),
                         (_table(200.0, -390.0, 191.0), False), (_table(-33.0, 0.0, 0.0), False)):
        assert _orthogonal(steps=1, table=table, **ok) == binding.EINVAL
        assert (b"workspace" in dblp.lib().dblp_worker_error()) == taken, list(table)
