"""Host side of the adapters', heads' and gradient calls, without a GPU: what
they refuse, that a refused call launches nothing, what they launch, and the
workspaces they ask for (the HIP runtime is the stand-in of ``fake_hip.cpp``)."""

import numpy as np
import pytest

from fakehip import fake_hip, run  # noqa: F401

torch = pytest.importorskip("torch")

import paper_2607_21985_amd as spdp  # noqa: E402

BODY = """
S = ctypes.c_size_t
def bank(rows=256, cols=128, count=4, rank=8, a=1 << 36, b=1 << 37, scale=1 << 38):
    return spdp._Bank(a, b, scale, rows, cols, count, rank)
def banks(*m):
    return (spdp._Bank * len(m))(*m)
def ptrs(*p):
    return (ctypes.c_void_p * len(p))(*p)
IDS, WS, H = 1 << 39, 1 << 46, 1 << 45
BASE, OUT = 1 << 41, 1 << 42
def need(m, n, ids=1):
    s = S(77)
    st = L.spdp_adapt_workspace(banks(*m), len(m), n, ids, ctypes.byref(s))
    return st, s.value
def adapt(m=None, n=40, ids=IDS, x=None, base=None, y=None, h=None, ws=WS, room=None, k=None):
    m = m or [bank()]
    k = len(m) if k is None else k
    room = need(m, n, ids is not None)[1] if room is None else room
    x = x or [X] * len(m)
    base = base or [BASE + (i << 30) for i in range(len(m))]
    y = y or [OUT + (i << 30) for i in range(len(m))]
    return L.spdp_adapt(banks(*m), k, ptrs(*x), ids, ptrs(*base), ptrs(*y), ptrs(*h) if h else None, n, ws, room, None)
def grad(m=None, n=40, ids=IDS, x=X, h=H, dy=Y, base=BASE, dx=OUT, da=1 << 47, db=1 << 48, ws=WS, room=None):
    m = m or bank()
    s = S()
    st = L.spdp_adapt_grad_workspace(ctypes.byref(m), n, ids is not None, ctypes.byref(s))
    room = s.value if room is None else room
    return L.spdp_adapt_grad(ctypes.byref(m), x, ids, h, dy, base, dx, da, db, n, ws, room, None)
def rotation(pos=1 << 36, c=1 << 37, s=1 << 38, table=64, dim=128, rot=128, inter=0, eps=1e-6):
    return spdp._Rotation(pos, c, s, table, dim, rot, inter, eps)
def heads(*m):
    return (spdp._Heads * len(m))(*m)
def one(x=X, w=0, dy=0, y=OUT, dw=0, n=8):
    return spdp._Heads(x, w, dy, y, dw, n)
def rotate(m=None, r=None, n=16, k=None):
    m, r = m or [one()], r or rotation()
    return L.spdp_rotate_heads(heads(*m), len(m) if k is None else k, ctypes.byref(r), n, None)
def rotate_grad(m, r=None, n=16, ws=WS, room=None):
    r, s = r or rotation(), S()
    st = L.spdp_rotate_heads_grad_workspace(heads(*m), len(m), ctypes.byref(r), n, ctypes.byref(s))
    return L.spdp_rotate_heads_grad(heads(*m), len(m), ctypes.byref(r), n, ws, s.value if room is None else room, None)
def expect(label, want, got):
    out[label] = [want, got, [k for k, _ in launches()]]
"""
INVALID, UNSUPPORTED = -1, -2


def _refused(fake_hip, body):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, body]))
    assert out
    wrong = {k: v for k, v in out.items() if v[0] != v[1] or v[2]}
    assert not wrong, wrong


def test_adapt_refusals(fake_hip):  # noqa: F811
    _refused(fake_hip, """
log()
I, U = -1, -2
expect("no bank", I, L.spdp_adapt(None, 1, ptrs(X), IDS, ptrs(BASE), ptrs(OUT), None, 4, WS, 1 << 20, None))
expect("0 banks", I, adapt(k=0))
expect("9 banks", I, adapt([bank() for _ in range(9)], room=1 << 30))
expect("no X", I, L.spdp_adapt(banks(bank()), 1, None, IDS, ptrs(BASE), ptrs(OUT), None, 4, WS, 1 << 20, None))
for f in ("a", "b", "scale"):
    expect("no " + f, I, adapt([bank(**{f: None})], room=1 << 30))
for f in ("rows", "cols", "count", "rank"):
    expect("0 " + f, I, adapt([bank(**{f: 0})], room=1 << 30))
expect("rank 129", U, adapt([bank(rank=129)], room=1 << 30))
expect("2049 adapters", U, adapt([bank(count=2049)], room=1 << 30))
expect("rows", U, adapt([bank(rows=(1 << 24) + 1)], room=1 << 30))
expect("mixed ranks", I, adapt([bank(), bank(rank=9)], room=1 << 30))
expect("mixed counts", I, adapt([bank(), bank(count=5)], room=1 << 30))
expect("0 tokens", I, adapt(n=0, room=1 << 30))
expect("tokens", U, adapt(n=(1 << 20) + 1, room=1 << 30))
expect("null entry", I, adapt(x=[None]))
expect("null output", I, adapt(y=[None]))
expect("null h", I, adapt(h=[None]))
expect("no workspace", I, adapt([bank(cols=4096)], n=200, ws=None))
expect("small workspace", I, adapt(n=200, room=need([bank()], 200)[1] - 1))
expect("odd workspace", I, adapt(n=200, ws=WS + 128))
expect("Y in X", I, adapt(y=[X + 40 * 128 * 2 - 2]))
expect("Y partly in its base", I, adapt(y=[BASE + 512]))
expect("Y in another's base", I, adapt([bank(), bank()], y=[OUT, BASE]))
expect("equal Y", I, adapt([bank(), bank()], y=[OUT, OUT]))
expect("h in Y", I, adapt(h=[OUT + 64]))
expect("h in X", I, adapt(h=[X]))
expect("size without a place", I, L.spdp_adapt_workspace(banks(bank()), 1, 4, 1, None))
""")


def test_adapt_grad_refusals(fake_hip):  # noqa: F811
    _refused(fake_hip, """
log()
I, U = -1, -2
for f in ("x", "h", "dy", "base", "dx", "da", "db"):
    expect("no " + f, I, grad(**{f: None}))
expect("rank", U, grad(bank(rank=200), room=1 << 30))
expect("0 tokens", I, grad(n=0, room=1 << 30))
expect("no workspace", I, grad(ws=None))
expect("small workspace", I, grad(room=8))
expect("dx in dy", I, grad(dx=Y + 16))
expect("dx is x", I, grad(dx=X))
expect("dx is x and base", I, grad(dx=X, base=X))
expect("dx partly in its base", I, grad(dx=BASE + 16))
expect("da in db", I, grad(da=1 << 47, db=(1 << 47) + 64))
expect("da in a", I, grad(da=1 << 36))
expect("db in h", I, grad(db=H))
""")


def test_heads_refusals(fake_hip):  # noqa: F811
    _refused(fake_hip, """
log()
I, U = -1, -2
expect("no inputs", I, L.spdp_rotate_heads(None, 1, ctypes.byref(rotation()), 4, None))
expect("no rotation", I, L.spdp_rotate_heads(heads(one()), 1, None, 4, None))
expect("0 inputs", I, rotate(k=0))
expect("9 inputs", I, rotate([one() for _ in range(9)]))
for f in ("pos", "c", "s"):
    expect("no " + f, I, rotate(r=rotation(**{f: None})))
expect("0 tokens", I, rotate(n=0))
expect("no table", I, rotate(r=rotation(table=0)))
for d, r in ((0, 0), (3, 2), (8, 0), (8, 3), (8, 10), (-2, -2)):
    expect(f"dim {d} rot {r}", I, rotate(r=rotation(dim=d, rot=r)))
expect("dim 514", U, rotate(r=rotation(dim=514, rot=2)))
for e in (-1.0, float("nan"), float("inf")):
    expect(f"eps {e}", I, rotate(r=rotation(eps=e)))
expect("no x", I, rotate([one(x=None)]))
expect("no y", I, rotate([one(y=None)]))
expect("0 heads", I, rotate([one(n=0)]))
expect("heads", U, rotate([one(n=65537)]))
expect("y partly x", I, rotate([one(y=X + 2)]))
expect("equal y", I, rotate([one(), one(x=Y)]))
expect("y in another x", I, rotate([one(), one(x=OUT, y=Y)]))
expect("y in the weight", I, rotate([one(w=OUT + 8)]))
expect("y in the positions", I, rotate(r=rotation(pos=OUT)))
expect("no dy", I, rotate_grad([one()]))
expect("weight without gradient", I, rotate_grad([one(dy=Y, w=1 << 35)]))
expect("gradient without weight", I, rotate_grad([one(dy=Y, dw=1 << 35)]))
expect("no workspace", I, rotate_grad([one(dy=Y, w=1 << 35, dw=1 << 34)], ws=None))
expect("small workspace", I, rotate_grad([one(dy=Y, w=1 << 35, dw=1 << 34)], room=4))
expect("y partly dy", I, rotate_grad([one(dy=OUT + 2)]))
expect("one gradient for two weights", I, rotate_grad([one(dy=Y, w=1 << 35, dw=1 << 34),
    one(x=X + (1 << 32), dy=Y, y=OUT + (1 << 32), w=1 << 35, dw=1 << 34)]))
expect("gradient in x", I, rotate_grad([one(dy=Y, w=1 << 35, dw=X + 16)]))
""")


def test_spmm_grad_refusals(fake_hip):  # noqa: F811
    _refused(fake_hip, """
I, U = -1, -2
m = ones(700, 328, (256, 16), 0.5)
s = S()
assert L.spdp_spmm_grad_workspace(m._h, 90, ctypes.byref(s)) == 0 and s.value > 0
bad = ones(64, 64, (128, 16))
codes = spdp.encode_rtn(np.ones((256, 64), np.float16), (256, 16), 4)
host = spdp.encode_host(np.ones((256, 64), np.float16), (256, 16))
log()
go = lambda h, dy=X, n=90, dx=Y, ws=WS, room=s.value: L.spdp_spmm_grad(h, dy, n, dx, ws, room, None)
expect("no handle", I, go(None))
expect("host", I, go(host._h))
expect("tile", U, go(bad._h))
expect("codes", U, go(codes._h))
expect("0 tokens", I, go(m._h, n=0))
expect("tokens", U, go(m._h, n=65535 * 32 + 1))
expect("no dY", I, go(m._h, dy=None))
expect("odd dX", I, go(m._h, dx=Y + 2))
expect("overlap", I, go(m._h, dx=X + 1024))
expect("no workspace", I, go(m._h, ws=None))
expect("small workspace", I, go(m._h, room=s.value - 1))
expect("odd workspace", I, go(m._h, ws=WS + 16))
expect("no place", I, L.spdp_spmm_grad_workspace(m._h, 90, None))
""")


def test_what_the_calls_launch(fake_hip):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, """
def names():
    return [next(k for k in ("sort", "shrink", "expand", "pack", "outer_reduce", "outer", "heads_sum", "heads", "grad_plain", "grad", "reduce")
                 if k in name) for name, _ in launches()]
log()
assert adapt(n=1) == 0
out["one token"] = names()
assert adapt([bank(cols=8192, rank=32)], n=1) == 0
out["a large first factor"] = names()
assert adapt([bank(count=1)], n=64) == 0
out["64 of one adapter"] = names()
assert adapt([bank(cols=4096, count=1)], n=64) == 0
out["64"] = names()
assert adapt(n=65) == 0
out["65"] = names()
assert adapt([bank(cols=4096)], n=65) == 0
out["65, wide"] = names()
assert adapt([bank(cols=4096)], n=500, ids=None, y=[BASE], h=[H], room=1 << 30) == 0
out["one adapter"] = names()
assert grad(n=4, dx=BASE) == 0
out["grad"] = names()
assert grad(n=600) == 0
out["grad of 600"] = names()
assert grad(bank(count=1), n=4096, ids=None) == 0
out["grad of many tokens"] = names()
assert rotate([one(y=X), one(x=Y, y=Y + (1 << 30))]) == 0
out["heads"] = names()
assert rotate_grad([one(dy=Y, w=1 << 35, dw=1 << 34)]) == 0
out["heads grad"] = names()
assert rotate_grad([one(dy=Y)], ws=None) == 0
out["heads grad without weights"] = names()
out["mallocs"] = sum(l[0] == "malloc" for l in log())
# the workspace that is asked for suffices whatever the sizes, and the queries agree
hip.fake_cus(256)
for n in (1, 31, 64, 65, 1000, 5000, 1 << 20):
    for rank in (1, 17, 128):
        for count in (1, 64, 2048):
            for ids in (0, 1):
                assert need([bank(rank=rank, count=count)], n, ids)[0] == 0
"""]))
    assert out["one token"] == out["64 of one adapter"] == ["expand"]
    assert out["a large first factor"] == out["64"] == out["one adapter"] == ["shrink", "expand"]
    assert out["65"] == ["sort", "expand"] and out["65, wide"] == ["sort", "shrink", "expand"]
    assert out["grad"] == ["sort", "shrink", "expand", "outer"]
    assert out["grad of 600"] == ["sort", "shrink", "expand", "pack", "outer"]
    assert out["grad of many tokens"] == ["shrink", "expand", "pack", "outer", "outer_reduce"]
    assert out["heads"] == out["heads grad without weights"] == ["heads"]
    assert out["heads grad"] == ["heads", "heads_sum"]
    assert out["mallocs"] == 0


def test_handles_without_records_take_the_plain_form(fake_hip):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, """
def go(m):
    s = S()
    assert L.spdp_spmm_grad_workspace(m._h, 90, ctypes.byref(s)) == 0
    log()
    assert L.spdp_spmm_grad(m._h, X, 90, Y, WS, s.value, None) == 0
    return [k for k, _ in launches()]
m = ones(700, 328, (256, 16), 0.5)
out["with"] = go(m)
used = hip.fake_used()
m.close()
hip.fake_budget(hip.fake_used() + used - 20000)
m = ones(700, 328, (256, 16), 0.5)
out["without"] = go(m)
"""]))
    assert any("grad_kernel" in k for k in out["with"]) and any("grad_plain" in k for k in out["without"]), out


def test_binding_refuses_host_tensors_and_shapes():
    f = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    with pytest.raises(ValueError):
        spdp.Adapters(f(2, 4, 8), f(2, 4, 8), torch.zeros(2))  # not on a GPU
    with pytest.raises(TypeError):
        spdp.Adapters(f(2, 4, 8).float(), f(2, 4, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        spdp.Adapters(f(2, 4, 8), f(2, 3, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        spdp.Adapters(f(4, 8), f(4, 8), torch.zeros(4))
    with pytest.raises(ValueError):
        spdp.Adapters(f(2, 8, 4).transpose(1, 2), f(2, 4, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        spdp.adapters_many([], [], None, [], [])
    pos, tab = torch.zeros(3, dtype=torch.int32), torch.zeros(5, 4)
    for bad in (dict(xs=[f(3, 12)]), dict(xs=[f(3, 0)]), dict(pos=pos[:2]), dict(cos=tab[0]), dict(sin=tab[:, :2]),
                dict(weights=[f(8), f(8)]), dict(xs=[]), dict(ys=[f(3, 8)]), dict(dim=0)):
        args = dict(xs=[f(3, 16)], dim=8, pos=pos, cos=tab, sin=tab, ys=[f(3, 16)])
        args.update(bad)
        with pytest.raises(ValueError):
            spdp.rotate_heads(**args)
    with pytest.raises(ValueError):  # not on a GPU
        spdp.rotate_heads([f(3, 16)], 8, pos, tab, tab, [f(3, 16)])
    with pytest.raises(TypeError):
        spdp.rotate_heads([f(3, 16)], 8, pos.long(), tab, tab, [f(3, 16)])
    m = spdp.encode_host(np.ones((64, 16), np.float16), (64, 16))
    with pytest.raises(ValueError):
        m.spmm_grad_into(f(3, 64), f(3, 16))
    with pytest.raises(ValueError):
        m.spmm_grad_into(f(3, 65), f(3, 16))
    m.close()
