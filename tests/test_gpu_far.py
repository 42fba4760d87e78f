"""Arrays of more than 2^31 numbers, wide matrices, and drawn sizes, against
the float64 oracle (for the large ones at some tokens)."""

import numpy as np
import pytest

from oracle import layer

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2607_21985_amd as spdp  # noqa: E402


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _np(t):
    return t.cpu().numpy()


def _rows(n):
    return np.unique(np.concatenate([np.arange(3), np.linspace(0, n - 1, 40).astype(int), np.arange(n - 3, n)]))


def _filled(n, width, scale=1.0):
    """fp16 [n, width] of normal numbers, part by part (no fp32 copy of it all)."""
    t = torch.empty(n, width, dtype=torch.float16, device="cuda")
    for part in t.split(max(1, (1 << 28) // width)):
        part.copy_(scale * torch.randn(part.shape, device="cuda"))
    return t


def test_adapters_beyond_32_bits():
    n, rows, cols, count, rank = 290_000, 8200, 72, 3, 5
    assert n * rows > 1 << 31
    rng = np.random.default_rng(1)
    a, b = (rng.normal(size=(count, rank, w)).astype(np.float16) for w in (cols, rows))
    scale, ids = np.array([0.5, 1.0, -2.0], dtype=np.float32), rng.integers(-1, count, n).astype(np.int32)
    m = spdp.Adapters(_dev(a), _dev(b), _dev(scale))
    x, base, di = _filled(n, cols, 0.3), _filled(n, rows), _dev(ids)
    y, h = torch.empty_like(base), torch.empty(n, rank, device="cuda")
    m.add_into(x, di, base, y, h=h)
    at = _rows(n)
    sel = torch.from_numpy(at).cuda()
    want, bound, hw, hb = layer.adapt(_np(x[sel]), ids[at], _np(base[sel]), a, b, scale)
    assert np.all(np.abs(_np(y[sel]) - want) <= bound) and np.all(np.abs(_np(h[sel]) - hw) <= hb)
    # backward: dY is the large array
    del base
    dx, da, db = torch.empty_like(x), torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    m.grad_into(x, di, h, y, x, dx, da, db)
    want, bound = layer.adapt_grad(_np(x[sel]), ids[at], _np(h[sel]), _np(y[sel]), _np(x[sel]), a, b, scale)[0]
    assert np.all(np.abs(_np(dx[sel]) - want) <= bound)
    # db of the last columns, in 64 bits: the sum over all tokens of an adapter
    own = torch.from_numpy(np.flatnonzero(ids == 2)).cuda()
    z, act = y[own, -8:].double(), h[own].double()
    want = -2.0 * act.t().contiguous() @ z
    size = 2.0 * act.abs().t().contiguous() @ z.abs()
    assert torch.all((db[2, :, -8:].double() - want).abs() <= (layer.SPLIT + 2 * own.numel() * layer.U32) * size)


@pytest.mark.parametrize("ids", [False, True])
@pytest.mark.parametrize("n,rows,cols,rank", [(9001, 5003, 3081, 40), (5100, 9000, 6000, 7), (2600, 4100, 777, 64)])
def test_gradients_of_many_tokens(n, rows, cols, rank, ids):
    # against float64 on the GPU, with the oracle's bounds
    torch.manual_seed(n + rank)
    count = 2 if ids else 1
    x, dy, base = _filled(n, cols), _filled(n, rows, 0.1), _filled(n, cols)
    a, b = (0.1 * torch.randn(count, rank, w, device="cuda").half() for w in (cols, rows))
    scale, h = torch.rand(count, device="cuda") + 0.5, torch.randn(n, rank, device="cuda")
    which = torch.randint(-1, 2, (n,), device="cuda", dtype=torch.int32) if ids else None
    m = spdp.Adapters(a, b, scale)
    dx, da, db = torch.empty_like(x), torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    m.grad_into(x, which, h, dy, base, dx, da, db)
    for i in range(count):
        at = torch.arange(n, device="cuda") if which is None else torch.nonzero(which == i).flatten()
        s, k = float(scale[i]), at.numel()
        z, g, act = x[at].double(), dy[at].double(), h[at].double()
        bt = b[i].double().t().contiguous()
        u = g @ bt
        ue = 2 * rows * layer.U32 * (g.abs() @ bt.abs())
        per = layer.SPLIT + 2 * (2 * k + 2) * layer.U32
        for got, v, ve, t in ((da[i], u, ue, z), (db[i], act, torch.zeros_like(act), g)):
            want = s * (v.t().contiguous() @ t)
            size = v.abs() + ve
            bound = s * ((ve + per * size + layer.TINY * size.max()).t().contiguous() @ t.abs()) + 4 * layer.U32 * want.abs()
            assert torch.all((got.double() - want).abs() <= bound)
        want = base[at].double() + s * (u @ a[i].double())
        size = u.abs() + ue
        part = ue + (layer.SPLIT + 2 * (2 * rank + 2) * layer.U32) * size + layer.TINY * size.amax(1, keepdim=True)
        bound = s * (part @ a[i].double().abs()) + 4 * layer.U32 * want.abs()
        bound += torch.clamp(2.0 ** -11 * (want.abs() + bound), min=2.0 ** -25)
        assert torch.all((dx[at].double() - want).abs() <= bound)
    if which is not None:
        none = which < 0
        assert torch.equal(dx[none], base[none])


def test_heads_beyond_32_bits():
    n, heads, dim = 140_000, 128, 128
    assert n * heads * dim > 1 << 31
    x, dy = _filled(n, heads * dim), _filled(n, heads * dim, 0.1)
    rng = np.random.default_rng(2)
    pos = rng.integers(0, 300, n).astype(np.int32)
    ang = np.arange(300)[:, None] * np.exp(-np.log(1e4) * np.arange(0, dim, 2) / dim)
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    w = (1 + 0.1 * rng.normal(size=dim)).astype(np.float16)
    tabs = (_dev(pos), _dev(cos), _dev(sin))
    y = torch.empty_like(x)
    spdp.rotate_heads([x], dim, *tabs, [y], weights=[_dev(w)])
    at = _rows(n)
    sel = torch.from_numpy(at).cuda()
    want, bound = layer.heads(_np(x[sel]), dim, pos[at], cos, sin, w, 1e-6, False, np.zeros((len(at), heads * dim)))
    assert np.all(np.abs(_np(y[sel]) - want) <= bound)
    dw = torch.empty(dim, device="cuda")
    spdp.rotate_heads_grad([x], dim, *tabs, [dy], [y], weights=[_dev(w)], dweights=[dw])
    (want, bound), _ = layer.heads_grad(_np(x[sel]), dim, pos[at], cos, sin, _np(dy[sel]), w, 1e-6, False)
    assert np.all(np.abs(_np(y[sel]) - want) <= bound)
    assert torch.isfinite(dw).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_larger_than_the_caches(interleaved):
    # two inputs of rows one number into their memory, with padding, a part of
    # the head rotated; in place gives the same bits
    n, dim, rot, counts = 9001, 112, 96, (20, 3)
    shift = lambda v: torch.cat([torch.zeros(1, dtype=torch.float16, device="cuda"), v.reshape(-1)])[1:].view(v.shape)  # noqa: E731
    xs = [shift(_filled(n, k * dim)) for k in counts]
    dys = [shift(_filled(n, k * dim, 0.1)) for k in counts]
    rng = np.random.default_rng(4)
    pos = rng.integers(-1, 301, n).astype(np.int32)
    ang = np.arange(300)[:, None] * np.exp(-np.log(1e4) * np.arange(0, rot, 2) / rot)
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    w = (1 + 0.1 * rng.normal(size=dim)).astype(np.float16)
    tabs, ws = (_dev(pos), _dev(cos), _dev(sin)), [_dev(w), None]
    ys = [shift(torch.full_like(x, 7.0)) for x in xs]
    spdp.rotate_heads(xs, dim, *tabs, ys, weights=ws, interleaved=interleaved)
    dxs, dw = [shift(torch.zeros_like(x)) for x in xs], [torch.empty(dim, device="cuda"), None]
    spdp.rotate_heads_grad(xs, dim, *tabs, dys, dxs, weights=ws, dweights=dw, interleaved=interleaved)
    at = _rows(n)
    sel = torch.from_numpy(at).cuda()
    for x, dy, y, dx, weight in zip(xs, dys, ys, dxs, (w, None)):
        xh, was = _np(x[sel]), np.full((len(at), x.shape[1]), 7.0)
        want, bound = layer.heads(xh, dim, pos[at], cos, sin, weight, 1e-6, interleaved, was)
        assert np.all(np.abs(_np(y[sel]) - want) <= bound)
        (want, bound), _ = layer.heads_grad(xh, dim, pos[at], cos, sin, _np(dy[sel]), weight, 1e-6, interleaved)
        assert np.all(np.abs(_np(dx[sel]) - want) <= bound)
    inside = torch.from_numpy((pos >= 0) & (pos < 300)).cuda()
    again, dw2 = [v.clone() for v in dys], [torch.empty_like(dw[0]), None]
    spdp.rotate_heads_grad(xs, dim, *tabs, again, again, weights=ws, dweights=dw2, interleaved=interleaved)
    assert torch.equal(again[0], dxs[0]) and torch.equal(again[1], dxs[1]) and torch.equal(dw[0], dw2[0])
    spdp.rotate_heads(xs, dim, *tabs, xs, weights=ws, interleaved=interleaved)
    assert all(torch.equal(x[inside], y[inside]) for x, y in zip(xs, ys))


def test_pruned_gradient_beyond_32_bits():
    rows, cols, n = 32_776, 72, 66_000
    assert n * rows > 1 << 31
    rng = np.random.default_rng(3)
    w = (rng.normal(size=(rows, cols)) * 0.05).astype(np.float16)
    w[rng.random(w.shape) < 0.5] = 0
    m = spdp.encode(w, (256, 16))
    dy = _filled(n, rows)
    dx = m.spmm_grad(dy)
    at = _rows(n)
    sel = torch.from_numpy(at).cuda()
    want, bound = layer.spmm_grad(w, _np(dy[sel]))
    assert np.all(np.abs(_np(dx[sel]) - want) <= bound)
    m.close()


@pytest.mark.parametrize("rows,cols", [(200_003, 40), (40, 200_003)])
def test_wide_adapters(rows, cols):
    rng = np.random.default_rng(4)
    n, count, rank = 5, 2, 9
    x, base, dy = (rng.normal(size=(n, w)).astype(np.float16) for w in (cols, rows, rows))
    a, b = (0.05 * rng.normal(size=(count, rank, w)).astype(np.float16) for w in (cols, rows))
    scale, ids = np.array([0.5, 1.5], dtype=np.float32), np.array([1, 0, -1, 1, 1], dtype=np.int32)
    m = spdp.Adapters(_dev(a), _dev(b), _dev(scale))
    y, h = torch.empty(n, rows, dtype=torch.float16, device="cuda"), torch.empty(n, rank, device="cuda")
    m.add_into(_dev(x), _dev(ids), _dev(base), y, h=h)
    want, bound, hw, hb = layer.adapt(x, ids, base, a, b, scale)
    assert np.all(np.abs(_np(y) - want) <= bound) and np.all(np.abs(_np(h) - hw) <= hb)
    outs = (torch.empty(n, cols, dtype=torch.float16, device="cuda"), torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda"))
    m.grad_into(_dev(x), _dev(ids), h, _dev(dy), _dev(x), *outs)
    for got, (want, bound) in zip(outs, layer.adapt_grad(x, ids, _np(h), dy, x, a, b, scale)):
        assert np.all(np.abs(_np(got) - want) <= bound)


@pytest.mark.parametrize("seed", range(24))
def test_drawn_adapters(seed):
    rng = np.random.default_rng(1000 + seed)
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    n, rows, cols, count, rank = log(1, 400), log(1, 1500), log(1, 1500), log(1, 40), log(1, 128)
    print(f"[gpu] drawn {n} {rows}x{cols} {count} adapters of rank {rank}", flush=True)
    x, base, dy = (rng.normal(size=(n, w)).astype(np.float16) for w in (cols, rows, rows))
    a, b = (0.1 * rng.normal(size=(count, rank, w)).astype(np.float16) for w in (cols, rows))
    scale = rng.normal(size=count).astype(np.float32)
    ids = None if seed % 4 == 0 else rng.integers(-1, count + 1, n).astype(np.int32)
    # unaligned rows: views one number into their memory
    shift = lambda v: torch.cat([torch.zeros(1, dtype=torch.float16, device="cuda"), _dev(v).reshape(-1)])[1:].view(v.shape)  # noqa: E731
    place = shift if seed % 2 else _dev
    m = spdp.Adapters(place(a), place(b), _dev(scale))
    di = None if ids is None else _dev(ids)
    y, h = place(np.zeros_like(base)), torch.empty(n, rank, device="cuda")
    m.add_into(place(x), di, place(base), y, h=h)
    want, bound, hw, hb = layer.adapt(x, ids, base, a, b, scale)
    assert np.all(np.abs(_np(y) - want) <= bound) and np.all(np.abs(_np(h) - hw) <= hb + 1e-300)
    outs = (place(np.zeros_like(x)), torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda"))
    m.grad_into(place(x), di, h, place(dy), place(x), *outs)
    for got, (want, bound) in zip(outs, layer.adapt_grad(x, ids, _np(h), dy, x, a, b, scale)):
        assert np.all(np.abs(_np(got) - want) <= bound + 1e-300)


@pytest.mark.parametrize("seed", range(16))
def test_drawn_pruned_gradients(seed):
    rng = np.random.default_rng(2000 + seed)
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    rows, cols, n, tile_k = log(1, 3000), log(1, 1200), log(1, 700), int(rng.choice([16, 16, 32, 128]))
    print(f"[gpu] drawn {rows}x{cols} {n} tile_k {tile_k}", flush=True)
    keep = rng.random(cols) ** 2  # columns of very different density
    w = (rng.normal(size=(rows, cols)) * (rng.random((rows, cols)) < keep)).astype(np.float16)
    dy = (rng.normal(size=(n, rows)) * np.exp(rng.normal(size=(n, 1)))).astype(np.float16)
    m = spdp.encode(w, (256, tile_k))
    got = _np(m.spmm_grad(_dev(dy)))
    want, bound = layer.spmm_grad(w, dy)
    assert np.all(np.abs(got - want) <= bound)
    m.close()
