"""The adapters and their gradients against the float64 oracle (`oracle.layer`),
within its bounds, and bit for bit on inputs whose sums are exact."""

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


def _ids(rng, n, count, how):
    if how == "none":
        return None
    if how == "same":
        return np.full(n, count - 1, dtype=np.int32)
    if how == "away":  # nobody has an adapter
        return np.where(rng.integers(0, 2, n) == 0, -1, count).astype(np.int32)
    if how == "runs":
        return np.sort(rng.integers(0, count, n)).astype(np.int32)
    return rng.integers(-1, count + 1, n).astype(np.int32)  # "mixed": -1 and count are none


def _problem(n, rows, cols, count, rank, how, seed, exact=False):
    rng = np.random.default_rng(seed)
    if exact:
        # multiples of 1/4 and small: every product and sum is an fp32 integer multiple of 1/4096
        draw = lambda s, m: rng.integers(-m, m + 1, s) / 4.0  # noqa: E731
        x, a, b = draw((n, cols), 4), draw((count, rank, cols), 2), draw((count, rank, rows), 2)
        base, scale = draw((n, rows), 8), 2.0 ** rng.integers(-4, 1, count)
    else:
        x = rng.laplace(size=(n, cols)) * np.where(rng.random(cols) < 0.02, 20.0, 1.0)
        a, b = rng.normal(size=(count, rank, cols)) / np.sqrt(cols), 0.05 * rng.normal(size=(count, rank, rows))
        base, scale = rng.normal(size=(n, rows)), np.exp(rng.normal(size=count))
    return (x.astype(np.float16), _ids(rng, n, count, how), base.astype(np.float16), a.astype(np.float16),
            b.astype(np.float16), scale.astype(np.float32))


def _bank(a, b, scale):
    return spdp.Adapters(_dev(a), _dev(b), _dev(scale))


def _within(got, want, bound, label):
    err = np.abs(got.astype(np.float64) - want)
    bad = ~(err <= bound)
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} out of bounds; first {at}: {got[at]} for {want[at]}, "
                             f"bound {bound[at]:.3g}; largest {np.nanmax(err / bound):.3g} of the bound")


# tokens, rows, cols, adapters, rank, ids
SIZES = [
    (1, 256, 256, 1, 8, "none"),
    (1, 1, 1, 1, 1, "mixed"),
    (1, 1024, 1024, 4, 8, "same"),
    (2, 65, 33, 3, 3, "mixed"),
    (7, 500, 1000, 4, 16, "mixed"),
    (32, 768, 512, 40, 16, "mixed"),
    (33, 255, 257, 2, 17, "mixed"),
    (64, 512, 2048, 64, 4, "mixed"),
    (64, 300, 300, 1, 33, "same"),
    (65, 300, 304, 3, 32, "mixed"),
    (128, 1000, 72, 7, 64, "away"),
    (333, 503, 308, 5, 12, "mixed"),
    (333, 264, 1031, 200, 5, "mixed"),
    (100, 640, 2000, 1, 64, "none"),
    (200, 512, 1024, 2, 128, "runs"),
    (1025, 128, 136, 2048, 2, "mixed"),
    (2100, 72, 520, 3, 100, "runs"),
    (512, 96, 1032, 5, 70, "mixed"),
    (513, 520, 96, 1, 24, "none"),
    (600, 200, 152, 3, 40, "mixed"),
    (700, 1000, 1000, 1, 128, "same"),
]


@pytest.mark.parametrize("n,rows,cols,count,rank,how", SIZES)
@pytest.mark.parametrize("exact", [False, True])
def test_adapt(n, rows, cols, count, rank, how, exact):
    print(f"[gpu] adapt {n} {rows}x{cols} {count} {rank} {how} exact={exact}", flush=True)
    x, ids, base, a, b, scale = _problem(n, rows, cols, count, rank, how, n + rows + rank, exact)
    m = _bank(a, b, scale)
    y = torch.full((n, rows), float("nan"), dtype=torch.float16, device="cuda")
    h = torch.full((n, rank), float("nan"), device="cuda")
    di = None if ids is None else _dev(ids)
    m.add_into(_dev(x), di, _dev(base), y, h=h)
    want, bound, hw, hb = layer.adapt(x, ids, base, a, b, scale)
    if exact:
        assert np.array_equal(_np(h), hw.astype(np.float32))
        assert np.array_equal(_np(y).astype(np.float64), want.astype(np.float16).astype(np.float64))
    else:
        _within(_np(h), hw, hb + 1e-300, "h")
        _within(_np(y), want, bound, "y")
    # in place, without h, gives the same bits
    z = _dev(base)
    m.add_into(_dev(x), di, z, z)
    assert torch.equal(z, y)


@pytest.mark.parametrize("n,rows,cols,count,rank,how", SIZES)
@pytest.mark.parametrize("exact", [False, True])
def test_adapt_grad(n, rows, cols, count, rank, how, exact):
    print(f"[gpu] adapt_grad {n} {rows}x{cols} {count} {rank} {how} exact={exact}", flush=True)
    x, ids, _, a, b, scale = _problem(n, rows, cols, count, rank, how, 7 * n + rows + rank, exact)
    rng = np.random.default_rng(n + 1)
    if exact:
        dy = (rng.integers(-2, 3, (n, rows)) / 4.0).astype(np.float16)
        base = (rng.integers(-8, 9, (n, cols)) / 4.0).astype(np.float16)
        h = (rng.integers(-64, 65, (n, rank)) / 16.0).astype(np.float32)
    else:
        size = np.exp(2 * rng.normal(size=(n, 1))) * 1e-2
        dy = (size * rng.normal(size=(n, rows))).astype(np.float16)
        base = (size * rng.normal(size=(n, cols))).astype(np.float16)
        h = layer.adapt(x, ids, np.zeros((n, rows)), a, b, scale)[2].astype(np.float32)
    m = _bank(a, b, scale)
    dx = torch.full((n, cols), float("nan"), dtype=torch.float16, device="cuda")
    da = torch.full(a.shape, float("nan"), device="cuda")
    db = torch.full(b.shape, float("nan"), device="cuda")
    args = (_dev(x), None if ids is None else _dev(ids), _dev(h), _dev(dy))
    m.grad_into(*args, _dev(base), dx, da, db)
    want = layer.adapt_grad(x, ids, h, dy, base, a, b, scale)
    for got, (w, bound), label in zip((dx, da, db), want, ("dx", "da", "db")):
        if exact:
            assert np.array_equal(_np(got).astype(np.float64), w.astype(_np(got).dtype).astype(np.float64)), label
        else:
            _within(_np(got), w, bound + 1e-300, label)
    # in place, and again: the same bits
    z, da2, db2 = _dev(base), torch.empty_like(da), torch.empty_like(db)
    m.grad_into(*args, z, z, da2, db2)
    assert torch.equal(z, dx) and torch.equal(da2, da) and torch.equal(db2, db)


def test_gradients_are_differences():
    # L = sum(dy * y): central differences of the fp64 formula
    n, rows, cols, count, rank = 5, 24, 40, 2, 3
    x, ids, base, a, b, scale = _problem(n, rows, cols, count, rank, "mixed", 3)
    dy = np.random.default_rng(4).normal(size=(n, rows)).astype(np.float16)
    m = _bank(a, b, scale)
    h = torch.empty(n, rank, device="cuda")
    y, dx = torch.empty(n, rows, dtype=torch.float16, device="cuda"), torch.empty(n, cols, dtype=torch.float16, device="cuda")
    da, db = torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    m.add_into(_dev(x), _dev(ids), _dev(base), y, h=h)
    m.grad_into(_dev(x), _dev(ids), h, _dev(dy), torch.zeros_like(dx), dx, da, db)
    loss = lambda x_, a_, b_: float((dy.astype(np.float64) * layer.adapt(x_, ids, base, a_, b_, scale)[0]).sum())  # noqa: E731
    args = [v.astype(np.float64) for v in (x, a, b)]
    rng = np.random.default_rng(5)
    for k, (got, rel) in enumerate(((dx, 2.0 ** -10), (da, 1e-5), (db, 1e-5))):
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in args[k].shape)
            lo, hi = [v.copy() for v in args], [v.copy() for v in args]
            lo[k][at] -= 1e-3
            hi[k][at] += 1e-3  # the loss is linear in each: the difference is exact but for fp64
            d = (loss(*hi) - loss(*lo)) / 2e-3
            assert abs(float(got[at]) - d) <= rel * abs(d) + 1e-6, (k, at)


def test_many_gives_each_projection_its_own_result():
    n, count, rank = 32, 5, 16
    for how in ("mixed", "none"):
        probs = [_problem(n, rows, cols, count, rank, how, 50 + rows) for rows, cols in ((512, 384), (128, 384), (129, 1024))]
        ids = probs[0][1]
        di = None if ids is None else _dev(ids)
        ms = [_bank(p[3], p[4], p[5]) for p in probs]
        xs, bases = [_dev(p[0]) for p in probs], [_dev(p[2]) for p in probs]
        ys, hs = [torch.empty_like(b) for b in bases], [torch.empty(n, rank, device="cuda") for _ in ms]
        spdp.adapters_many(ms, xs, di, bases, ys, hs=hs)
        for p, y, h in zip(probs, ys, hs):
            want, bound, hw, hb = layer.adapt(p[0], ids, p[2], p[3], p[4], p[5])
            _within(_np(y), want, bound, "y")
            _within(_np(h), hw, hb + 1e-300, "h")


def test_far_sizes_infinities_and_nan():
    # h beyond fp16's range, and far below it, keep their digits; infinities
    # and NaN stay with their tokens
    n, rows, cols, rank = 40, 96, 64, 16
    rng = np.random.default_rng(11)
    x = (rng.normal(size=(n, cols)) * 10.0 ** rng.uniform(-4, 4, (n, 1))).astype(np.float16)
    a = (rng.normal(size=(2, rank, cols)) * 100).astype(np.float16)
    b = (rng.normal(size=(2, rank, rows)) * 1e-3).astype(np.float16)
    scale = np.array([1e-3, 2.0], dtype=np.float32)
    base = np.zeros((n, rows), dtype=np.float16)
    ids = rng.integers(0, 2, n).astype(np.int32)
    ids[x.astype(np.float64).__abs__().max(1) > 300] = 0
    x[5, 3], x[9, 0] = np.inf, np.nan
    m = _bank(a, b, scale)
    y, h = torch.empty(n, rows, dtype=torch.float16, device="cuda"), torch.empty(n, rank, device="cuda")
    m.add_into(_dev(x), _dev(ids), _dev(base), y, h=h)
    ok = np.ones(n, dtype=bool)
    ok[[5, 9]] = False
    with np.errstate(invalid="ignore"):
        want, bound, hw, hb = layer.adapt(x[ok], ids[ok], base[ok], a, b, scale)
    assert np.abs(hw).max() > 1e5 and np.abs(want).max() < 6e4
    _within(_np(h)[ok], hw, hb, "h")
    _within(_np(y)[ok], want, bound, "y")
    assert not np.isfinite(_np(h)[~ok]).any() and not np.isfinite(_np(y)[~ok]).any()


def test_stream_and_replays():
    n, rows, cols, count, rank = 90, 520, 776, 3, 24
    x, ids, base, a, b, scale = _problem(n, rows, cols, count, rank, "mixed", 21)
    m = _bank(a, b, scale)
    X, I, base_d = _dev(x), _dev(ids), _dev(base)
    dy, h = torch.randn(n, rows, device="cuda").half(), torch.empty(n, rank, device="cuda")
    y, dx = torch.empty_like(base_d), torch.empty(n, cols, dtype=torch.float16, device="cuda")
    da, db = torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")

    def step(stream=None):
        m.add_into(X, I, base_d, y, h=h, stream=stream)
        m.grad_into(X, I, h, dy, X, dx, da, db, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    first = [t.clone() for t in (y, h, dx, da, db)]
    step()
    assert all(torch.equal(s, t) for s, t in zip(first, (y, h, dx, da, db)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(4):
        X.copy_(torch.randn(n, cols, device="cuda"))
        I.copy_(torch.randint(-1, count + 1, (n,), device="cuda"))
        for t in (y, h, dx, da, db):
            t.fill_(float("nan"))
        g.replay()
        got = [t.clone() for t in (y, h, dx, da, db)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(got, (y, h, dx, da, db))), rep
