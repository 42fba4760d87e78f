"""The gradient of the pruned product with respect to its input against the
float64 oracle: bit for bit on inputs whose sums are exact in fp32, and within
the oracle's bound on realistic ones; every token tile, forced splits, ragged
sizes, handles without word records."""

import numpy as np
import pytest

import oracle
import synth
from oracle import layer

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2607_21985_amd as spdp  # noqa: E402


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _run(m, dy):
    dx = torch.full((dy.shape[0], m.cols), float("nan"), dtype=torch.float16, device="cuda")
    m.spmm_grad_into(_dev(dy), dx)
    return dx.cpu().numpy()


def _exact(rows, cols, n, sw, seed):
    rng = np.random.default_rng(seed)
    w = (rng.integers(1, 9, (rows, cols)) * rng.choice([-1, 1], (rows, cols)) / 64.0).astype(np.float16)
    w[rng.random((rows, cols)) < sw] = 0
    return w, (rng.integers(-4, 5, (n, rows)) / 4.0).astype(np.float16)


def _check_exact(m, w, dy, label):
    got = _run(m, dy)
    want = layer.spmm_grad(w, dy)[0].astype(np.float16)
    bad = got.astype(np.float64) != want.astype(np.float64)
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} differ; first (token, column) {at}: {got[at]} for {want[at]}")


# rows, cols, tile_k, weight sparsity, tokens
SIZES = [
    (256, 16, 16, 0.5, 1),
    (1, 8, 16, 0.0, 1),
    (1, 40, 16, 0.3, 7),
    (64, 64, 16, 0.0, 32),
    (256, 128, 16, 0.5, 33),
    (333, 517, 16, 0.5, 5),
    (700, 1000, 16, 0.6, 129),
    (512, 1024, 32, 0.7, 300),
    (1000, 1536, 64, 0.5, 64),
    (2056, 200, 128, 0.9, 257),
    (300, 520, 256, 0.5, 100),
    (513, 130, 16, 0.0, 96),
    (1100, 72, 16, 1.0, 40),
    (4096, 264, 16, 0.5, 16),
]


@pytest.mark.parametrize("rows,cols,tile_k,sw,n", SIZES)
def test_exact(rows, cols, tile_k, sw, n):
    print(f"[gpu] spmm_grad {rows}x{cols} tile_k {tile_k} {n}", flush=True)
    w, dy = _exact(rows, cols, n, sw, rows + cols + n)
    m = spdp.encode(w, (256, tile_k))
    _check_exact(m, w, dy, "default")
    m.close()


@pytest.mark.parametrize("form", range(-1, 8))
@pytest.mark.parametrize("splits", [1, 3, 100])
def test_every_form_and_split(monkeypatch, form, splits):
    monkeypatch.setenv("SPDP_GRAD_FORM", str(form))
    monkeypatch.setenv("SPDP_GRAD_SPLITS", str(splits))
    for rows, cols, sw, n in ((1000, 200, 0.5, 300), (803, 333, 0.6, 70), (520, 136, 0.3, 31)):
        print(f"[gpu] spmm_grad {rows}x{cols} {n} form {form} splits {splits}", flush=True)
        w, dy = _exact(rows, cols, n, sw, rows + n)
        m = spdp.encode(w, (256, 16))
        _check_exact(m, w, dy, f"{rows}x{cols} {n}")
        m.close()


@pytest.mark.parametrize("rows,cols,sw,n", [(1024, 1024, 0.5, 200), (2048, 768, 0.7, 77), (503, 1001, 0.5, 50)])
def test_realistic_inputs(rows, cols, sw, n):
    w = oracle.magnitude_prune(synth.weights(rows, cols, rows + n), sw)
    rng = np.random.default_rng(n)
    dy = (0.01 * np.exp(rng.normal(size=(n, 1))) * rng.normal(size=(n, rows))).astype(np.float16)
    m = spdp.encode(w, (256, 16))
    got = _run(m, dy).astype(np.float64)
    want, bound = layer.spmm_grad(w, dy)
    assert np.all(np.abs(got - want) <= bound)
    # <dY, X W^T> = <dY W, X>: the forward product's own gradient
    x = synth.laplace_activations(n, cols, 5)
    y = m.spmm(_dev(x)).cpu().numpy().astype(np.float64)
    y_err = 2 * cols * layer.U32 * (np.abs(x.astype(np.float64)) @ np.abs(w.astype(np.float64)).T)
    y_err += layer.half_step(np.abs(y) + y_err)
    slack = (np.abs(dy) * y_err).sum() + (np.abs(x) * bound).sum()
    assert abs((dy.astype(np.float64) * y).sum() - (got * x.astype(np.float64)).sum()) <= slack
    m.close()


def test_bits_do_not_depend_on_the_stream_and_replays():
    w, dy = _exact(700, 328, 90, 0.5, 9)
    m = spdp.encode(w, (256, 16))
    d, dx = _dev(dy), torch.empty(90, 328, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m.spmm_grad_into(d, dx, stream=side)
    side.synchronize()
    assert torch.equal(dx, m.spmm_grad(d))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.spmm_grad_into(d, dx)
    for rep in range(4):
        d.copy_(torch.randn(90, 700, device="cuda"))
        dx.fill_(float("nan"))
        g.replay()
        got = dx.clone()
        assert torch.equal(got, m.spmm_grad(d)), rep
    m.close()


def test_a_bad_token_stays_apart():
    w, dy = _exact(300, 100, 40, 0.5, 12)
    dy[7, 299], dy[20, 0] = np.inf, np.nan
    m = spdp.encode(w, (256, 16))
    got = _run(m, dy)
    ok = np.ones(40, dtype=bool)
    ok[[7, 20]] = False
    assert np.array_equal(got[ok].astype(np.float64), layer.spmm_grad(w, dy[ok])[0].astype(np.float16).astype(np.float64))
    m.close()
