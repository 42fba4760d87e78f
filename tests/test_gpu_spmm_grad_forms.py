"""The forms of the pruned product's gradient, each where it is known to run (the
stand-in runtime's tests hold the same lists): bit for bit on inputs whose sums
are exact in fp32."""

import numpy as np
import pytest

from test_operator_limits import GRAD_DEFAULTS, GRAD_FORMS, GRAD_SPARSE

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2607_21985_amd as spdp  # noqa: E402


def _check(rows, cols, keep, n):
    # multiples of 1/64 up to 1/8 times multiples of 1/4 up to 1: sums of 2051 of them
    # are multiples of 1/256 below 2^9
    rng = np.random.default_rng(rows + cols + n)
    w = (rng.integers(1, 9, (rows, cols)) * rng.choice([-1, 1], (rows, cols)) / 64.0).astype(np.float16)
    w[rng.random((rows, cols)) >= keep] = 0
    dy = (rng.integers(-4, 5, (n, rows)) / 4.0).astype(np.float16)
    m = spdp.encode(w, (256, 16))
    d = torch.from_numpy(dy).cuda()
    dx = torch.full((n, cols), float("nan"), dtype=torch.float16, device="cuda")
    m.spmm_grad_into(d, dx)
    want = (d.double() @ torch.from_numpy(w).cuda().double()).half()
    bad = torch.nonzero(dx.double() != want.double())
    assert len(bad) == 0, f"{len(bad)} of {dx.numel()} differ, the first at {bad[0].tolist()}"
    m.close()


@pytest.mark.parametrize("rows,cols,keep,n,form", GRAD_DEFAULTS)
def test_by_default(rows, cols, keep, n, form):
    print(f"[gpu] spmm_grad {rows}x{cols} {n}: {form}", flush=True)
    _check(rows, cols, keep, n)


@pytest.mark.parametrize("place", range(len(GRAD_FORMS)))
@pytest.mark.parametrize("splits", [1, 2, 100])
def test_forced(monkeypatch, place, splits):
    monkeypatch.setenv("SPDP_GRAD_FORM", str(place))
    monkeypatch.setenv("SPDP_GRAD_SPLITS", str(splits))
    for rows, cols, keep in GRAD_SPARSE:
        for n in (1, 300, 700):
            print(f"[gpu] spmm_grad {rows}x{cols} {n}: form {place}, {splits} ranges", flush=True)
            _check(rows, cols, keep, n)
