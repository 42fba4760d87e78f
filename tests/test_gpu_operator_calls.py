"""Calls of the adapters', heads' and gradient operators as programs make them
around the operators themselves: chains whose weights change."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2607_21985_amd as spdp  # noqa: E402


def _half(*shape, scale=1.0):
    return (scale * torch.randn(shape, device="cuda")).half()


def _bank(count, rank, rows, cols):
    return spdp.Adapters(_half(count, rank, cols, scale=cols ** -0.5), _half(count, rank, rows, scale=0.1),
                         torch.rand(count, device="cuda") + 0.5)


def _tables(positions, rot):
    ang = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * torch.exp(
        -np.log(1e4) * torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return ang.cos().float(), ang.sin().float()


def test_a_chain_whose_weights_change():
    torch.manual_seed(1)
    n, rows, cols, dim, count = 7, 384, 520, 64, 3
    bank, weight = _bank(count, 16, rows, cols), (1 + 0.1 * torch.randn(dim, device="cuda")).half()
    x, base = _half(n, cols), _half(n, rows)
    ids = torch.randint(-1, count, (n,), device="cuda", dtype=torch.int32)
    pos, (cos, sin) = torch.arange(n, device="cuda", dtype=torch.int32), _tables(40, dim)
    y, z = torch.empty_like(base), torch.empty_like(base)
    ch = spdp.Chain().add_adapters(bank, x, ids, base, y).add_heads([y], dim, pos, cos, sin, [z], weights=[weight])
    ch.capture()

    def check():
        y.fill_(float("nan"))
        z.fill_(float("nan"))
        ch.replay()
        want, turned = bank(x, ids, base), torch.empty_like(base)
        spdp.rotate_heads([want], dim, pos, cos, sin, [turned], weights=[weight])
        assert torch.equal(y, want) and torch.equal(z, turned)

    check()
    # in place: the next replay has them
    for change in (lambda: bank.a.mul_(-1), lambda: bank.b.add_(0.01), lambda: bank.scale.mul_(2), lambda: weight.mul_(0.5)):
        before = z.clone()
        change()
        check()
        assert not torch.equal(z, before)
    # replaced: refused until the chain is captured again

    def data():
        bank.b.data = bank.b.data.clone() + 0.02

    def norm():
        weight.data = weight.data.clone() + 1

    for change in (lambda: setattr(bank, "a", 0.5 * bank.a), data, lambda: setattr(bank, "scale", bank.scale + 1), norm):
        change()
        before = z.clone()
        with pytest.raises(RuntimeError, match="captur"):
            ch.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, before)
        ch.capture()
        check()
        assert not torch.equal(z, before)


def test_results_on_another_stream():
    # the current stream has work left on a block that it has given back: a result
    # on another stream must not take it
    torch.manual_seed(2)
    n, rows, cols = 200, 512, 512
    bank = _bank(2, 16, rows, cols)
    w = np.random.default_rng(3).normal(size=(rows, cols)).astype(np.float16)
    w[np.random.default_rng(4).random(w.shape) < 0.5] = 0
    m = spdp.encode(w, (256, 16))
    x, base = _half(n, cols), _half(n, rows)
    ids = torch.randint(-1, 2, (n,), device="cuda", dtype=torch.int32)
    side = torch.cuda.Stream()
    for call in (lambda s: bank(x, ids, base, stream=s), lambda s: m.spmm_grad(base, stream=s),
                 lambda s: m.spmm(x, stream=s), lambda s: m(x[:4], 0.1, stream=s)):
        want = call(None)
        torch.cuda.synchronize()
        scratch = torch.empty_like(want)
        torch.cuda._sleep(20_000_000)
        scratch.fill_(float("nan"))
        del scratch
        got = call(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    m.close()


@pytest.mark.parametrize("dim,rot", [(128, 128), (96, 32), (34, 6), (250, 126), (512, 512)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("where", ["table", "weight", "infinite weight"])
def test_gradients_of_padding_are_0_beside_bad_numbers(dim, rot, interleaved, where):
    # bad numbers that padding tokens have nothing to do with: the first position's
    # angles, which no token has, or the weight
    torch.manual_seed(dim + rot)
    n, heads, table = 9, 3, 20
    cos, sin = _tables(table, rot)
    weight = (1 + 0.1 * torch.randn(dim, device="cuda")).half()
    if where == "table":
        cos[0], sin[0] = float("nan"), float("inf")
    else:
        weight[1] = float("nan") if where == "weight" else float("inf")
    pos = torch.tensor([3, -1, 5, table, 1, 2 ** 31 - 1, -2 ** 31, 19, 1], device="cuda", dtype=torch.int32)
    padding = (pos < 0) | (pos >= table)
    x, dy = _half(n, heads * dim), _half(n, heads * dim)
    x[padding], dy[padding] = float("nan"), float("inf")
    for dx in (torch.full_like(x, 7.0), x.clone(), dy.clone()):
        dw = torch.full((dim,), 7.0, device="cuda")
        spdp.rotate_heads_grad([x], dim, pos, cos, sin, [dy], [dx], weights=[weight], dweights=[dw], interleaved=interleaved)
        assert torch.equal(dx[padding], torch.zeros_like(dx[padding]))
        assert torch.isfinite(dx[~padding]).all() == (where == "table")
        assert torch.isfinite(dw).all()  # (the weight's gradient does not depend on the weight)


@pytest.mark.parametrize("n,count,rank,how,rows,cols", [
    (1, 1, 1, "one", 264, 520), (1, 1, 24, "one", 264, 520), (4, 1, 16, "one", 264, 520), (64, 1, 33, "one", 264, 520),
    (30, 4, 24, "mixed", 264, 520), (200, 12, 8, "mixed", 264, 520), (64, 1, 128, "one", 264, 520),
    (16, 2, 64, "mixed", 264, 520), (300, 40, 16, "mixed", 4104, 4100), (300, 40, 40, "mixed", 4104, 4100),
    (600, 40, 24, "mixed", 264, 520), (700, 20, 40, "mixed", 264, 520), (540, 64, 128, "mixed", 264, 520),
    (520, 20, 100, "mixed", 264, 520),
    (600, 40, 24, "mixed", 4104, 4100), (600, 40, 40, "mixed", 4104, 4100), (600, 40, 100, "mixed", 4104, 4100),
    # one adapter has almost all tokens, split over the launch, the others have few;
    # the last two with 128 columns a workgroup
    (3000, 3, 20, "few", 264, 520), (6000, 2, 20, "few", 264, 520), (6000, 2, 64, "few", 264, 520),
    (6000, 2, 100, "few", 264, 520),
    (6000, 2, 20, "few", 8202, 4104), (6000, 2, 64, "few", 8202, 4104)])
def test_gradients_of_few_tokens_have_the_bits_of_fp32(n, count, rank, how, rows, cols):
    # ranks whose activations lie far below one another: each has the error of fp32
    # products and sums in any order (2 2^-24 of the magnitudes for each addition: the
    # tokens, the waves, the ranges and the scale), whatever the others' size
    u32 = 2.0 ** -24
    rng = np.random.default_rng(n + rank)
    sizes = 2.0 ** -rng.permutation(np.linspace(0, 24, rank).astype(int)) if rank > 1 else np.ones(1)
    ids = np.zeros(n, dtype=np.int32) if how == "one" else rng.integers(-1, count, n).astype(np.int32)
    if how == "few":
        ids[:] = 0
        ids[rng.permutation(n)[:17 * (count - 1)]] = np.repeat(np.arange(1, count), 17)
    a = rng.normal(size=(count, rank, cols)).astype(np.float16)
    b = (rng.normal(size=(count, rank, rows)) * sizes[None, :, None]).astype(np.float16)
    b[:, :, 2:] = 0  # u is a sum of two products, so that its own error is small
    scale = np.exp(rng.normal(size=count)).astype(np.float32)
    x, dy = rng.normal(size=(n, cols)).astype(np.float16), rng.normal(size=(n, rows)).astype(np.float16)
    h = (rng.normal(size=(n, rank)) * sizes).astype(np.float32)
    dev = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    bank = spdp.Adapters(dev(a), dev(b), dev(scale))
    dx, da, db = torch.empty(n, cols, dtype=torch.float16, device="cuda"), torch.empty(a.shape, device="cuda"), \
        torch.empty(b.shape, device="cuda")
    bank.grad_into(dev(x), None if how == "one" else dev(ids), dev(h), dev(dy), torch.zeros_like(dx), dx, da, db)
    few = 0
    for i in range(count):
        at = np.flatnonzero(ids == i)
        k = at.size
        if k == 0 or k > 64:
            continue
        few += 1
        front, b2 = dy[at, :2].astype(np.float64), b[i, :, :2].astype(np.float64).T
        # (the matrix cores align the products of a subnormal fp16 as those of 2^-14)
        u, u_err = front @ b2, 4 * u32 * (np.abs(front) @ np.maximum(np.abs(b2), 2.0 ** -14))
        for got, act, own, z in ((da[i], u, u_err, x[at]), (db[i], h[at].astype(np.float64), np.zeros_like(u), dy[at])):
            z, s = z.astype(np.float64), float(scale[i])
            want, size = s * (act.T @ z), s * ((np.abs(act) + own).T @ np.abs(z))
            bound = s * (own.T @ np.abs(z)) + 2 * (k + 26) * u32 * size  # (at most 8 waves, 16 ranges)
            err = np.abs(got.cpu().numpy().astype(np.float64) - want)
            assert np.all(err <= bound), (i, k, np.max(err / np.maximum(size, 1e-300)))
    assert few
