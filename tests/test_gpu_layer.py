"""The products and what stands beside them, run together as a layer: a decode
step captured as one graph, and a training step through a pruned projection
with adapters."""

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


def _bank(rng, count, rank, rows, cols):
    return spdp.Adapters(_dev((rng.normal(size=(count, rank, cols)) / np.sqrt(cols)).astype(np.float16)),
                         _dev((0.1 * rng.normal(size=(count, rank, rows))).astype(np.float16)),
                         _dev(np.exp(rng.normal(size=count)).astype(np.float32)))


def test_decode_step_in_a_chain():
    rng = np.random.default_rng(1)
    width, dim, n, count = 512, 64, 6, 4
    rows = (512, 128, 128)
    mats = [spdp.encode(oracle.magnitude_prune(synth.weights(r, width, 10 + i), 0.5), (256, 16)) for i, r in enumerate(rows)]
    banks = [_bank(rng, count, 8, r, width) for r in rows]
    o, obank = spdp.encode(oracle.magnitude_prune(synth.weights(width, 512, 20), 0.5), (256, 16)), _bank(rng, count, 8, width, 512)
    x = torch.zeros(n, width, dtype=torch.float16, device="cuda")
    ids, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    ang = np.arange(100)[:, None] * np.exp(-np.log(1e4) * np.arange(0, dim, 2) / dim)
    cos, sin = _dev(np.cos(ang).astype(np.float32)), _dev(np.sin(ang).astype(np.float32))
    ws = [_dev((1 + 0.1 * rng.normal(size=dim)).astype(np.float16)) for _ in range(2)]

    def outputs():
        return [torch.zeros(n, r, dtype=torch.float16, device="cuda") for r in rows + (width,)]

    def record(ch, ys):
        ch.add(mats, [x] * 3, [0.4] * 3, ys[:3])
        ch.add_adapters(banks, [x] * 3, ids, ys[:3], ys[:3])
        ch.add_heads(ys[:2], dim, pos, cos, sin, ys[:2], weights=ws)
        ch.add(o, ys[0], 0.2, ys[3])
        ch.add_adapters(obank, ys[0], ids, ys[3], ys[3])
        return ch

    ys = outputs()
    one, two = record(spdp.Chain(), ys).capture(), record(spdp.Chain(), ys).capture()
    with pytest.raises(RuntimeError):
        one.add_adapters(obank, x, ids, ys[3], ys[3])
    with pytest.raises(RuntimeError):
        one.add_heads(ys[:2], dim, pos, cos, sin, ys[:2])
    for rep in range(4):
        x.copy_(torch.from_numpy(synth.laplace_activations(n, width, 100 + rep)))
        ids.copy_(torch.from_numpy(rng.integers(-1, count, n).astype(np.int32)))
        pos.copy_(torch.from_numpy(rng.integers(0, 100, n).astype(np.int32)))
        for chain in (one, two):
            for y in ys:
                y.fill_(float("nan"))
            chain.replay()
            got = [y.clone() for y in ys]
            # the same calls by themselves
            want = outputs()
            spdp.spmspv_many(mats, [x] * 3, [0.4] * 3, want[:3])
            base = [w.clone() for w in want[:3]]
            spdp.adapters_many(banks, [x] * 3, ids, base, want[:3])
            raw = [w.clone() for w in want[:2]]
            spdp.rotate_heads(raw, dim, pos, cos, sin, want[:2], weights=ws)
            o.spmspv_into(want[0], 0.2, want[3])
            obank.add_into(want[0], ids, want[3], want[3])
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want)), rep
        # and the last replay's keys against the oracle
        xn, i, p = x.cpu().numpy(), ids.cpu().numpy(), pos.cpu().numpy()
        m = banks[1]
        y, bound, _, _ = layer.adapt(xn, i, base[1].cpu().numpy(), *(v.cpu().numpy() for v in (m.a, m.b, m.scale)))
        assert np.all(np.abs(raw[1].cpu().numpy() - y) <= bound)
        k, bound = layer.heads(raw[1].cpu().numpy(), dim, p, cos.cpu().numpy(), sin.cpu().numpy(), ws[1].cpu().numpy(),
                               1e-6, False, y)
        assert np.all(np.abs(got[1].cpu().numpy() - k) <= bound)
    for m in mats + [o]:
        m.close()


def test_training_step_through_a_pruned_projection():
    rng = np.random.default_rng(2)
    rows, cols, n, count, rank = 520, 392, 150, 3, 8
    w = oracle.magnitude_prune(synth.weights(rows, cols, 3), 0.5)
    m, bank = spdp.encode(w, (256, 16)), _bank(rng, count, rank, rows, cols)
    x, dy = _dev(synth.laplace_activations(n, cols, 4)), _dev((0.1 * rng.normal(size=(n, rows))).astype(np.float16))
    ids = _dev(rng.integers(-1, count, n).astype(np.int32))
    h = torch.empty(n, rank, device="cuda")
    da, db = torch.empty(count, rank, cols, device="cuda"), torch.empty(count, rank, rows, device="cuda")
    y = m.spmm(x)
    bank.add_into(x, ids, y, y, h=h)
    dx = m.spmm_grad(dy)
    base = dx.cpu().numpy()
    bank.grad_into(x, ids, h, dy, dx, dx, da, db)
    want, bound = layer.spmm_grad(w, dy.cpu().numpy())
    assert np.all(np.abs(base - want) <= bound)
    arrays = [t.cpu().numpy() for t in (x, ids, h, dy)]
    got = layer.adapt_grad(*arrays, base, *(v.cpu().numpy() for v in (bank.a, bank.b, bank.scale)))
    for t, (v, e) in zip((dx, da, db), got):
        assert np.all(np.abs(t.cpu().numpy() - v) <= e)
    # a step of the weights in place, in other memory or as another tensor counts
    # in the next call
    before = y.clone()
    bank.b -= (0.5 * db).half()
    bank.a.data = bank.a.data - (0.5 * da).half()
    bank.scale = bank.scale * 1.5
    y = m.spmm(x)
    bank.add_into(x, ids, y, y, h=h)
    assert not torch.equal(y, before)
    v, e, _, _ = layer.adapt(arrays[0], arrays[1], m.spmm(x).cpu().numpy(), *(t.cpu().numpy() for t in (bank.a, bank.b, bank.scale)))
    got = y.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - v) <= e)
    big = np.abs(v) - e > 65520.0  # beyond fp16 for certain
    assert np.all(np.isinf(got[big])) and np.all(np.abs(got[np.abs(v) < 60000.0]) < 65504.0)
    m.close()


def test_two_streams_at_once():
    # calls on one bank and one matrix may overlap: nothing is shared but the weights
    rng = np.random.default_rng(5)
    rows, cols, n = 1024, 1024, 200
    m = spdp.encode(oracle.magnitude_prune(synth.weights(rows, cols, 6), 0.5), (256, 16))
    bank = _bank(rng, 2, 16, rows, cols)
    streams = [torch.cuda.Stream() for _ in range(2)]
    xs = [_dev(synth.laplace_activations(n, cols, 30 + i)) for i in range(2)]
    dys = [_dev(synth.laplace_activations(n, rows, 40 + i)) for i in range(2)]
    ids = _dev(rng.integers(0, 2, n).astype(np.int32))
    bases = [torch.zeros(n, rows, dtype=torch.float16, device="cuda") for _ in range(2)]

    def go(i, stream=None):
        outs = []
        for _ in range(3):
            y, dx = torch.empty_like(bases[i]), torch.empty_like(xs[i])
            bank.add_into(xs[i], ids, bases[i], y, stream=stream)
            m.spmm_grad_into(dys[i], dx, stream=stream)
            outs += [y, dx]
        return outs

    want = [go(i) for i in range(2)]
    torch.cuda.synchronize()
    got = []
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            got.append(go(i, s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    m.close()
