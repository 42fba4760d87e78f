"""The binding of the adapters', heads' and gradient calls, without a GPU: which
tensors reach the library (its entry points are recorded, and tensors of host
memory pass for a GPU's)."""

import pytest

torch = pytest.importorskip("torch")

import paper_2607_21985_amd as spdp  # noqa: E402


class _Library:
    """Records the calls; each succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    rec = _Library()
    monkeypatch.setattr(spdp, "lib", lambda: rec)
    monkeypatch.setattr(spdp, "_stream", lambda stream, tensors: 0)
    return rec


def _half(*shape):
    return torch.zeros(shape, dtype=torch.float16)


COUNT, RANK, COLS, ROWS, TOKENS = 4, 8, 8, 24, 5


def _calls(bank):
    """Every call that reads the bank's weights."""
    x, base, ids = _half(TOKENS, COLS), _half(TOKENS, ROWS), torch.zeros(TOKENS, dtype=torch.int32)
    h = torch.zeros(TOKENS, RANK)
    da, db = torch.zeros(COUNT, RANK, COLS), torch.zeros(COUNT, RANK, ROWS)
    yield lambda: bank.add_into(x, ids, base, torch.empty_like(base))
    yield lambda: bank(x, ids, base)
    yield lambda: spdp.adapters_many([bank], [x], None, [base], [torch.empty_like(base)], hs=[h])
    yield lambda: bank.grad_into(x, ids, h, base, x, torch.empty_like(x), da, db)


# replacements at the address of the weights that they replace
SAME_ADDRESS = {
    "fewer adapters": (lambda b: ("a", b.a[:2]), ValueError),
    "fewer ranks": (lambda b: ("a", b.a[:, :4]), ValueError),
    "fewer rows": (lambda b: ("b", b.b[:, :, :8]), ValueError),
    "fewer scales": (lambda b: ("scale", b.scale[:3]), ValueError),
    "another order": (lambda b: ("a", b.a.transpose(1, 2)), ValueError),  # (as many ranks as columns)
    "broadcast scales": (lambda b: ("scale", b.scale[:1].expand(COUNT)), ValueError),
    "another type": (lambda b: ("a", b.a.view(torch.bfloat16)), TypeError),
    "whole numbers": (lambda b: ("scale", b.scale.view(torch.int32)), TypeError),
}


@pytest.mark.parametrize("how", SAME_ADDRESS)
def test_replaced_weights_are_looked_at(library, how):
    change, error = SAME_ADDRESS[how]
    for k in range(4):
        bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
        call = list(_calls(bank))[k]
        call()
        name, new = change(bank)
        assert new.data_ptr() == getattr(bank, name).data_ptr()
        setattr(bank, name, new)
        library.calls.clear()
        with pytest.raises(error):
            call()
        assert not library.calls


def test_weights_whose_memory_is_replaced_are_looked_at(library):
    bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
    bank.b.data = bank.b.data[:1]
    for call in _calls(bank):
        library.calls.clear()
        with pytest.raises(ValueError):
            call()
        assert not library.calls


def test_gradients_have_the_banks_own_shapes(library):
    # the shapes that the kernels write, whatever the weights' are by now
    bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
    x, dy, h = _half(TOKENS, COLS), _half(TOKENS, ROWS), torch.zeros(TOKENS, RANK)
    bank.a = bank.a[:2]
    library.calls.clear()
    with pytest.raises(ValueError, match="da"):
        bank.grad_into(x, None, h, dy, x, torch.empty_like(x), torch.zeros(2, RANK, COLS), torch.zeros(COUNT, RANK, ROWS))
    assert not library.calls


def test_weights_of_the_same_form_may_be_replaced(library):
    bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
    bank.a, bank.scale = bank.a.clone(), bank.scale + 1
    bank.b.data = bank.b.data.clone()
    for call in _calls(bank):
        library.calls.clear()
        call()
        assert library.calls


class _Graph:
    replays = 0

    def replay(self):
        _Graph.replays += 1


@pytest.fixture
def graphs(library, monkeypatch):
    """torch's streams and graphs stand still; the chain's own calls are recorded."""
    import contextlib

    class Stream:
        def __init__(self, device=None):
            pass

        def wait_stream(self, other):
            pass

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: Stream())
    monkeypatch.setattr(torch.cuda, "synchronize", lambda dev=None: None)
    monkeypatch.setattr(torch.cuda, "CUDAGraph", _Graph)
    monkeypatch.setattr(torch.cuda, "graph", lambda g, stream=None: contextlib.nullcontext())
    _Graph.replays = 0
    return library


def _chain():
    bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
    weight, tables = _half(8), (torch.zeros(TOKENS, dtype=torch.int32), torch.zeros(9, 4), torch.zeros(9, 4))
    y = _half(TOKENS, ROWS)
    ch = spdp.Chain().add_adapters(bank, _half(TOKENS, COLS), None, y, y)
    return ch.add_heads([y], 8, *tables, [y], weights=[weight]), bank, weight


def _new_data(t):
    t.data = t.data.clone()


REPLACED = {
    "a": lambda bank, weight: setattr(bank, "a", bank.a.clone()),
    "b's memory": lambda bank, weight: _new_data(bank.b),
    "scale": lambda bank, weight: setattr(bank, "scale", bank.scale * 2),
    "the norm's memory": lambda bank, weight: _new_data(weight),
}


@pytest.mark.parametrize("what", REPLACED)
def test_a_chain_notices_replaced_weights(graphs, what):
    ch, bank, weight = _chain()
    ch.capture()
    ch.replay()
    old = [t.data_ptr() for t in (bank.a, bank.b, bank.scale, weight)]
    REPLACED[what](bank, weight)
    for _ in range(2):
        with pytest.raises(RuntimeError, match="captur"):
            ch.replay()
    assert _Graph.replays == 1
    # the captured memory is not handed out again while the graph is there
    assert [t.data_ptr() for t in ch._alive] == old
    ch.capture()
    ch.replay()
    assert _Graph.replays == 2


def test_a_chain_replays_weights_rewritten_in_place(graphs):
    ch, bank, weight = _chain()
    ch.capture()
    bank.a += 1
    bank.scale.mul_(2)
    weight += 1
    ch.replay()
    assert _Graph.replays == 1


def test_a_chain_refuses_weights_of_another_form(graphs):
    ch, bank, _ = _chain()
    ch.capture()
    bank.a = bank.a[:2]  # at the same address
    with pytest.raises(ValueError):
        ch.replay()
    assert _Graph.replays == 0


@pytest.fixture
def streams(library, monkeypatch):
    """Which stream each tensor was taken on, by address, and the streams that
    were recorded for it; "caller" is the current one."""
    import contextlib
    state = {"current": "caller", "taken": {}, "recorded": {}}

    @contextlib.contextmanager
    def on(stream):
        state["current"], before = stream, state["current"]
        yield
        state["current"] = before

    empty, empty_like = torch.empty, torch.empty_like

    def taken(t):
        state["taken"][t.data_ptr()] = state["current"]
        return t

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: state["current"])
    monkeypatch.setattr(torch, "empty", lambda *a, **k: taken(empty(*a, **k)))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: taken(empty_like(*a, **k)))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: state["recorded"].setdefault(t.data_ptr(), []).append(s))
    return state


def _matrix():
    m = spdp.Matrix.__new__(spdp.Matrix)
    m._h, m.rows, m.cols, m.device = None, ROWS, COLS, 0
    return m


VALUES = {
    "adapters": lambda bank, m, s: bank(_half(TOKENS, COLS), None, _half(TOKENS, ROWS), stream=s),
    "pruned gradient": lambda bank, m, s: m.spmm_grad(_half(TOKENS, ROWS), stream=s),
}


@pytest.mark.parametrize("what", VALUES)
def test_results_belong_to_the_calls_stream(streams, what):
    bank = spdp.Adapters(_half(COUNT, RANK, COLS), _half(COUNT, RANK, ROWS), torch.zeros(COUNT))
    m = _matrix()
    out = VALUES[what](bank, m, "side")
    assert out.dtype == torch.float16 and tuple(out.shape) == (TOKENS, COLS if what == "pruned gradient" else ROWS)
    assert streams["taken"][out.data_ptr()] == "side"
    assert streams["recorded"][out.data_ptr()] == ["caller"]
    streams["recorded"].clear()
    out = VALUES[what](bank, m, None)
    assert streams["taken"][out.data_ptr()] == "caller" and not streams["recorded"]


@pytest.mark.parametrize("call", [lambda m, s: m.spmm(_half(TOKENS, COLS), stream=s),
                                  lambda m, s: m(_half(TOKENS, COLS), 0.5, stream=s)])
def test_products_belong_to_the_calls_stream(streams, monkeypatch, call):
    into = []
    monkeypatch.setattr(spdp.Matrix, "spmm_into", lambda self, x, y, stream=None: into.append((y, stream)))
    monkeypatch.setattr(spdp.Matrix, "spmspv_into", lambda self, x, t, y, stream=None, mask="token": into.append((y, stream)))
    out = call(_matrix(), "side")
    assert into == [(out, "side")] and tuple(out.shape) == (TOKENS, ROWS)
    assert streams["taken"][out.data_ptr()] == "side" and streams["recorded"][out.data_ptr()] == ["caller"]
    assert streams["taken"][call(_matrix(), None).data_ptr()] == "caller"
