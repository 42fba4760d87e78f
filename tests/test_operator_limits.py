"""More of the host side of the adapters', heads' and gradient calls, without a
GPU: which arrays may not overlap."""

import pytest

from fakehip import fake_hip, run  # noqa: F401
from test_operator_calls import BODY

pytest.importorskip("torch")


def _refused(fake_hip, body):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, body]))
    assert out
    wrong = {k: v for k, v in out.items() if v[0] != v[1] or v[2]}
    assert not wrong, wrong


def test_outputs_in_weights_and_ids(fake_hip):  # noqa: F811
    # a of the bank: 4 x 8 x 128 fp16 from 1 << 36 on, b: 4 x 8 x 256 from 1 << 37, four
    # scales from 1 << 38, 40 ids from 1 << 39
    _refused(fake_hip, """
log()
I = -1
A, B, S4 = 1 << 36, 1 << 37, 1 << 38
inside = {"a": A + 4 * 8 * 128 * 2 - 2, "b": B + 64, "scale": S4 + 12, "ids": IDS + 156}
for name, at in inside.items():
    expect("Y in " + name, I, adapt(y=[at]))
    expect("Y and base in " + name, I, adapt(y=[at], base=[at]))
    expect("h in " + name, I, adapt(h=[at // 4 * 4]))
    for out_ in ("dx", "da", "db"):
        expect(out_ + " in " + name, I, grad(**{out_: at // 4 * 4}))
    expect("dx and base in " + name, I, grad(dx=at, base=at))
other = bank(a=1 << 33, b=1 << 34, scale=1 << 35)
for name, at in (("a", 1 << 33), ("b", (1 << 34) + 2), ("scale", (1 << 35) + 4)):
    expect("Y in the other's " + name, I, adapt([bank(), other], y=[at, OUT]))
    expect("h in the other's " + name, I, adapt([bank(), other], h=[at // 4 * 4, H]))
for name, at in (("positions", 1 << 36), ("cosine", (1 << 37) + 64 * 64 * 4 - 4), ("sine", (1 << 38) + 16)):
    expect("a weight's gradient in the " + name, I, rotate_grad([one(dy=Y, w=1 << 35, dw=at)]))
    expect("dx in the " + name, I, rotate_grad([one(dy=Y, y=at)]))
""")


def test_outputs_beside_weights_and_ids(fake_hip):  # noqa: F811
    # right behind an array, or before it, is no overlap
    out = run(fake_hip, "\n".join([BODY, """
A, B, S4 = 1 << 36, 1 << 37, 1 << 38
y, h = 40 * 256 * 2, 40 * 8 * 4
out["statuses"] = [adapt(y=[A + 4 * 8 * 128 * 2]), adapt(y=[A - y]), adapt(y=[S4 + 16]), adapt(y=[IDS + 160]), adapt(y=[IDS - y]),
                   adapt(h=[B + 4 * 8 * 256 * 2]), adapt(h=[IDS - h]), adapt(ids=None, y=[IDS]), adapt(ids=None, h=[IDS]),
                   grad(da=S4 + 16), grad(db=IDS + 160), grad(ids=None, dx=IDS),
                   rotate_grad([one(dy=Y, w=1 << 35, dw=(1 << 36) + 64)])]
"""]))
    assert out["statuses"] == [0] * 13


# rows, cols, share of the values that are kept, tokens; and the form (blocks of 32
# tokens of a wave, groups of 32 columns, groups of tokens) that the calls take by
# themselves on 256 compute units
GRAD_DEFAULTS = [
    (1000, 2056, 0.2, 70, (1, 4, 1)),
    (1003, 1280, 0.2, 1000, (2, 4, 1)),
    (2048, 2048, 0.5, 700, (4, 4, 2)),
    (1536, 6144, 0.25, 16, (1, 8, 1)),
    (2051, 8192, 0.25, 70, (1, 8, 1)),
    (2048, 2048, 0.5, 200, (2, 8, 1)),
    (2051, 8192, 0.25, 500, (2, 8, 1)),
    (1536, 6144, 0.25, 100, (4, 8, 1)),
    (2051, 8192, 0.25, 300, (4, 8, 1)),
    (1536, 6144, 0.25, 1500, (8, 8, 1)),
    (2051, 8192, 0.25, 1500, (8, 8, 1)),
]
# the forms by their place in the table, and matrices sparse enough for each (with rows
# that are 16-byte aligned and rows that are not, the last columns a part of a workgroup's)
GRAD_FORMS = [(1, 4, 1), (2, 4, 1), (4, 4, 1), (4, 4, 2), (1, 8, 1), (2, 8, 1), (4, 8, 1), (8, 8, 1)]
GRAD_SPARSE = [(1000, 1016, 0.2), (803, 616, 0.25), (2056, 328, 0.3)]

GRAD = """
def form(m, n):
    s = S()
    assert L.spdp_spmm_grad_workspace(m._h, n, ctypes.byref(s)) == 0
    log()
    assert L.spdp_spmm_grad(m._h, X, n, Y, WS, s.value, None) == 0
    name = launches()[0][0]
    found = re.match(r"grad_kernelILi(\\d+)ELi(\\d+)ELi(\\d+)ELb(\\d)E", name)
    return [int(v) for v in found.groups()] if found else name
"""


def test_the_gradients_forms_by_default(fake_hip):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, GRAD, f"""
hip.fake_cus(256)
out["got"] = []
for rows, cols, keep, n, _ in {GRAD_DEFAULTS}:
    m = ones(rows, cols, (256, 16), keep)
    out["got"].append(form(m, n))
    m.close()
"""]))
    assert out["got"] == [[*f, int(rows % 8 == 0)] for rows, _, _, _, f in GRAD_DEFAULTS]


@pytest.mark.parametrize("place", range(len(GRAD_FORMS)))
def test_a_forced_form_of_the_gradient_is_the_one_that_runs(fake_hip, place):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, GRAD, f"""
hip.fake_cus(256)
out["got"] = []
for rows, cols, keep in {GRAD_SPARSE}:
    m = ones(rows, cols, (256, 16), keep)
    out["got"] += [form(m, n) for n in (1, 300, 700)]
    m.close()
"""]), env={"SPDP_GRAD_FORM": str(place)})
    assert out["got"] == [[*GRAD_FORMS[place], int(rows % 8 == 0)] for rows, _, _ in GRAD_SPARSE for _ in range(3)]


def test_a_forced_form_that_does_not_fit_is_the_plain_one(fake_hip):  # noqa: F811
    # 256 tokens and 256 columns of a dense matrix: 64 KB of dY and 256 of values
    out = run(fake_hip, "\n".join([BODY, GRAD, """
out["got"] = form(ones(512, 512, (256, 16)), 600)
"""]), env={"SPDP_GRAD_FORM": "7"})
    assert out["got"].startswith("grad_plain")


def test_the_workspace_asked_for_suffices_and_less_is_refused(fake_hip):  # noqa: F811
    out = run(fake_hip, "\n".join([BODY, """
hip.fake_cus(256)
out["wrong"], out["asked"] = [], 0
def check(label, size, call):
    enough = call(size)
    less = call(size - 1) if size else -1
    out["asked"] += size > 0
    if enough != 0 or less != -1:
        out["wrong"].append([label, size, enough, less])
sizes = (1, 31, 64, 65, 512, 513, 1000, 5000, 1 << 20)
for n in sizes:
    for rank in (1, 17, 40, 128):
        for count in (1, 64, 2048):
            for ids in (None, IDS):
                for wide in (1, 16):
                    m = bank(rows=256 * wide, cols=128 * wide, rank=rank, count=count)
                    label = [n, rank, count, bool(ids), wide]
                    for k in (1, 3):
                        check(label + ["adapt", k], need([m] * k, n, ids is not None)[1],
                              lambda room: adapt([m] * k, n=n, ids=ids, room=room, x=[X] * k,
                                                 base=[BASE + (i << 38) for i in range(k)],
                                                 y=[OUT + (i << 38) for i in range(k)]))
                    s = S()
                    assert L.spdp_adapt_grad_workspace(ctypes.byref(m), n, ids is not None, ctypes.byref(s)) == 0
                    check(label + ["grad"], s.value, lambda room: grad(m, n=n, ids=ids, room=room))
for n in sizes:
    for dim, rot in ((128, 128), (512, 2), (34, 6)):
        for k in (1, 2):
            ms = [one(x=X + (i << 40), dy=Y + (i << 42), y=OUT + (i << 41), w=1 << 35, dw=(1 << 34) + 4096 * i, n=1 + 7 * i)
                  for i in range(k)]
            s, r = S(), rotation(dim=dim, rot=rot)
            assert L.spdp_rotate_heads_grad_workspace(heads(*ms), k, ctypes.byref(r), n, ctypes.byref(s)) == 0
            check([n, dim, rot, k], s.value, lambda room: rotate_grad(ms, r, n, room=room))
m = ones(1000, 328, (256, 16), 0.5)
for n in (1, 90, 700, 5000):
    s = S()
    assert L.spdp_spmm_grad_workspace(m._h, n, ctypes.byref(s)) == 0
    check([n, "pruned"], s.value, lambda room: L.spdp_spmm_grad(m._h, X, n, Y, WS, room, None))
"""]))
    assert not out["wrong"], out["wrong"][:5]
    assert out["asked"] > 500
