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
