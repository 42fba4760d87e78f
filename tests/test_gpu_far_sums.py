"""Long sums of the gradients that are exact in fp32, in any order, so that a head,
a token or a workgroup's share that is missing or met twice shows: the heads'
weight gradients and the adapters' factors', of many tokens and of arrays beyond
the caches and beyond 2^31 numbers."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2607_21985_amd as spdp  # noqa: E402


def _parts(n, width):
    step = max(1, (1 << 27) // width)
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


def _whole(n, width, most, over=1.0):
    """fp16 [n, width] of whole numbers in [-most, most] over `over`."""
    t = torch.empty(n, width, dtype=torch.float16, device="cuda")
    for p in _parts(n, width):
        t[p] = torch.randint(-most, most + 1, t[p].shape, device="cuda", dtype=torch.int8).half() / over
    return t


# tokens, heads of each input, dim (a power of two), rot, interleaved. 16-byte vectors:
# arrays below and beyond 32 MB; pairs and single numbers; more than 2^31 numbers
HEADS = [
    (300, (3, 1), 128, 128, False),
    (2048, (20, 4), 64, 32, True),
    (9001, (20, 3), 128, 96, False),
    (9001, (20, 3), 128, 128, True),
    (20_001, (6, 2), 128, 36, False),
    (20_001, (5,), 8, 6, True),
    (20_001, (5,), 64, 62, False),
    (10_003, (3, 1), 512, 510, False),
    (140_000, (128,), 128, 128, False),
]


@pytest.mark.parametrize("n,heads,dim,rot,interleaved", HEADS)
def test_weight_gradients_of_heads(n, heads, dim, rot, interleaved):
    # numbers of +-1 have a mean square of 1 (dim is a power of two), so that the norm
    # with eps 0 leaves them; quarter turns; dy of quarters up to 1: dw sums multiples of
    # 1/4, some thousands of their root in size, below 2^22
    torch.manual_seed(n + dim)
    turns = torch.randint(0, 4, (50, rot // 2), device="cuda")
    cos = torch.tensor([1.0, 0.0, -1.0, 0.0], device="cuda")[turns]
    sin = torch.tensor([0.0, 1.0, 0.0, -1.0], device="cuda")[turns]
    pos = torch.randint(-2, 53, (n,), device="cuda", dtype=torch.int32)
    inside = (pos >= 0) & (pos < 50)
    xs = [2 * _whole(n, k * dim, 1).abs() - 1 for k in heads]
    dys = [_whole(n, k * dim, 4, 4.0) for k in heads]
    ws = [torch.ones(dim, dtype=torch.float16, device="cuda") for _ in heads]
    dxs, dws = [torch.empty_like(x) for x in xs], [torch.full((dim,), float("nan"), device="cuda") for _ in heads]
    spdp.rotate_heads_grad(xs, dim, pos, cos, sin, dys, dxs, weights=ws, dweights=dws, eps=0.0, interleaved=interleaved)
    i = torch.arange(rot // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    for x, dy, dw, k in zip(xs, dys, dws, heads):
        want = torch.zeros(dim, dtype=torch.float64, device="cuda")
        for p in _parts(n, 4 * k * dim):
            at = inside[p]
            g = dy[p][at].float().reshape(-1, k, dim)
            c, s = cos[pos[p][at].long()][:, None], sin[pos[p][at].long()][:, None]
            a, b = g[..., first], g[..., second]
            g[..., first], g[..., second] = a * c + b * s, b * c - a * s
            want += (g * x[p][at].float().reshape(-1, k, dim)).sum(0, dtype=torch.float64).sum(0)
        assert want.abs().max() < 2.0 ** 22
        assert torch.equal(dw.double(), want)


@pytest.mark.parametrize("n,rows,cols,count,rank,ids", [
    (290_000, 8200, 72, 3, 5, True),   # dY beyond 2^31 numbers
    (60_000, 264, 520, 1, 64, False),
    (5000, 5000, 4000, 2, 20, True),   # dY and x beyond the caches
    (3000, 520, 264, 40, 100, True),
    (500, 1032, 776, 6, 33, True),
])
def test_gradients_of_the_factors(n, rows, cols, count, rank, ids):
    # dY and the factors are -1, 0 or 1, x and h whole numbers up to 2: u is a whole number
    # of some hundreds, and the sums are below 2^24
    torch.manual_seed(n + rank)
    x, dy, base = _whole(n, cols, 2), _whole(n, rows, 1), torch.zeros(n, cols, dtype=torch.float16, device="cuda")
    a, b = (_whole(count * rank, w, 1).reshape(count, rank, w) for w in (cols, rows))
    h = torch.randint(-2, 3, (n, rank), device="cuda").float()
    scale = torch.tensor([0.5, 1.0, -2.0] * count, device="cuda")[:count].contiguous()
    which = torch.randint(-1, count + 1, (n,), device="cuda", dtype=torch.int32) if ids else None
    da, db = torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    spdp.Adapters(a, b, scale).grad_into(x, which, h, dy, base, base, da, db)
    own = which if ids else torch.zeros(n, device="cuda", dtype=torch.int32)
    for i in range(count):
        wa, wb = (torch.zeros(rank, w, dtype=torch.float64, device="cuda") for w in (cols, rows))
        bt = b[i].double().t().contiguous()
        for p in _parts(n, 8 * max(rows, cols)):
            at = own[p] == i
            z = dy[p][at].double()
            u = z @ bt
            wa += u.t().contiguous() @ x[p][at].double()
            wb += h[p][at].double().t().contiguous() @ z
        assert max(wa.abs().max(), wb.abs().max()) < 2.0 ** 24
        assert torch.equal(da[i].double(), float(scale[i]) * wa) and torch.equal(db[i].double(), float(scale[i]) * wb)
