"""Timed cases of the operators beside the pruned products.

Around the products of ``perf/cases.py`` a decoder layer needs what these
calls do: low-rank adapters of many requests added to a shared projection
(``Adapters.add_into``, ``adapters_many``), the adapters' gradients
(``Adapters.grad_into``), the gradient of a pruned product with respect to its
input (``Matrix.spmm_grad``), and the norm and position rotation of the heads
of queries and keys (``rotate_heads``, ``rotate_heads_grad``).

With ``own`` false ``run`` computes them with elementary torch operations in
fp32, rounded once at the end; with ``own`` true it makes the package's calls.

A case is a dict of plain values. ``op`` and ``tokens`` are in each, and

* "adapt", "adapt_grad": ``shapes`` (the projections, "ROWSxCOLS" each, that
  read one input), ``adapters`` (how many there are), ``rank``, ``ids``
  ("one": a single adapter for every token; "mixed": any adapter, or none, for
  each token; "runs": consecutive tokens of a request share one), ``keep``
  (return the rank activations that a backward pass reads);
* "spmm_grad": ``shapes`` (one), ``weight_sparsity``;
* "heads", "heads_grad": ``q_heads``, ``k_heads``, ``dim``, ``rot`` (leading
  dimensions of a head that are rotated), ``norm``, ``interleaved`` (pairs are
  neighbours, else the halves), ``positions`` (length of the angle tables).
"""

from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6  # of the heads' norm


def _adapt(name, op, shapes, tokens, adapters, rank, ids, keep=False):
    return {"name": name, "op": op, "shapes": shapes, "tokens": tokens, "adapters": adapters, "rank": rank,
            "ids": ids, "keep": keep}


def _heads(name, op, tokens, q_heads, k_heads, dim, rot, norm, interleaved, positions):
    return {"name": name, "op": op, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "rot": rot,
            "norm": norm, "interleaved": interleaved, "positions": positions}


def _pruned(name, shapes, tokens, weight_sparsity):
    return {"name": name, "op": "spmm_grad", "shapes": shapes, "tokens": tokens, "weight_sparsity": weight_sparsity}


def listed():
    return [
        # one request on a small layer: the fixed cost of a call
        _adapt("adapt 1024, 1 token", "adapt", "1024x1024", 1, 4, 8, "mixed"),
        # a decode step of 32 requests, each with its own adapter of a 7B block's q, k and v
        _adapt("adapt 7B qkv, 32 requests", "adapt", "4096x4096 4096x4096 4096x4096", 32, 32, 16, "mixed"),
        # ragged rows and width, a rank that no vector load fits, tokens without an adapter
        _adapt("adapt 5003x3080, 333", "adapt", "5003x3080", 333, 5, 12, "mixed"),
        # a batch of long prompts on the largest projection
        _adapt("adapt 70B gate, 2048", "adapt", "28672x8192", 2048, 4, 32, "runs"),
        # a training step's forward pass, which keeps what the backward one reads
        _adapt("adapt 7B down, 1000, training", "adapt", "4096x11008", 1000, 1, 64, "one", keep=True),
        # the gradients of a small batch of two adapters trained side by side
        _adapt("adapt gradients 7B q, 256", "adapt_grad", "4096x4096", 256, 2, 16, "runs"),
        # the gradients of an ordinary training batch
        _adapt("adapt gradients 13B gate, 4096", "adapt_grad", "13824x5120", 4096, 1, 64, "one"),
        # the gradient through a pruned projection: a short batch, and an ordinary one
        _pruned("pruned gradient 7B q, 256", "4096x4096", 256, 0.5),
        _pruned("pruned gradient 13B gate, 2048", "13824x5120", 2048, 0.7),
        # a decode step of 8 requests: queries and keys of 70B heads, far positions
        _heads("heads 64+8, 8 tokens", "heads", 8, 64, 8, 128, 128, True, False, 32768),
        # a prompt: rotation alone, as the 7B attention has it
        _heads("heads 32+32, 4096 tokens", "heads", 4096, 32, 32, 128, 128, False, False, 4096),
        # a training batch with the norms' gradients, half of each head rotated
        _heads("heads gradients 40+8, 2048", "heads_grad", 2048, 40, 8, 96, 48, True, True, 2048),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the same ranges: widths mostly multiples of 8, some odd;
    tokens, rows and ranks of any value."""
    op = rng.choice(["adapt", "adapt", "adapt_grad", "spmm_grad", "heads", "heads_grad"])

    def shape(cap):
        while True:
            r, c = _log_int(rng, 512, 28672), _log_int(rng, 512, 28672)
            if r * c <= cap:
                break
        if rng.random() < 0.5:
            r = (r + 127) // 128 * 128
        return r, (c + 7) // 8 * 8 if rng.random() < 0.9 else c

    if op in ("adapt", "adapt_grad"):
        ids = rng.choice(["one", "mixed", "runs"])
        rank = rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 128)])
        adapters = 1 if ids == "one" else _log_int(rng, 1, 64)
        if op == "adapt_grad":
            r, c = shape(70_000_000)
            adapters = min(adapters, 8)
            tokens = _log_int(rng, 32, min(4096, 60_000_000 // (r + c)))
            return _unnamed(_adapt("", op, f"{r}x{c}", tokens, adapters, min(rank, 64), ids))
        decode = rng.random() < 0.5
        tokens = _log_int(rng, 1, 32) if decode else _log_int(rng, 33, 2048)
        count = rng.choice([1, 2, 3]) if decode else 1
        r, c = shape(235_000_000 if decode else 120_000_000)
        while adapters * rank * (r * count + c) > 200_000_000 or (not decode and adapters * rank > 512):
            adapters = (adapters + 1) // 2 if adapters > 1 else adapters
            rank = rank if adapters > 1 else min(rank, 32)
        return _unnamed(_adapt("", op, " ".join([f"{r}x{c}"] * count), tokens, adapters, rank, ids,
                               keep=rng.random() < 0.3))
    if op == "spmm_grad":
        r, c = shape(60_000_000)
        return _unnamed(_pruned("", f"{r}x{c}", _log_int(rng, 16, 2048), rng.choice([0.5, 0.6, 0.7, 0.8])))
    dim = rng.choice([64, 80, 96, 128, 128, 256, 2 * rng.randint(8, 128)])
    rot = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
    k_heads = rng.choice([1, 2, 4, 8])
    q_heads = k_heads * rng.choice([1, 2, 4, 5, 8])
    tokens = _log_int(rng, 1, min(4096, 4096 * 64 * 128 // ((q_heads + k_heads) * dim)))
    return _unnamed(_heads("", op, tokens, q_heads, k_heads, dim, rot, rng.random() < 0.6, rng.random() < 0.3,
                           rng.choice([4096, 32768])))


def _unnamed(case):
    del case["name"]
    return case


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split()]


def _activations(tokens, cols, gen):
    """Attention inputs: Laplace with 1 % outlier channels."""
    u = torch.rand((tokens, cols), device="cuda", generator=gen) - 0.5
    x = -torch.sign(u) * torch.log1p(-2.0 * u.abs().clamp(max=0.4999999))
    outliers = torch.randperm(cols, device="cuda", generator=gen)[: max(1, cols // 100)]
    x[:, outliers] *= 20.0
    return x.half()


def _gradients(shape, gen):
    """Gradients as a scaled loss gives them: tokens of very different size."""
    size = 0.01 * torch.exp(torch.randn((shape[0],) + (1,) * (len(shape) - 1), device="cuda", generator=gen))
    return (size * torch.randn(shape, device="cuda", generator=gen)).half()


def _ids(case, gen):
    """Each token's adapter, -1 for none; None: adapter 0 for all."""
    n, count = case["tokens"], case["adapters"]
    if case["ids"] == "one":
        return None
    if case["ids"] == "mixed":
        i = torch.randint(0, count, (n,), device="cuda", generator=gen, dtype=torch.int32)
        none = torch.rand(n, device="cuda", generator=gen) < (0.1 if n > 1 else 0.0)
        return torch.where(none, torch.full_like(i, -1), i)
    # requests of some ten to some hundred tokens behind one another
    ends = torch.rand(n, device="cuda", generator=gen) < min(1.0, max(count, 2) / n)
    which = torch.randint(0, count, (n,), device="cuda", generator=gen, dtype=torch.int32)
    return which[torch.cumsum(ends.int(), 0).clamp(max=n - 1)].contiguous()


def prepare(case, seed):
    """Inputs, weights and outputs on the GPU, all from the seed; with ``own``
    the handles that a user's program holds."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 29)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    n, op = case["tokens"], case["op"]
    st = {"case": case}
    if op in ("adapt", "adapt_grad"):
        shapes, k, r = _shapes(case), case["adapters"], case["rank"]
        cols = shapes[0][1]
        st["x"] = _activations(n, cols, gen)
        st["ids"] = _ids(case, gen)
        st["a"] = [(randn(k, r, cols) / math.sqrt(cols)).half() for _ in shapes]
        st["b"] = [(0.02 * randn(k, r, rows)).half() for rows, _ in shapes]  # rank by rank: B transposed
        st["scale"] = [torch.exp(0.5 * randn(k)) for _ in shapes]
        if op == "adapt":
            st["base"] = [randn(n, rows).half() for rows, _ in shapes]
        else:
            st["dy"] = _gradients((n, shapes[0][0]), gen)
            st["base"] = [_gradients((n, cols), gen)]
            st["h"] = _rank_activations(st["x"], st["a"][0], st["ids"])[1]
        if own:
            import paper_2607_21985_amd as spdp
            st["banks"] = [spdp.Adapters(a, b, s) for a, b, s in zip(st["a"], st["b"], st["scale"])]
    elif op == "spmm_grad":
        (rows, cols), s = _shapes(case)[0], case["weight_sparsity"]
        w = 0.02 * randn(rows, cols) * torch.exp(0.5 * randn(cols))
        some = w.reshape(-1)[:: max(1, rows * cols // 1_000_003)].abs().sort().values
        st["w"] = w.masked_fill_(w.abs() < some[int(s * (some.numel() - 1))], 0.0).half()
        st["dy"] = _gradients((n, rows), gen)
        if own:
            import paper_2607_21985_amd as spdp
            st["m"] = spdp.encode(st["w"].cpu().numpy(), (256, 16))
    else:
        d, rot = case["dim"], case["rot"]
        heads = (case["q_heads"], case["k_heads"])
        st["x"] = [randn(n, h * d).half() for h in heads]
        st["w"] = [(1.0 + 0.2 * randn(d)).half() if case["norm"] else None for _ in heads]
        angle = torch.arange(case["positions"], device="cuda", dtype=torch.float64)[:, None] * torch.exp(
            -math.log(1e4) * torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        if n <= 64:  # requests at places of their own
            st["pos"] = torch.randint(0, case["positions"], (n,), device="cuda", generator=gen, dtype=torch.int32)
        else:
            st["pos"] = (torch.arange(n, device="cuda") % case["positions"]).int()
        if op == "heads_grad":
            st["dy"] = [_gradients((n, h * d), gen) for h in heads]
    return st


def _rank_activations(x, a, ids):
    """fp32 [tokens, adapters, rank] of each token's own adapter, the others'
    0, and their sum over the adapters."""
    k, r, cols = a.shape
    h = (x.float() @ a.reshape(k * r, cols).float().t()).reshape(-1, k, r)
    if ids is not None:
        h = torch.where((ids[:, None] == torch.arange(k, device=x.device))[:, :, None], h, torch.zeros_like(h))
    return h, h.sum(1)


def _add(base, h, scale, b):
    k, r, rows = b.shape
    y = (h * scale[:, None]).reshape(-1, k * r) @ b.reshape(k * r, rows).float()
    return (base.float() + y).half()


def _rank_gradient(t, h, scale):
    """fp32 [adapters, rank, features]: scale of the adapter times the sum over
    the tokens of h and t."""
    n, k, r = h.shape
    return (h * scale[:, None]).reshape(n, k * r).t().contiguous().matmul(t.float()).reshape(k, r, -1)


def _rotate(v, cos, sin, interleaved, back):
    """v [tokens, heads, dim]; pairs (2 i, 2 i + 1), or (i, i + rot / 2)."""
    half = cos.shape[1]
    c, s = cos[:, None], -sin[:, None] if back else sin[:, None]
    lead, rest = v[..., :2 * half], v[..., 2 * half:]
    p, q = (lead[..., 0::2], lead[..., 1::2]) if interleaved else (lead[..., :half], lead[..., half:])
    p, q = p * c - q * s, q * c + p * s
    lead = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((lead, rest), -1)


def _heads_plain(x, w, cos, sin, case):
    v = x.float().reshape(x.shape[0], -1, case["dim"])
    if w is not None:
        v = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _rotate(v, cos, sin, case["interleaved"], False).reshape(x.shape).half()


def _heads_grad_plain(x, w, dy, cos, sin, case):
    v = x.float().reshape(x.shape[0], -1, case["dim"])
    g = _rotate(dy.float().reshape(v.shape), cos, sin, case["interleaved"], True)
    if w is None:
        return g.reshape(x.shape).half(), None
    r = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    dw = (g * v * r).sum((0, 1))
    g = g * w.float()
    return (r * (g - v * (r * r * (g * v).mean(-1, keepdim=True)))).reshape(x.shape).half(), dw


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        import paper_2607_21985_amd as spdp
    if op == "adapt":
        x, ids = state["x"], state["ids"]
        if own:
            ys = [torch.empty_like(b) for b in state["base"]]
            hs = [torch.empty((x.shape[0], case["rank"]), dtype=torch.float32, device=x.device) for _ in ys] \
                if case["keep"] else None
            if len(ys) == 1:
                state["banks"][0].add_into(x, ids, state["base"][0], ys[0], h=hs[0] if hs else None)
            else:
                spdp.adapters_many(state["banks"], [x] * len(ys), ids, state["base"], ys, hs=hs)
            return ys + (hs or [])
        hs = [_rank_activations(x, a, ids) for a in state["a"]]
        ys = [_add(p, h[0], s, b) for p, h, s, b in zip(state["base"], hs, state["scale"], state["b"])]
        return ys + ([h[1] for h in hs] if case["keep"] else [])
    if op == "adapt_grad":
        x, ids, dy, a, b, scale = state["x"], state["ids"], state["dy"], state["a"][0], state["b"][0], state["scale"][0]
        if own:
            dx, da, db = torch.empty_like(x), torch.empty_like(a, dtype=torch.float32), torch.empty_like(b, dtype=torch.float32)
            state["banks"][0].grad_into(x, ids, state["h"], dy, state["base"][0], dx, da, db)
            return [dx, da, db]
        u = _rank_activations(dy, b, ids)[0]
        hit = torch.ones_like(u[:, :, :1]) if ids is None else \
            (ids[:, None] == torch.arange(a.shape[0], device=x.device)).float()[:, :, None]
        return [_add(state["base"][0], u, scale, a), _rank_gradient(x, u, scale),
                _rank_gradient(dy, state["h"][:, None] * hit, scale)]
    if op == "spmm_grad":
        if own:
            return state["m"].spmm_grad(state["dy"])
        return (state["dy"].float() @ state["w"].float()).half()
    qk, w, pos, cos, sin = state["x"], state["w"], state["pos"], state["cos"], state["sin"]
    d, rot = case["dim"], {"interleaved": case["interleaved"]}
    if op == "heads":
        if own:
            ys = [torch.empty_like(x) for x in qk]
            spdp.rotate_heads(qk, d, pos, cos, sin, ys, weights=w, eps=EPS, **rot)
            return ys
        c, s = cos[pos.long()], sin[pos.long()]
        return [_heads_plain(x, v, c, s, case) for x, v in zip(qk, w)]
    if own:
        dx = [torch.empty_like(x) for x in qk]
        dw = [torch.empty(d, dtype=torch.float32, device=x.device) for x in qk] if case["norm"] else None
        spdp.rotate_heads_grad(qk, d, pos, cos, sin, state["dy"], dx, weights=w, dweights=dw, eps=EPS, **rot)
        return [dx, dw or []]
    c, s = cos[pos.long()], sin[pos.long()]
    got = [_heads_grad_plain(x, v, g, c, s, case) for x, v, g in zip(qk, w, state["dy"])]
    return [[g[0] for g in got], [g[1] for g in got if g[1] is not None]]


def work(case):
    """Bytes: every input and output once (of the adapters those that tokens
    have; of a pruned matrix its bitmap and nonzeros). Flops: two per product
    that meets; of the heads' the norm's and the rotation's."""
    n, op = case["tokens"], case["op"]
    if op in ("adapt", "adapt_grad"):
        k, r = case["adapters"], case["rank"]
        met = min(k, n)
        if op == "adapt":
            cols = _shapes(case)[0][1]
            by = 2.0 * n * cols + sum(4.0 * n * m + 2.0 * met * r * (m + cols) for m, _ in _shapes(case))
            return {"bytes": by + (4.0 * n * r * len(_shapes(case)) if case["keep"] else 0.0),
                    "flops": sum(2.0 * n * r * (m + cols) for m, _ in _shapes(case))}
        m, cols = _shapes(case)[0]
        return {"bytes": 2.0 * n * (3 * cols + m) + 4.0 * n * r + 2.0 * met * r * (m + cols) + 4.0 * k * r * (m + cols),
                "flops": 4.0 * n * r * (m + cols)}
    if op == "spmm_grad":
        m, cols = _shapes(case)[0]
        nnz = (1.0 - case["weight_sparsity"]) * m * cols
        return {"bytes": 2.0 * nnz + m * cols / 8.0 + 2.0 * n * (m + cols), "flops": 2.0 * nnz * n}
    e = 1.0 * n * (case["q_heads"] + case["k_heads"]) * case["dim"]
    tables = 4.0 * min(n, case["positions"]) * case["rot"]
    back = op == "heads_grad"
    return {"bytes": (6.0 if back and case["norm"] else 4.0) * e + tables,
            "flops": e * (3.0 + (5.0 if case["norm"] else 0.0)) * (2.0 if back else 1.0)}


def _exact_low_rank(x, a, b, scale, ids, base):
    """base + scale B (A x) token by token's adapter, and A x."""
    y, h = base.double(), torch.zeros((x.shape[0], a.shape[1]), dtype=torch.float64, device=x.device)
    for i in range(a.shape[0]):
        at = torch.arange(x.shape[0], device=x.device) if ids is None else torch.nonzero(ids == i).flatten()
        if at.numel() == 0 or (ids is None and i > 0):
            continue
        h[at] = x[at].double() @ a[i].double().t()
        y[at] += float(scale[i]) * (h[at] @ b[i].double())
    return y, h


def _exact_heads(x, w, dy, st, case):
    """The rotated heads by complex numbers, or the gradients by those."""
    d, half = case["dim"], case["rot"] // 2
    v = x.double().reshape(x.shape[0], -1, d)
    turn = torch.complex(st["cos"].double(), st["sin"].double())[st["pos"].long()][:, None]
    i = torch.arange(half, device=x.device)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)

    def turned(t, by):
        z = torch.complex(t[..., first], t[..., second]) * by
        t = t.clone()
        t[..., first], t[..., second] = z.real, z.imag
        return t

    rms = torch.sqrt((v * v).sum(-1, keepdim=True) / d + EPS)
    if dy is None:
        return turned(v if w is None else v / rms * w.double(), turn).reshape(x.shape)
    g = turned(dy.double().reshape(v.shape), turn.conj())
    if w is None:
        return g.reshape(x.shape), None
    n = v / rms
    gw = g * w.double()
    return ((gw - n * (gw * n).sum(-1, keepdim=True) / d) / rms).reshape(x.shape), (g * n).sum((0, 1))


def exact(case, seed):
    global own
    mine, own = own, False
    st = prepare(case, seed)
    own = mine
    op = case["op"]
    if op == "adapt":
        got = [_exact_low_rank(st["x"], a, b, s, st["ids"], p) for a, b, s, p in zip(st["a"], st["b"], st["scale"], st["base"])]
        return [g[0] for g in got] + ([g[1] for g in got] if case["keep"] else [])
    if op == "adapt_grad":
        x, dy, a, b, scale, ids = st["x"], st["dy"], st["a"][0], st["b"][0], st["scale"][0], st["ids"]
        dx, u = _exact_low_rank(dy, b, a, scale, ids, st["base"][0])
        da, db = torch.zeros_like(a, dtype=torch.float64), torch.zeros_like(b, dtype=torch.float64)
        for i in range(a.shape[0]):
            at = slice(None) if ids is None else torch.nonzero(ids == i).flatten()
            if ids is None and i > 0:
                continue
            da[i] = float(scale[i]) * (u[at].t().contiguous() @ x[at].double())
            db[i] = float(scale[i]) * (st["h"][at].double().t().contiguous() @ dy[at].double())
        return [dx, da, db]
    if op == "spmm_grad":
        return torch.cat([part.double() @ st["w"].double() for part in st["dy"].split(512)])
    if op == "heads":
        return [_exact_heads(x, w, None, st, case) for x, w in zip(st["x"], st["w"])]
    got = [_exact_heads(x, w, g, st, case) for x, w, g in zip(st["x"], st["w"], st["dy"])]
    return [[g[0] for g in got], [g[1] for g in got if g[1] is not None]]
