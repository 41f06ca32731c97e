"""The operators in front of a model's blocks, inside them and behind its backward pass: what is measured of them.

- embedding: the rows of a table by the types of atoms, of edges or of tokens, scaled, as scalars of irrep features
  whose higher degrees are zero; `kind` "train" with the table's gradient, a sum over the atoms of each type;
- layer: the layer norm of irrep features (mean and variance of the scalars, one root mean square of all higher
  degrees) and of plain rows, with the activation of a radial network, and all their gradients;
- ortho: the update of weight matrices from their momentum, orthogonalised by Newton-Schulz steps.

Sizes are those of the benchmark's workloads (a cluster of 32 atoms, 256 molecules of 30 atoms, 20,000 atoms with 25
components of 128 channels, a million edges, mixing matrices of every degree) and generic ones. `exact` takes float64
and derives gradients by automatic differentiation; the plain form writes them out.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5          # of the layer norm
TINY = 1e-7         # added to a matrix's norm
MU = 0.95           # of the momentum
COEF = (3.4445, -4.7750, 2.0315)

_kept = {}


def _context():
    """The package and the context that a program keeps."""
    if not _kept:
        import paper_2501_19216_amd as e2f
        _kept["e2f"], _kept["ctx"] = e2f, e2f.e2f_create(0, 0)
    return _kept["e2f"], _kept["ctx"]


# ------------------------------------------------------------------ cases
def listed():
    a = dict(op="embedding", kind="train", n=32, V=100, C=16, L=2, table="f32", dtype="f32", index="i32", pad=False)
    b = dict(op="layer", kind="train", n=32, L=2, C=16, gap=0, dtype="f32", silu=False)
    c = dict(op="ortho", count=1, batch=3, rows=16, cols=16, steps=5, grad="f32", dtype="f32", moments=True)
    return [
        # the first features of a small cluster in an MD loop: launches and latency
        dict(a, name="embedding_cluster32", kind="forward"),
        # protein scale in training: a few types hold nearly all atoms, 24 of 25 components are zeros
        dict(a, name="embedding_protein20k_train", n=20000, L=4, C=128),
        # a type for every edge of a large graph in training, bfloat16 activations
        dict(a, name="embedding_edges_train", n=1500000, V=100, L=0, C=64, dtype="bf16"),
        # a large vocabulary: sequences of tokens, some padded, both in bfloat16, most tokens rare
        dict(a, name="embedding_tokens_train", n=16384, V=32768, L=0, C=1024, table="bf16", dtype="bf16", index="i64",
             pad=True),
        # the norm of one small cluster
        dict(b, name="layer_cluster32", kind="forward"),
        # protein scale in training
        dict(b, name="layer_protein20k_train", n=20000, L=4, C=128),
        # the radial network's norm and activation on a million edges, bfloat16, columns of a wider projection
        dict(b, name="layer_edges_train", n=1000003, L=0, C=64, gap=64, dtype="bf16", silu=True),
        # long rows of an odd number of channels
        dict(b, name="layer_wide5001_train", n=517, L=0, C=5001),
        # the mixing matrices of one small layer: launches and latency
        dict(c, name="ortho_cluster16"),
        # those of a model of twelve layers with degrees up to 4
        dict(c, name="ortho_mixing128", count=12, batch=5, rows=128, cols=128),
        # odd sizes, tall, bfloat16, the update alone
        dict(c, name="ortho_ragged", count=6, batch=1, rows=517, cols=200, grad="bf16", dtype="bf16", moments=False),
        # wide matrices
        dict(c, name="ortho_wide1024", count=4, batch=1, rows=1024, cols=4096),
    ]


def _cost(c):
    train = 2 if c["kind"] == "train" else 1
    if c["op"] == "embedding":
        return c["n"] * (c["L"] + 1) ** 2 * c["C"] * train + c["V"] * c["C"] + 8 * c["n"]
    return c["n"] * (c["L"] + 1) ** 2 * (c["C"] + c["gap"]) * train


def _flops(c):
    m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    # (the products of a matrix with its transpose are symmetric: one triangle of them)
    return c["count"] * c["batch"] * c["steps"] * (m * (m + 1.0) * n + m * (m + 1.0) * m + 2.0 * m * m * n)


def draw(rng):
    cases = listed()
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        op = rng.choice(["embedding", "layer", "ortho"])
        if op == "embedding":
            c = dict(op=op, kind=rng.choice(["forward", "train", "train"]), n=log(24, 1500000), V=log(3, 40000),
                     C=log(4, 1024), L=rng.choice([0, 0, 0, 1, 2, 3, 4, 6]), table=rng.choice(["f32", "f32", "bf16"]),
                     dtype=rng.choice(["f32", "bf16"]), index=rng.choice(["i32", "i64"]), pad=rng.random() < 0.4)
        elif op == "layer":
            c = dict(op=op, kind=rng.choice(["forward", "train", "train"]), n=log(24, 1500000),
                     L=rng.choice([0, 0, 0, 1, 2, 3, 4, 6]), C=log(3, 8192), gap=rng.choice([0, 0, 5, 64]),
                     dtype=rng.choice(["f32", "bf16"]), silu=rng.random() < 0.5)
            if c["L"]:
                c.update(C=4 * log(1, 64), gap=0, silu=False)
        else:
            dt = rng.choice(["f32", "f32", "bf16"])
            c = dict(op=op, count=log(1, 12), batch=rng.choice([1, 1, 3, 5]), rows=log(3, 2048), cols=log(3, 2048),
                     steps=rng.choice([3, 5, 5, 6]), grad=rng.choice([dt, "f32"]), dtype=dt,
                     moments=rng.random() < 0.6)
            if _flops(c) <= max(_flops(x) for x in cases if x["op"] == op):
                return c
            continue
        if _cost(c) <= max(_cost(x) for x in cases if x["op"] == op):
            return c


def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    c = case
    if c["op"] == "ortho":
        e = c["count"] * c["batch"] * c["rows"] * c["cols"]
        b = e * (_size(c["grad"]) + _size(c["dtype"]))
        if c["moments"]:  # the momentum and the weights, read and written
            b += e * (8 + _size(c["dtype"]))
        return {"bytes": float(b), "flops": _flops(c)}
    train = c["kind"] == "train"
    n, K, C, s = c["n"], (c["L"] + 1) ** 2, c["C"], _size(c["dtype"])
    if c["op"] == "embedding":
        idx = n * (4 if c["index"] == "i32" else 8)
        b = idx + min(n, c["V"]) * C * _size(c["table"]) + n * K * C * s
        if train:
            b += idx + n * C * s + c["V"] * C * _size(c["table"])
        return {"bytes": float(b), "flops": n * C * (2.0 if train else 1.0)}
    e, w = n * K * C, 4 * (c["L"] + 2) * C
    b = 2 * s * e + w
    if train:
        b += 3 * s * e + 2 * w
    return {"bytes": float(b), "flops": e * (20.0 if train else 6.0)}


# ------------------------------------------------------------------ inputs
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, device=DEV, generator=g)  # noqa: E731
    s = {"case": case}
    c = case
    if c["op"] == "embedding":
        n, V, C, L = c["n"], c["V"], c["C"], c["L"]
        if V <= 128:  # types of atoms: five in six are one of the first few, with shares of 1/2, 1/4 ..
            common = (-torch.log2(rand(n).clamp_min(1e-9))).long().clamp_max(V - 1)
            idx = torch.where(rand(n) < 5.0 / 6.0, common, (rand(n) * V).long().clamp_max(V - 1))
        else:         # tokens: as often as one over their rank
            idx = (torch.exp(rand(n) * math.log(V + 1.0)) - 1.0).long().clamp(0, V - 1)
        if c["pad"]:
            idx = torch.where(rand(n) < 0.1, torch.full_like(idx, -1), idx)
        s["index"] = idx.int() if c["index"] == "i32" else idx
        s["table"] = randn(V, C).to(_type(c["table"]))
        if c["kind"] == "train":
            s["g"] = randn(n, (L + 1) ** 2, C).to(_type(c["dtype"])) if L else randn(n, C).to(_type(c["dtype"]))
        return s
    if c["op"] == "layer":
        n, L, C, t = c["n"], c["L"], c["C"], _type(c["dtype"])
        shape = (n, (L + 1) ** 2, C) if L else (n, C + c["gap"])
        x = randn(*shape).mul_(torch.exp(0.5 * randn(n, *[1] * (len(shape) - 1))))
        x += 0.7 * randn(n, *[1] * (len(shape) - 1))
        x = x.to(t)
        s["x"] = x if L else x[:, :C]
        s["w"], s["b"] = (1.0 + 0.2 * randn(L + 1, C), 0.3 * randn(C))
        if c["kind"] == "train":
            s["g"] = randn(*s["x"].shape).to(t)
        return s
    B, r, k = c["batch"], c["rows"], c["cols"]

    def matrices():
        """Gradients of weights: a few strong directions and noise."""
        few = max(1, min(r, k) // 8)
        return [(randn(B, r, few) @ randn(B, few, k)).mul_(few ** -0.5).add_(randn(B, r, k), alpha=0.2).mul_(1e-3)
                for _ in range(c["count"])]
    s["grads"] = [x.to(_type(c["grad"])) for x in matrices()]
    s["outs"] = [torch.empty(B, r, k, dtype=_type(c["dtype"]), device=DEV) for _ in range(c["count"])]
    if c["moments"]:
        s["moments"] = [x.mul_(8.0) for x in matrices()]
        s["news"] = [torch.empty_like(x) for x in s["moments"]]
        s["weights"] = [randn(B, r, k).mul_(k ** -0.5).to(_type(c["dtype"])) for _ in range(c["count"])]
    return s


def _rates(c):
    """What the orthogonal matrix is multiplied with and what the weights are."""
    return (-0.02 * math.sqrt(max(1.0, c["rows"] / c["cols"])), 1.0 - 0.02 * 0.1) if c["moments"] else (1.0, 0.0)


def _scale(c):
    return math.sqrt(c["C"])


# ------------------------------------------------------------------ one pass
def _own_embedding(s):
    e2f, ctx = _context()
    c = s["case"]
    out = {"out": e2f.e2f_embedding_forward(ctx, s["table"], s["index"], lmax=c["L"], scale=_scale(c),
                                            dtype=_type(c["dtype"]))}
    if c["kind"] == "train":
        out["grad_table"] = e2f.e2f_embedding_backward(ctx, s["index"], s["g"], c["V"], lmax=c["L"], scale=_scale(c),
                                                       dtype=_type(c["table"]))
    return out


def _own_layer(s):
    e2f, ctx = _context()
    c = s["case"]
    kw = dict(lmax=c["L"], weight=s["w"], bias=s["b"], eps=EPS, silu=c["silu"])
    got = {"out": e2f.e2f_layer_norm_forward(ctx, s["x"], **kw)}
    if c["kind"] == "train":
        got["grad_x"], got["grad_w"], got["grad_b"] = e2f.e2f_layer_norm_backward(ctx, s["x"], s["g"], **kw)
    return got


def _own_ortho(s):
    e2f, ctx = _context()
    c = s["case"]
    scale, decay = _rates(c)
    e2f.e2f_orthogonalize(ctx, s["grads"], outs=s["outs"], weights=s.get("weights"), moments=s.get("moments"),
                          new_moments=s.get("news"), momentum=MU, nesterov=True, steps=c["steps"], coefs=COEF,
                          scale=scale, decay=decay, eps=TINY)
    return {"outs": s["outs"], "moments": s["news"]} if c["moments"] else {"outs": s["outs"]}


def _plain_embedding(s):
    c = s["case"]
    idx, t = s["index"].long(), _type(c["dtype"])
    there = ((idx >= 0) & (idx < c["V"]))[:, None]
    at = idx.clamp(0, c["V"] - 1)
    rows = torch.where(there, s["table"].float()[at] * _scale(c), 0.0)
    if c["L"]:
        out = torch.zeros(c["n"], (c["L"] + 1) ** 2, c["C"], dtype=t, device=DEV)
        out[:, 0] = rows.to(t)
    else:
        out = rows.to(t)
    if c["kind"] != "train":
        return {"out": out}
    g = (s["g"][:, 0] if c["L"] else s["g"]).float()
    if c["V"] <= 1024:
        # products with truth values, a few thousand rows each, so that no sum of 32 bits is long
        more = -c["n"] % 4096
        one = (torch.nn.functional.pad(idx, (0, more), value=-1)[:, None] == torch.arange(c["V"], device=DEV)).float()
        g = torch.nn.functional.pad(g, (0, 0, 0, more)).view(-1, 4096, c["C"])
        total = torch.matmul(one.view(-1, 4096, c["V"]).transpose(1, 2), g).sum(0)
    else:
        total = torch.zeros(c["V"], c["C"], device=DEV).index_add(0, at, torch.where(there, g, 0.0))
    return {"out": out, "grad_table": (total * _scale(c)).to(s["table"].dtype)}


def _plain_layer(s):
    c = s["case"]
    L, C, n = c["L"], c["C"], c["n"]
    t = s["x"].dtype
    x = s["x"].float().view(n, -1, C) if L else s["x"].float()[:, None, :]
    l = torch.arange((L + 1) ** 2, device=DEV).float().add(0.5).sqrt().long()[1:]
    a = (1.0 / (max(L, 1) * C * (2 * l + 1)))[:, None]
    x0, w0 = x[:, 0], s["w"][0]
    d = x0 - x0.mean(1, keepdim=True)
    r0 = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
    h = d * r0
    z = h * w0 + s["b"]
    gate = 1.0 / (1.0 + torch.exp(-z)) if c["silu"] else None
    y = torch.empty_like(x)
    y[:, 0] = z * gate if c["silu"] else z
    if L:
        x1, w1 = x[:, 1:], s["w"][l]
        r1 = torch.rsqrt((x1 * x1 * a).sum((1, 2), keepdim=True) + EPS)
        y[:, 1:] = x1 * r1 * w1
    got = {"out": y.to(t).view(s["x"].shape)}
    if c["kind"] != "train":
        return got
    g = s["g"].float().view(x.shape)
    g0 = g[:, 0]
    if c["silu"]:
        g0 = g0 * gate * (1.0 + z * (1.0 - gate))
    u = g0 * w0
    gx = torch.empty_like(x)
    gx[:, 0] = r0 * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
    gw = torch.zeros(L + 1, C, device=DEV)
    gw[0] = (g0 * h).sum(0)
    if L:
        u = g[:, 1:] * w1
        gx[:, 1:] = r1 * u - r1 ** 3 * a * x1 * (u * x1).sum((1, 2), keepdim=True)
        gw.index_add_(0, l, (g[:, 1:] * x1 * r1).sum(0))
    got.update(grad_x=gx.to(t).view(s["x"].shape), grad_w=gw, grad_b=g0.sum(0))
    return got


def _plain_ortho(s):
    c = s["case"]
    scale, decay = _rates(c)
    u = torch.cat(s["grads"]).float()
    news = None
    if c["moments"]:
        news = torch.cat(s["moments"]) * MU + u
        u = u + MU * news
    x = u / (u.square().sum((1, 2), keepdim=True).sqrt() + TINY)
    tall = c["rows"] > c["cols"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(c["steps"]):
        p = x @ x.transpose(1, 2)
        x = COEF[0] * x + (COEF[1] * p + COEF[2] * (p @ p)) @ x
    if tall:
        x = x.transpose(1, 2)
    x = scale * x
    if c["moments"]:
        x = x + decay * torch.cat(s["weights"]).float()
    got = {"outs": list(x.to(_type(c["dtype"])).split(c["batch"]))}
    if c["moments"]:
        got["moments"] = list(news.split(c["batch"]))
    return got


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_embedding if op == "embedding" else _own_layer if op == "layer" else _own_ortho)(state)
    return (_plain_embedding if op == "embedding" else _plain_layer if op == "layer" else _plain_ortho)(state)


# ------------------------------------------------------------------ 64 bits
def _exact_embedding(s):
    c = s["case"]
    n, V, C = c["n"], c["V"], c["C"]
    # a row of zeros behind the table, for the indices outside of it
    table = torch.cat([s["table"].double(), torch.zeros(1, C, dtype=torch.float64, device=DEV)])
    idx = s["index"].long()
    idx = torch.where((idx < 0) | (idx >= V), V, idx)
    out = math.sqrt(C) * table.index_select(0, idx)
    got = {"out": torch.nn.functional.pad(out[:, None], (0, 0, 0, (c["L"] + 1) ** 2 - 1)) if c["L"] else out}
    if c["kind"] == "train":
        # sums over the sorted rows: differences of running sums, a block of columns at a time
        order = torch.sort(idx, stable=True).indices
        ends = torch.cumsum(torch.bincount(idx, minlength=V + 1), 0)
        g = s["g"].view(n, -1, C)[:, 0]
        grad = torch.zeros(V, C, dtype=torch.float64, device=DEV)
        for at in range(0, C, 64):
            run = torch.cumsum(g[:, at:at + 64][order].double(), 0)
            run = torch.cat([torch.zeros_like(run[:1]), run])
            grad[:, at:at + 64] = (run[ends[:V]] - run[torch.cat([ends[:1] * 0, ends[:V - 1]])]) * math.sqrt(C)
        got["grad_table"] = grad
    return got


def _exact_layer(s):
    c = s["case"]
    L, C, n = c["L"], c["C"], c["n"]
    train = c["kind"] == "train"
    x, w, b = (v.double().contiguous().requires_grad_(train) for v in (s["x"], s["w"], s["b"]))
    v = x.view(n, (L + 1) ** 2, C)
    var, mean = torch.var_mean(v[:, :1], dim=2, correction=0, keepdim=True)
    y = (v[:, :1] - mean) / (var + EPS).sqrt() * w[:1] + b
    parts = [y * torch.sigmoid(y) if c["silu"] else y]
    if L:
        by = [v[:, l * l:(l + 1) ** 2].square().mean((1, 2)) for l in range(1, L + 1)]
        rms = (sum(by) / L + EPS).sqrt()[:, None, None]
        parts += [v[:, l * l:(l + 1) ** 2] / rms * w[l] for l in range(1, L + 1)]
    out = torch.cat(parts, dim=1).view(x.shape)
    got = {"out": out.detach()}
    if train:
        (out * s["g"].double()).sum().backward()
        got.update(grad_x=x.grad, grad_w=w.grad, grad_b=b.grad)
    return got


def _exact_ortho(s):
    c = s["case"]
    a, b, d = COEF
    scale, decay = _rates(c)
    outs, news = [], []
    for i, g in enumerate(s["grads"]):
        u = g.double()
        if c["moments"]:
            news.append(MU * s["moments"][i].double() + u)
            u = u + MU * news[-1]
        x = u / (torch.linalg.matrix_norm(u)[:, None, None] + TINY)
        for _ in range(c["steps"]):  # on the shorter side's products
            if c["rows"] > c["cols"]:
                p = x.mT @ x
                x = a * x + x @ (b * p + d * p @ p)
            else:
                p = x @ x.mT
                x = a * x + (b * p + d * p @ p) @ x
        outs.append(scale * x + (decay * s["weights"][i].double() if c["moments"] else 0.0))
    return {"outs": outs, "moments": news} if c["moments"] else {"outs": outs}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    return (_exact_embedding if op == "embedding" else _exact_layer if op == "layer" else _exact_ortho)(s)
