"""The operators of a Transformer block around the Wigner-6j convolution, and of its training step: what is measured
of them.

- attention: the weights of a graph's edges from capped scores with a bias by distance, under a mask by graph, and
  the gradients of the scalar features, the radial weights and the positions (`kind` "forward" is the forward alone,
  "train" the transposed graph, the forward and the backward);
- norm: the norm of a block's output, its gate, scale and residual sum, and the norm before the next block, and all
  their gradients;
- clip: the norm over all gradients of a step and the gradients clipped by it.

Sizes are those of the benchmark's workloads (a cluster of 32 atoms, 256 molecules of 30 atoms, liquid density up to
20,000 atoms, degrees up to 6, 8 heads) and generic ones. `exact` takes float64 and derives gradients by automatic
differentiation; the plain form writes them out.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5      # of the norms
TINY = 1e-6     # added to the gradient norm

_kept = {}


def _context():
    """The package and the context that a program keeps."""
    if not _kept:
        import paper_2501_19216_amd as e2f
        _kept["e2f"], _kept["ctx"] = e2f, e2f.e2f_create(0, 0)
    return _kept["e2f"], _kept["ctx"]


# ------------------------------------------------------------------ cases
def listed():
    a = dict(op="attention", kind="forward", graph="radius", n=32, cutoff=5.0, near=0, H=4, Hk=4, dk=4, R=8, cap=0.0,
             dtype="f32")
    b = dict(op="norm", kind="forward", n=32, L=2, C=16, gate=1, dtype="f32", post=True, pre=True)
    c = dict(op="clip", count=12, total=9000, mixed=False, max_norm=1.0)
    return [
        # one layer of a small cluster in an MD loop: launches and latency
        dict(a, name="attention_cluster32"),
        # a batch of small molecules in training, bfloat16 features, capped scores: short rows
        dict(a, name="attention_molecules_train", kind="train", graph="molecules", n=7680, H=8, Hk=8, dk=16, R=16,
             cap=5.0, dtype="bf16"),
        # ragged: an odd number of atoms, six heads that share two heads of keys, 20 features, 10 radial functions
        dict(a, name="attention_ragged1517_train", kind="train", graph="nearest", near=40, n=1517, cutoff=6.0, H=6,
             Hk=2, dk=20, R=10, cap=20.0),
        # packed graphs of every size in blocks of 500 slots, every pair of a block listed: most pairs masked,
        # the slots without an atom left without any
        dict(a, name="attention_packed4000", graph="packed", near=500, n=4000, cutoff=12.0, H=8, Hk=8, dk=16, R=16,
             cap=20.0),
        # protein scale: the benchmark's headline graph, inference and training
        dict(a, name="attention_protein20k", n=20000, cutoff=6.0, H=8, Hk=8, dk=16, R=32, cap=20.0),
        dict(a, name="attention_protein20k_train", kind="train", n=20000, cutoff=6.0, H=8, Hk=8, dk=16, R=32,
             cap=20.0),
        # the residual sum of one small cluster
        dict(b, name="norm_cluster32"),
        # a batch of molecules in training, a gate for each degree
        dict(b, name="norm_molecules_train", kind="train", n=7680, L=3, C=64, gate=4),
        # protein scale, bfloat16 activations, inference; and float32, training
        dict(b, name="norm_protein20k_bf16", n=20000, L=4, C=128, gate=1, dtype="bf16"),
        dict(b, name="norm_protein20k_train", kind="train", n=20000, L=4, C=128, gate=5),
        # the gradients of one layer, and of a whole model of some 30 million parameters, some of them bfloat16
        dict(c, name="clip_layer"),
        dict(c, name="clip_model33M", count=300, total=33000000, mixed=True),
    ]


def _edges(c):
    n = c["n"]
    if c["graph"] == "packed":
        b = c["near"]
        full, rest = n // b, n % b
        return full * b * (b - 1) + rest * max(rest - 1, 0)
    if c["graph"] == "nearest":
        return n * min(c["near"], n - 1)
    if c["graph"] == "molecules":
        return int(n * min(6.0 * (c["cutoff"] / 5.0) ** 2, 20.0))
    side = (n / 0.1) ** (1.0 / 3.0)  # of the cube, whose faces cut the neighbourhoods of the atoms at them
    return int(n * min(0.7 * (n - 1), 0.1 * 3.98 * c["cutoff"] ** 3 * (1.0 - 0.375 * min(1.0, c["cutoff"] / side)) ** 3))


def _cost(c):
    if c["op"] == "attention":
        return _edges(c) * c["H"] * (c["dk"] + c["R"] + 8) * (3 if c["kind"] == "train" else 1)
    if c["op"] == "norm":
        return c["n"] * (c["L"] + 1) ** 2 * c["C"] * (2 if c["kind"] == "train" else 1)
    return c["total"]


def draw(rng):
    cases = listed()
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        op = rng.choice(["attention", "attention", "norm", "clip"])
        if op == "attention":
            H = rng.choice([1, 2, 4, 6, 8, 8, 12, 16])
            c = dict(op=op, kind=rng.choice(["forward", "train", "train"]),
                     graph=rng.choice(["radius", "molecules", "nearest", "packed"]), n=log(24, 20000),
                     cutoff=rng.randint(256, 448) / 64.0, near=0, H=H,
                     Hk=rng.choice([h for h in range(1, H + 1) if H % h == 0] + [H, H]),
                     dk=rng.choice([3, 4, 8, 12, 16, 16, 20, 32]), R=rng.choice([0, 5, 8, 16, 20, 32, 32]),
                     cap=rng.choice([0.0, 5.0, 20.0, 50.0]), dtype=rng.choice(["f32", "f32", "bf16"]))
            if c["graph"] == "molecules":
                c["n"] = 30 * max(1, c["n"] // 30)
            elif c["graph"] == "nearest":
                c["near"] = min(rng.randint(3, 64), (c["n"] - 1) * 2 // 3)
            elif c["graph"] == "packed":
                c.update(near=log(20, 1000), cutoff=12.0)
        elif op == "norm":
            L = rng.choice([0, 1, 2, 3, 4, 4, 5, 6])
            c = dict(op=op, kind=rng.choice(["forward", "train"]), n=log(24, 30000), L=L,
                     C=4 * log(2, 64 if L else 256), gate=rng.choice([0, 1, L + 1]),
                     dtype=rng.choice(["f32", "bf16"]), post=True, pre=rng.random() < 0.8)
            if rng.random() < 0.15:  # the norm before the first block alone
                c.update(post=False, pre=True, gate=0)
        else:
            count = log(4, 400)
            c = dict(op=op, count=count, total=max(count, log(2000, 33000000)), mixed=rng.random() < 0.5,
                     max_norm=rng.choice([0.1, 1.0, 10.0, 1e6]))
        if _cost(c) <= max(_cost(x) for x in cases if x["op"] == op):
            return c


def work(case):
    c = case
    if c["op"] == "clip":
        b = c["total"] * (3.33 if c["mixed"] else 4.0)  # a third of the tensors has two bytes a value
        return {"bytes": 2.0 * b, "flops": 3.0 * c["total"]}
    train = c["kind"] == "train"
    s = 4 if c["dtype"] == "f32" else 2
    n = c["n"]
    if c["op"] == "norm":
        e = n * (c["L"] + 1) ** 2 * c["C"]
        g, p = n * c["gate"] * c["C"], 4.0 * (c["L"] + 1) * c["C"]
        fwd = (1 + 2 * c["post"] + c["pre"]) * e + g
        if not train:
            return {"bytes": s * fwd + 3 * p, "flops": 12.0 * e}
        # the gradients of what the forward returns, and those of what it takes
        both = fwd + (c["post"] + c["pre"]) * e + (1 + c["post"]) * e + g
        return {"bytes": s * both + 6 * p, "flops": 40.0 * e}
    E, H, R = _edges(c), c["H"], c["R"]
    feat = s * n * (H + c["Hk"]) * c["dk"]
    b = 12.0 * n + feat + 4.0 * H * R + 8.0 * (n + 1) + 4.0 * E + 4.0 * E * H + 4.0 * n * H + 4.0 * n * (c["graph"] == "packed")
    f = E * H * (2.0 * c["dk"] + 2.0 * R + 20) + E * (8.0 * R + 20)
    if train:  # the transposed graph, the weights' gradient, and those of features, radial weights and positions
        b += 8.0 * (n + 1) + 8.0 * E + 4.0 * E * H + feat + 4.0 * H * R + 12.0 * n
        f += E * H * (4.0 * c["dk"] + 4.0 * R + 20) + E * (8.0 * R + 30)
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ inputs
def _lattice(n, g):
    """Positions at liquid density (0.1 atoms per cubic Angstrom) in random index order, [n, 3]."""
    m, a = 1, 10.0 ** (1.0 / 3.0)
    while m ** 3 < n:
        m += 1
    site = torch.randperm(m ** 3, device=DEV, generator=g)[:n]
    ijk = torch.stack([site // (m * m), site // m % m, site % m], dim=1).float()
    return (ijk + 0.5) * a + 0.55 * (2 * torch.rand(n, 3, device=DEV, generator=g) - 1)


def _graph(case, g):
    """Positions, the graph of every atom or None, and the CSR rows."""
    n, kind = case["n"], case["graph"]
    atom = torch.arange(n, device=DEV)
    if kind == "packed":
        # blocks of `near` slots; graphs of 30 atoms on average, one in seven slots without an atom (a graph of its
        # own): every pair of a block is listed
        block = atom // case["near"]
        pos = _lattice(min(n, case["near"]), g).repeat(int(block[-1]) + 1, 1)[:n]
        pos = (pos + 0.05 * torch.randn(n, 3, device=DEV, generator=g)).contiguous()
        alone = torch.rand(n, device=DEV, generator=g) < 1.0 / 7.0
        first = (torch.rand(n, device=DEV, generator=g) < 1.0 / 30.0) | (atom % case["near"] == 0)
        gid = torch.where(alone, n + atom, first.cumsum(0)).int()
    elif kind == "molecules":
        m, per, a = n // 30, 30, 1.9
        t = torch.arange(-4, 5, device=DEV, dtype=torch.float32) * a
        sites = torch.cartesian_prod(t, t, t)
        sites = sites[sites.norm(dim=1) < 6.6]
        pick = torch.rand(m, sites.shape[0], device=DEV, generator=g).topk(per, dim=1).indices
        pos = (sites[pick] + 0.45 * (2 * torch.rand(m, per, 3, device=DEV, generator=g) - 1)).reshape(n, 3).contiguous()
        block, gid = atom // per, None  # (a molecule's rows list its own atoms)
    else:
        pos, block, gid = _lattice(n, g), None, None
    # the closest pairs, as many as _edges() says for every seed: about those within the cutoff
    reach = 1.15 * case["cutoff"] if kind == "radius" and n > 2048 else math.inf
    recv, send, dist = [], [], []
    for s in range(0, n, 1024):
        rows = atom[s:s + 1024]
        d2 = (pos[rows, None, :] - pos[None, :, :]).square().sum(2)
        keep = (rows[:, None] != atom[None, :]) & (d2 < reach ** 2)
        if block is not None:
            keep &= block[rows, None] == block[None, :]
        if kind == "nearest":  # between a half and one and a half times `near`, by the atom's index
            want = case["near"] - case["near"] // 2 + 7 * rows % (2 * (case["near"] // 2) + 1)
            order = d2.masked_fill(~keep, math.inf).argsort(dim=1)[:, :2 * case["near"]]
            few = torch.zeros_like(keep)
            few.scatter_(1, order, torch.arange(order.shape[1], device=DEV)[None, :] < want[:, None])
            keep &= few
        at = keep.nonzero()
        recv.append(at[:, 0] + s)
        send.append(at[:, 1])
        dist.append(d2[keep])
    recv, send, dist = torch.cat(recv), torch.cat(send), torch.cat(dist)
    if kind in ("radius", "molecules"):
        at = dist.argsort(stable=True)[:_edges(case)].sort().values
        recv, send = recv[at], send[at]
    rp = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    rp[1:] = torch.bincount(recv, minlength=n).cumsum(0)
    return pos, gid, rp, send.int()


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _sizes(case):
    """Ragged sizes over four decades that add up to about `total`, every seventeenth 0."""
    r = random.Random(case["count"] * 1000003 + case["total"])
    share = [0.0 if i % 17 == 16 else math.exp(r.uniform(0.0, 9.0)) for i in range(case["count"])]
    return [int(x and max(1, x * case["total"] / sum(share))) for x in share]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    s = {"case": case}
    if case["op"] == "attention":
        n, H, Hk, dk, t = case["n"], case["H"], case["Hk"], case["dk"], _type(case)
        s["pos"], s["gid"], s["rp"], s["ci"] = _graph(case, g)
        qk = (1.5 * randn(n, (H + Hk) * dk)).to(t)  # one projection gives both
        s["q"], s["k"] = qk[:, :H * dk].view(n, H, dk), qk[:, H * dk:].view(n, Hk, dk)
        s["w"] = randn(H, case["R"]) if case["R"] else None
        if case["kind"] == "train":
            s["ga"] = randn(s["ci"].numel(), H)
        return s
    if case["op"] == "norm":
        n, L, C, t = case["n"], case["L"], case["C"], _type(case)
        K = (L + 1) ** 2
        s["x"] = (2.0 * randn(n, K, C) * torch.exp(0.5 * randn(n, 1, 1))).to(t)
        s["block"] = randn(n, K, C).mul_(torch.exp(randn(n, 1, 1))).to(t) if case["post"] else None
        s["gate"] = randn(n, case["gate"], C).to(t) if case["gate"] else None
        s["post_w"], s["scale"] = (1.0 + 0.2 * randn(L + 1, C), 0.5 * randn(L + 1, C)) if case["post"] else (None, None)
        s["pre_w"] = 1.0 + 0.2 * randn(L + 1, C) if case["pre"] else None
        if case["kind"] == "train":
            s["g_out"] = randn(n, K, C).to(t)
            s["g_normed"] = randn(n, K, C).to(t) if case["pre"] else None
        return s
    # the gradients are pieces of one buffer for each type, as a program that sums them over GPUs keeps them: with
    # gaps of a few values between them, which are no gradients and stay as they are
    sizes = _sizes(case)
    low = [case["mixed"] and i % 3 == 2 for i in range(len(sizes))]
    s["flat"], s["grads"], s["outs"] = {}, [None] * len(sizes), [None] * len(sizes)
    for name, t, want in (("f32", torch.float32, False), ("bf16", torch.bfloat16, True)):
        mine = [i for i in range(len(sizes)) if low[i] == want]
        if not mine:
            continue
        buf = randn(sum(sizes[i] + i % 5 for i in mine))
        at = 0
        for i in mine:
            buf[at:at + sizes[i] + i % 5] *= 10.0 ** (-2.0 - i % 3)
            at += sizes[i] + i % 5
        buf = buf.to(t)
        s["flat"][name] = buf.clone()
        at = 0
        for i in mine:
            s["grads"][i], s["outs"][i] = buf[at:at + sizes[i]], s["flat"][name][at:at + sizes[i]]
            at += sizes[i] + i % 5
    return s


# ------------------------------------------------------------------ one pass
def _own_attention(s):
    e2f, ctx = _context()
    c = s["case"]
    kw = dict(q=s["q"], k=s["k"], rbf_w=s["w"], scale=c["dk"] ** -0.5, cap=c["cap"], graph_id=s["gid"])
    alpha, lse = e2f.e2f_attention_forward(ctx, s["pos"], s["rp"], s["ci"], c["cutoff"], **kw)
    out = {"alpha": alpha, "lse": lse}
    if c["kind"] == "train":
        row_t, col_t, perm = e2f.e2f_transpose_graph(ctx, c["n"], s["rp"], s["ci"])
        gq, gk, gw, gp = e2f.e2f_attention_backward(ctx, s["pos"], s["rp"], s["ci"], c["cutoff"], alpha, lse, s["ga"],
                                                    row_t, col_t, perm, **kw)
        out.update(row_t=row_t, col_t=col_t, perm=perm, grad_q=gq, grad_k=gk, grad_w=gw, grad_pos=gp)
    return out


def _own_norm(s):
    e2f, ctx = _context()
    kw = dict(block=s["block"], gate=s["gate"], post_w=s["post_w"], res_scale=s["scale"], pre_w=s["pre_w"], eps=EPS)
    L = s["case"]["L"]
    out, normed, rstd = e2f.e2f_block_norm_forward(ctx, s["x"], L, **kw)
    got = {"out": out if s["case"]["post"] else None, "normed": normed}
    if s["case"]["kind"] == "train":
        names = ("grad_x", "grad_block", "grad_gate", "grad_post_w", "grad_scale", "grad_pre_w")
        got.update(zip(names, e2f.e2f_block_norm_backward(ctx, s["x"], rstd, L, grad_out=s["g_out"],
                                                          grad_normed=s["g_normed"], **kw)))
    return got


def _own_clip(s):
    e2f, ctx = _context()
    norm = e2f.e2f_clip_grad_norm(ctx, s["grads"], s["case"]["max_norm"], outs=s["outs"])
    return {"norm": norm, **s["flat"]}


def _rows(s):
    rp, ci = s["rp"], s["ci"].long()
    return torch.repeat_interleave(rp[1:] - rp[:-1]), ci


def _plain_attention(s):
    c = s["case"]
    n, H, dk, R, cap, rc = c["n"], c["H"], c["dk"], c["R"], c["cap"], c["cutoff"]
    i, j = _rows(s)
    recv, send, E, share = i, j, i.numel(), H // c["Hk"]
    if s["gid"] is not None:  # the edges of one graph alone
        at = (s["gid"][i] == s["gid"][j]).nonzero()[:, 0]
        i, j = i[at], j[at]
    q, k = s["q"].float(), s["k"].float().repeat_interleave(share, dim=1)
    v = s["pos"][i] - s["pos"][j]
    d = v.square().sum(1).sqrt()
    env = torch.where(d < rc, 0.5 * (torch.cos(math.pi / rc * d) + 1.0), 0.0)
    qi, kj = q[i], k[j]
    score = (qi * kj).sum(2) * dk ** -0.5
    if R:
        z = (d[:, None] - torch.arange(R, device=DEV) * (rc / (R - 1))) * ((R - 1) / rc)
        basis = torch.exp(-z * z)
        score = score + basis @ s["w"].t()
    if cap:
        bent = torch.tanh(score / cap)
        score = cap * bent
    rows = i[:, None].expand(-1, H)
    top = torch.full((n, H), -math.inf, device=DEV).scatter_reduce(0, rows, score, "amax")
    p = torch.exp(score - top[i])
    den = torch.zeros(n, H, device=DEV).index_add(0, i, p)
    p = p / den[i]
    lse = top + torch.log(den)
    alpha = env[:, None] * p
    whole = alpha
    if s["gid"] is not None:
        whole = torch.zeros(E, H, device=DEV)
        whole[at] = alpha
    out = {"alpha": whole, "lse": lse}
    if c["kind"] != "train":
        return out
    col, perm = torch.sort(send, stable=True)
    row_t = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    row_t[1:] = torch.bincount(col, minlength=n).cumsum(0)
    ga = s["ga"] if s["gid"] is None else s["ga"][at]
    both = torch.zeros(n, H, device=DEV).index_add(0, i, alpha * ga)
    ds = p * (ga * env[:, None] - both[i])
    if cap:
        ds = ds * (1.0 - bent * bent)
    grad_q = torch.zeros_like(q).index_add(0, i, ds[:, :, None] * kj) * dk ** -0.5
    grad_k = torch.zeros_like(q).index_add(0, j, ds[:, :, None] * qi) * dk ** -0.5
    grad_k = grad_k.reshape(n, c["Hk"], share, dk).sum(2)
    dd = (ga * p).sum(1) * torch.where(d < rc, -0.5 * math.pi / rc * torch.sin(math.pi / rc * d), 0.0)
    grad_w = None
    if R:
        grad_w = ds.t() @ basis
        dd = dd + ((ds @ s["w"]) * basis * z).sum(1) * (-2.0 * (R - 1) / rc)
    f = v * torch.where(d > 0, dd / d, 0.0)[:, None]
    grad_pos = torch.zeros_like(s["pos"]).index_add(0, i, f).index_add(0, j, -f)
    out.update(row_t=row_t, col_t=recv[perm].int(), perm=perm.int(), grad_q=grad_q.to(s["q"].dtype),
               grad_k=grad_k.to(s["k"].dtype), grad_w=grad_w, grad_pos=grad_pos)
    return out


def _degree_of(L):
    """The degree of each of the (L+1)^2 components."""
    return torch.arange((L + 1) ** 2, device=DEV).float().add(0.5).sqrt().long()


def _weights_of(L, C):
    """What each component's square counts in the mean over degrees, [K, 1]."""
    l = _degree_of(L)
    return (1.0 / ((L + 1) * C * (2 * l + 1)))[:, None]


def _by_degree(v, L):
    """Sums over the components of each degree of [K, C]."""
    return torch.zeros(L + 1, v.shape[1], device=DEV).index_add(0, _degree_of(L), v)


def _plain_norm(s):
    c = s["case"]
    L, C = c["L"], c["C"]
    l, a = _degree_of(L), _weights_of(c["L"], c["C"])
    o, nb, got, t = s["x"].float(), None, {}, s["x"].dtype
    if s["block"] is not None:
        b = s["block"].float()
        rb = torch.rsqrt((b * b * a).sum((1, 2), keepdim=True) + EPS)
        nb = b * rb * s["post_w"][l]
        gate = torch.ones_like(nb[:, :1]) if s["gate"] is None else 1.0 / (1.0 + torch.exp(-s["gate"].float()))
        gl = gate if gate.shape[1] == 1 else gate[:, l]
        o = o + s["scale"][l] * gl * nb
        got["out"] = o.to(t)
    if s["pre_w"] is not None:
        ro = torch.rsqrt((o * o * a).sum((1, 2), keepdim=True) + EPS)
        got["normed"] = (o * ro * s["pre_w"][l]).to(t)
    if c["kind"] != "train":
        return got
    do = s["g_out"].float()
    if s["pre_w"] is not None:
        dn = s["g_normed"].float()
        got["grad_pre_w"] = _by_degree((dn * o * ro).sum(0), L)
        dn = dn * s["pre_w"][l]
        do = do + ro * dn - ro ** 3 * a * o * (dn * o).sum((1, 2), keepdim=True)
    got["grad_x"] = do.to(t)
    if s["block"] is not None:
        got["grad_scale"] = _by_degree((do * gl * nb).sum(0), L)
        u = do * s["scale"][l]
        if s["gate"] is not None:
            m = u * nb
            m = m.sum(1, keepdim=True) if gate.shape[1] == 1 else torch.zeros_like(gate).index_add(1, l, m)
            got["grad_gate"] = (m * gate * (1.0 - gate)).to(t)
        u = u * gl
        got["grad_post_w"] = _by_degree((u * b * rb).sum(0), L)
        u = u * s["post_w"][l]
        got["grad_block"] = (rb * u - rb ** 3 * a * b * (u * b).sum((1, 2), keepdim=True)).to(t)
    return got


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    coef = (s["case"]["max_norm"] / (norm + TINY)).clamp(max=1.0).float()
    for g, o in zip(s["grads"], s["outs"]):
        o.copy_(g.float() * coef)
    return {"norm": norm.float(), **s["flat"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_attention if op == "attention" else _own_norm if op == "norm" else _own_clip)(state)
    return (_plain_attention if op == "attention" else _plain_norm if op == "norm" else _plain_clip)(state)


# ------------------------------------------------------------------ 64 bits
def _exact_attention(s):
    c = s["case"]
    n, H, R, rc = c["n"], c["H"], c["R"], c["cutoff"]
    train = c["kind"] == "train"
    leaf = lambda x: None if x is None else x.double().contiguous().requires_grad_(train)  # noqa: E731
    pos, q, k, w = leaf(s["pos"]), leaf(s["q"]), leaf(s["k"]), leaf(s["w"])
    counts = s["rp"].diff()
    i = torch.arange(n, device=DEV).repeat_interleave(counts)
    j = s["ci"].long()
    ok = torch.ones_like(i, dtype=torch.bool) if s["gid"] is None else s["gid"][i] == s["gid"][j]
    i, j = i[ok], j[ok]
    d = (pos[i] - pos[j]).norm(dim=1)
    head = torch.arange(H, device=DEV) // (H // c["Hk"])
    score = torch.zeros(i.numel(), H, dtype=torch.float64, device=DEV)
    for t in range(c["dk"]):  # (a column at a time: the gathered features of every edge are large)
        score = score + q[:, :, t][i] * k[:, head, t][j]
    score = score / math.sqrt(c["dk"])
    if R:
        sigma = rc / (R - 1)
        score = score + torch.exp(-((d[:, None] - sigma * torch.arange(R, device=DEV, dtype=torch.float64)) / sigma) ** 2) @ w.t()
    if c["cap"]:
        score = c["cap"] * torch.tanh(score / c["cap"])
    top = torch.full((n, H), -math.inf, dtype=torch.float64, device=DEV)
    top = top.scatter_reduce(0, i[:, None].expand(-1, H), score.detach(), "amax")
    ex = torch.exp(score - top[i])
    total = torch.zeros(n, H, dtype=torch.float64, device=DEV).index_add(0, i, ex)
    env = torch.where(d < rc, 0.5 * (1.0 + torch.cos(math.pi * d / rc)), torch.zeros_like(d))
    alpha = torch.zeros(s["ci"].numel(), H, dtype=torch.float64, device=DEV)
    alpha = alpha.masked_scatter(ok[:, None].expand(-1, H), env[:, None] * ex / total[i])
    out = {"alpha": alpha.detach(), "lse": (top + total.log()).detach()}
    if train:
        (alpha * s["ga"].double()).sum().backward()
        order = torch.from_numpy(s["ci"].cpu().numpy().argsort(kind="stable")).to(DEV)
        out.update(col_t=torch.arange(n, device=DEV).repeat_interleave(counts)[order].int(), row_t=torch.cat([s["rp"][:1], torch.bincount(s["ci"].long(), minlength=n).cumsum(0)]),
                   perm=order.int(), grad_q=q.grad, grad_k=k.grad,
                   grad_w=None if w is None else w.grad, grad_pos=pos.grad)
    return out


def _exact_norm(s):
    c = s["case"]
    L, C, n = c["L"], c["C"], c["n"]
    train = c["kind"] == "train"
    leaf = lambda x: None if x is None else x.double().requires_grad_(train)  # noqa: E731
    x, b, gate, wp, sc, wn = (leaf(s[name]) for name in ("x", "block", "gate", "post_w", "scale", "pre_w"))
    spread = lambda v: torch.cat([v[..., l:l + 1, :].expand(*v.shape[:-2], 2 * l + 1, C) for l in range(L + 1)], dim=-2)  # noqa: E731

    def normal(v):
        by = [v[:, l * l:(l + 1) ** 2].square().mean((1, 2)) for l in range(L + 1)]
        return v / (sum(by) / (L + 1) + EPS).sqrt()[:, None, None]

    out, got = x, {}
    if b is not None:
        y = normal(b) * spread(wp) * spread(sc)
        if gate is not None:
            open_ = torch.sigmoid(gate)
            y = y * (open_ if gate.shape[1] == 1 else spread(open_))
        out = x + y
        got["out"] = out.detach()
    normed = None
    if wn is not None:
        normed = normal(out) * spread(wn)
        got["normed"] = normed.detach()
    if train:
        loss = (out * s["g_out"].double()).sum()
        if normed is not None:
            loss = loss + (normed * s["g_normed"].double()).sum()
        loss.backward()
        for name, v in (("grad_x", x), ("grad_block", b), ("grad_gate", gate), ("grad_post_w", wp),
                        ("grad_scale", sc), ("grad_pre_w", wn)):
            if v is not None:
                got[name] = v.grad
    return got


def _exact_clip(s):
    total = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    coef = min(1.0, s["case"]["max_norm"] / (math.sqrt(total) + TINY))
    flat = {name: v.double() for name, v in s["flat"].items()}
    for name, v in flat.items():
        at = 0
        for i, g in enumerate(s["grads"]):
            if g.dtype == s["flat"][name].dtype:
                v[at:at + g.numel()] = g.double() * coef
                at += g.numel() + i % 5
    return {"norm": torch.tensor(math.sqrt(total), dtype=torch.float64, device=DEV), **flat}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    return (_exact_attention if op == "attention" else _exact_norm if op == "norm" else _exact_clip)(s)
