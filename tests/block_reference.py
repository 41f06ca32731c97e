"""Plain float64 forms of the operators around the convolution (capped
attention, block norms, gradient clipping) on the CPU, with bounds on what
float32 arithmetic may add to each value.  Gradients come from automatic
differentiation of the definitions; the bounds from the formulas' terms: u =
2^-24 is half a step of a float32, and every bound counts roundings times the
absolute values of what is summed."""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ attention
def attention(pos, rp, ci, rc, q=None, k=None, w=None, heads=None, scale=1.0, cap=0.0, gid=None, ga=None):
    """{name: (value, bound)} of e2f_attention_forward, and with ga of the backward, for CPU tensors of any type."""
    f64 = lambda t: None if t is None else t.detach().double().contiguous().requires_grad_(True)  # noqa: E731
    pos, q, k, w = f64(pos), f64(q), f64(k), f64(w)
    n = pos.shape[0]
    H = heads or (q.shape[1] if q is not None else w.shape[0])
    i = torch.arange(n).repeat_interleave(rp[1:] - rp[:-1])
    j = ci.long()
    ok = torch.ones_like(i, dtype=torch.bool) if gid is None else gid[i] == gid[j]
    E, at = i.numel(), ok.nonzero()[:, 0]
    i, j = i[ok], j[ok]
    v = pos[i] - pos[j]
    d2 = v.square().sum(1)
    d = torch.where(d2 > 0, d2.clamp_min(1e-300).sqrt(), torch.zeros_like(d2))  # (no gradient at 0)
    x = torch.zeros(i.numel(), H, dtype=torch.float64)
    # roundings of a score: the product's terms and their sum, the distance (differences of positions up to
    # 4 u d, the root 1), which z takes (R - 1) / rc times, the exponential's argument and value
    bx = torch.zeros_like(x)
    if q is not None:
        dk, share = q.shape[2], H // k.shape[1]
        kj = k.repeat_interleave(share, dim=1)[j]
        x = x + scale * (q[i] * kj).sum(2)
        bx = bx + U * (dk + 3) * abs(scale) * (q[i] * kj).abs().sum(2)
    if w is not None:
        R = w.shape[1]
        z = d[:, None] * ((R - 1) / rc) - torch.arange(R)
        g = torch.exp(-z * z)
        x = x + g @ w.t()
        bz = U * 10 * (d[:, None] * ((R - 1) / rc) + torch.arange(R))
        bg = (2 * z.abs() * bz + U * (3 * z * z + 4)) * g + 1e-38
        bx = bx + bg @ w.abs().t() + U * (R + 1) * (g @ w.abs().t())
    b = bx.detach()
    t = torch.zeros_like(x)
    s, bs = x, b
    if cap:
        t = torch.tanh(x / cap)
        s = cap * t
        # tanh contracts; its own value and argument add a few steps of it
        bs = b + U * 8 * s.abs()
    m = torch.full((n, H), -math.inf, dtype=torch.float64)
    m = m.scatter_reduce(0, i[:, None].expand(-1, H), s.detach(), "amax")
    ex = torch.exp(s - m[i])
    den = torch.zeros(n, H, dtype=torch.float64).index_add(0, i, ex)
    deg = torch.bincount(i, minlength=n).double()[:, None]
    p = ex / den[i]
    env = torch.where(d < rc, 0.5 * (torch.cos(math.pi / rc * d) + 1.0), torch.zeros_like(d))
    alpha = torch.zeros(E, H, dtype=torch.float64).index_add(0, at, env[:, None] * p)
    lse = m + den.log()
    # a row's scores shift its sum by at most the largest of their errors; its terms and their sum, and
    # exponents up to |s - lse|
    bs = bs.detach()
    worst = torch.zeros(n, H, dtype=torch.float64).scatter_reduce(0, i[:, None].expand(-1, H), bs, "amax")
    blse = worst + U * (deg + 8) + U * 4 * lse.detach().abs()
    rel = bs + blse[i] + U * (8 + 4 * (s.detach() - lse.detach()[i]).abs())
    # the envelope: its cosine's argument is a distance over the cutoff
    benv = torch.where(d < rc * (1 + 1e-5), U * 16, 0.0).detach()
    balpha = (env[:, None] * p * rel).detach() + benv[:, None] * p.detach() + 1e-37
    out = {"alpha": (alpha.detach(), torch.zeros(E, H, dtype=torch.float64).index_add(0, at, balpha)),
           "lse": (lse.detach(), blse)}
    if ga is None:
        return out
    ga = ga.double()
    leaves = [a for a in (q, k, w, pos) if a is not None]
    use = torch.where(ok[:, None], ga, torch.zeros_like(ga))  # (what a masked edge holds does not count)
    grads = dict(zip([id(a) for a in leaves],
                     torch.autograd.grad((alpha * use).sum(), leaves, allow_unused=True)))
    zero = lambda a: torch.zeros_like(a) if grads[id(a)] is None else grads[id(a)]  # noqa: E731
    with torch.no_grad():
        g_e, a_e, e_ = ga[at], (env[:, None] * p), env[:, None]
        D = torch.zeros(n, H, dtype=torch.float64).index_add(0, i, a_e * g_e)
        bD = torch.zeros(n, H, dtype=torch.float64).index_add(0, i, g_e.abs() * (balpha + U * (deg[i] + 2) * a_e))
        turn = 1 - t * t
        bturn = 2 * t.abs() * (b / cap if cap else 0.0) + U * 12
        core = (g_e * e_ - D[i])
        bcore = g_e.abs() * (benv[:, None] + U * 4 * e_) + bD[i] + U * 2 * core.abs()
        ds = p * core * turn
        bds = p * (core.abs() * (turn * (rel + U * 4) + bturn) + bcore * (turn + bturn)) + 1e-37
        if q is not None:
            bq = scale * torch.zeros_like(q).index_add(0, i, (bds + U * (deg[i] + 4) * ds.abs())[:, :, None] * kj.abs())
            degt = torch.bincount(j, minlength=n).double()[:, None]
            bk = scale * torch.zeros_like(q).index_add(0, j, (bds + U * (share * degt[j] + 4) * ds.abs())[:, :, None] * q[i].abs())
            bk = bk.reshape(n, k.shape[1], share, dk).sum(2)
            out["grad_q"], out["grad_k"] = (zero(q), bq.abs()), (zero(k), bk.abs())
        slope = torch.where(d < rc, -0.5 * math.pi / rc * torch.sin(math.pi / rc * d), torch.zeros_like(d))
        bdd = (g_e.abs() * p * (rel + U * 8)).sum(1) * slope.abs() + (g_e.abs() * p).sum(1) * U * 16 * math.pi / rc
        mag = (g_e.abs() * p).sum(1) * slope.abs()
        if w is not None:
            # up to E terms in one chain at worst
            out["grad_w"] = (zero(w), bds.t() @ g + ds.abs().t() @ bg + U * (i.numel() / 16 + 64) * (ds.abs().t() @ g))
            lean = 2 * (R - 1) / rc
            uw = ds.abs() @ w.abs()
            buw = bds @ w.abs() + U * (H + 2) * uw
            mag = mag + lean * (uw * z.abs() * g).sum(1)
            bdd = bdd + lean * (buw * z.abs() * g + uw * (bz * g + z.abs() * bg) + U * (R + 4) * uw * z.abs() * g).sum(1)
        bdd = bdd + U * (H + 6) * mag
        bf = bdd + U * 8 * mag
        bpos = torch.zeros(n, dtype=torch.float64).index_add(0, i, bf).index_add(0, j, bf)
        sums = torch.zeros(n, dtype=torch.float64).index_add(0, i, mag).index_add(0, j, mag)
        count = torch.bincount(i, minlength=n) + torch.bincount(j, minlength=n)
        out["grad_pos"] = (zero(pos), (bpos + U * (count + 4) * sums)[:, None].expand(-1, 3))
    return out


def check(got, ref, dtype=torch.float32, name=""):
    """got within the reference's bound and the output type's own rounding, elementwise; what is not finite alike."""
    value, bound = ref
    got = got.detach().cpu().double()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    fine = torch.isfinite(value)
    assert torch.equal(fine, torch.isfinite(got)), name
    assert torch.equal(got[~fine & ~value.isnan()], value[~fine & ~value.isnan()]), name
    room = bound + half_step(dtype) * (value.abs() + bound)
    over = ((got - value).abs() / room.clamp_min(1e-300))[fine]
    worst = float(over.max()) if over.numel() else 0.0
    print("%s: %.3f of the bound" % (name, worst))
    assert worst <= 1.0, (name, worst)


# ------------------------------------------------------------------ norms
def spread(v, L):
    return torch.cat([v[..., l:l + 1, :].expand(*v.shape[:-2], 2 * l + 1, v.shape[-1]) for l in range(L + 1)], dim=-2)


def block_norm(x, L, block=None, gate=None, post_w=None, res_scale=None, pre_w=None, eps=1e-5, g_out=None,
               g_normed=None, grads=False):
    """{name: (value, bound)} of e2f_block_norm_forward, and with grads of the backward; x [n, (L+1)^2, C]."""
    f64 = lambda t: None if t is None else t.detach().cpu().double().requires_grad_(True)  # noqa: E731
    x, block, gate, post_w, res_scale, pre_w = map(f64, (x, block, gate, post_w, res_scale, pre_w))
    g_out, g_normed = (None if g is None else g.detach().cpu().double() for g in (g_out, g_normed))
    n, K, C = x.shape
    a = torch.cat([torch.full((2 * l + 1, 1), 1.0 / ((L + 1) * (2 * l + 1) * C)) for l in range(L + 1)]).double()
    rnorm = lambda v: ((v * v * a).sum((1, 2), keepdim=True) + eps).rsqrt()  # noqa: E731
    y, rb = torch.zeros_like(x), torch.ones(n, 1, 1, dtype=torch.float64)
    S = torch.ones(K, C, dtype=torch.float64) if res_scale is None else spread(res_scale, L)
    P = torch.ones(K, C, dtype=torch.float64) if post_w is None else spread(post_w, L)
    G = torch.ones(n, 1, C, dtype=torch.float64)
    if gate is not None:
        G = torch.sigmoid(gate) if gate.shape[1] == 1 else spread(torch.sigmoid(gate), L)
    if block is not None:
        if post_w is not None:
            rb = rnorm(block)
        y = S * G * P * block * rb
    out = x + y
    # a norm: up to 4 K terms a thread, ten sums across threads, root and quotient; the sigmoid and products
    c = 4 * K + 40
    ref = {}
    bo = U * (c * y.abs() + out.abs()).detach()
    if block is not None:
        ref["out"] = (out.detach(), bo)
    ro = torch.ones(n, 1, 1, dtype=torch.float64)
    if pre_w is not None:
        W = spread(pre_w, L)
        ro = rnorm(out)
        normed = out * ro * W
        # the norm moves by at most as much as the largest relative shift of out in the root mean square
        shift = (bo.square() * a).sum((1, 2), keepdim=True).sqrt() * ro
        brel = (shift + U * c).detach()
        ref["normed"] = (normed.detach(), (ro * W.abs() * bo).detach() + normed.abs().detach() * brel)
    ref["rstd"] = (torch.cat([rb, ro], dim=1)[:, :, 0].detach(),
                   torch.cat([rb * U * c, ro * (U * c + (shift if pre_w is not None else 0.0))], dim=1)[:, :, 0].detach())
    if not grads:
        return ref
    loss = torch.zeros((), dtype=torch.float64)
    if g_out is not None:
        loss = loss + (out * g_out).sum()
    if g_normed is not None:
        loss = loss + (normed * g_normed).sum()
    leaves = [(name, t) for name, t in (("grad_x", x), ("grad_block", block), ("grad_gate", gate),
                                        ("grad_post_w", post_w), ("grad_scale", res_scale), ("grad_pre_w", pre_w))
              if t is not None]
    got = torch.autograd.grad(loss, [t for _, t in leaves], allow_unused=True) if loss.requires_grad else [None] * 6
    got = {name: torch.zeros_like(t) if g is None else g for (name, t), g in zip(leaves, got)}
    with torch.no_grad():
        c = 2 * c + 40
        by_degree = lambda v: torch.stack([v[l * l:(l + 1) ** 2].sum(0) for l in range(L + 1)])  # noqa: E731
        ab = (g_out.abs() if g_out is not None else torch.zeros_like(x)) + 0.0
        bt = U * ab
        if g_normed is not None:
            wd = (W * g_normed).abs()
            inner = (wd * (out.abs() + y.abs())).sum((1, 2), keepdim=True)
            second = ro ** 3 * a * (out.abs() + y.abs()) * inner
            first = ro * wd
            ab = ab + first + second
            bt = bt + (first + 3 * second) * (U * c + 3 * brel) + ro ** 3 * a * (bo * inner + out.abs() * (wd * bo).sum((1, 2), keepdim=True))
            terms = (g_normed.abs() * (out.abs() + y.abs()) * ro).sum(0)
            extra = (g_normed.abs() * ro * (out.abs() * brel + bo)).sum(0)
            # n rows: at most n / 8 in a thread's chain, then float64
            ref["grad_pre_w"] = (got["grad_pre_w"], by_degree(terms * U * (c + n / 8) + extra))
        elif pre_w is not None:
            ref["grad_pre_w"] = (got["grad_pre_w"], torch.zeros_like(pre_w))
        ref["grad_x"] = (got["grad_x"], bt)
        if block is not None:
            sa = (S * G * P).abs()
            u, bu = ab * sa, bt * sa + U * c * ab * sa
            inner, binner = (u * block.abs()).sum((1, 2), keepdim=True), (bu * block.abs()).sum((1, 2), keepdim=True)
            normed_term = rb ** 3 * a * block.abs() if post_w is not None else torch.zeros_like(block)
            ref["grad_block"] = (got["grad_block"], rb * (bu + U * c * u) + normed_term * (binner + U * c * inner))
            dot, bdot = ab * block.abs() * rb, (bt + U * c * ab) * block.abs() * rb
            if post_w is not None:
                ref["grad_post_w"] = (got["grad_post_w"], by_degree(((bdot + U * (n / 8) * dot) * (S * G).abs()).sum(0)))
            if res_scale is not None:
                ref["grad_scale"] = (got["grad_scale"], by_degree(((bdot + U * (n / 8) * dot) * (P * G).abs()).sum(0)))
            if gate is not None:
                # 1 - sigmoid loses its digits where the gate is open: to within u of 1
                each = (bdot + U * c * dot) * (S * P * G * (1 - G)).abs() + U * 4 * dot * (S * P * G).abs()
                if gate.shape[1] == 1:
                    each = each.sum(1, keepdim=True)
                else:
                    each = torch.stack([each[:, l * l:(l + 1) ** 2].sum(1) for l in range(L + 1)], dim=1)
                ref["grad_gate"] = (got["grad_gate"], each)
    return ref
