"""Float64 forms of embedding, layer norm and orthogonalised updates on the CPU, with bounds of what float32 arithmetic
may add.  U = 2^-24 is half a step of a float32; every bound counts roundings times the absolute values of what is
summed."""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check(got, want, name):
    """|got - value| <= bound, elementwise, and the rounding to got's type."""
    value, bound = want
    got = got.detach().cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    room = bound + (bound + value.abs()) * (half_step(got.dtype) if got.dtype != torch.float32 else 0.0) + 1e-37
    off = (got.double() - value).abs()
    bad = ~(off <= room)
    assert not bad.any(), (name, int(bad.sum()), float((off / room).nan_to_num(math.inf).max()))


# ------------------------------------------------------------------ embedding
def float32(scale):
    """The C interface's scale is a float."""
    return float(torch.tensor(scale, dtype=torch.float32))


def embedding(table, index, K, scale):
    scale = float32(scale)
    V, C = table.shape
    idx = index.long()
    there = (idx >= 0) & (idx < V)
    out = torch.zeros(idx.shape[0], K, C, dtype=torch.float64)
    out[there, 0] = table.double()[idx[there]] * scale
    return out, 1.01 * U * out.abs()


def embedding_grad(g, index, V, scale):
    """g [n, C]: the scalars' gradients."""
    scale = float32(scale)
    idx = index.long()
    there = (idx >= 0) & (idx < V)
    at, rows = idx[there], g.double()[there]
    zero = torch.zeros(V, g.shape[1], dtype=torch.float64)
    value, size = zero.index_add(0, at, rows), zero.index_add(0, at, rows.abs())
    # a stretch of up to 64 sorted rows one after the other, up to 256 such parts of a workgroup in their order, the workgroups'
    # sums in up to 1024 strides and 10 halvings, the scale; never more than the rows there are, and those last ones
    k = torch.bincount(at, minlength=V).double()[:, None]
    count = k.clamp_max(64 + 256) + k / 1024 + 20
    return value * scale, U * count * size * abs(scale)


# ------------------------------------------------------------------ layer norm
def degrees(L):
    return torch.cat([torch.full((2 * l + 1,), l) for l in range(L + 1)])


def layer_norm(x, L, w=None, b=None, eps=1e-5, silu=False, g=None):
    """{name: (value, bound)} for x [n, K, C] (K = (L+1)^2), with g of the backward; values by automatic
    differentiation, bounds from the formulas' terms."""
    n, K, C = x.shape
    l = degrees(L)
    x = x.double().requires_grad_(True)
    w = (torch.ones(L + 1, C) if w is None else w).double().requires_grad_(True)
    b = (torch.zeros(C) if b is None else b).double().requires_grad_(True)
    x0 = x[:, 0]
    m = x0.mean(1, keepdim=True)
    d = x0 - m
    var = d.square().mean(1, keepdim=True)
    r0 = (var + eps).rsqrt()
    h = d * r0
    z = h * w[0] + b
    q = torch.sigmoid(z)
    parts = [(z * q if silu else z)[:, None]]
    if L:
        a = (1.0 / (L * C * (2 * l[1:] + 1)))[:, None].double()
        x1 = x[:, 1:]
        r1 = ((x1 * x1 * a).sum((1, 2), keepdim=True) + eps).rsqrt()
        parts.append(x1 * r1 * w[l[1:]])
    y = torch.cat(parts, dim=1)
    out = {}
    with torch.no_grad():
        # a sum over a row: up to 32 values of a thread (200 above the scalars), 6 exchanges, 8 waves
        D, D1 = 48, 220
        em = U * D * x0.abs().mean(1, keepdim=True)
        ed = em + 2 * U * (d.abs() + em)
        evar = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + U * (D + 2) * var
        er = (0.5 * evar / (var + eps) + 4 * U)  # relative
        eh = r0 * ed + h.abs() * (er + 2 * U)
        ez = w[0].abs() * eh + 2 * U * ((h * w[0]).abs() + z.abs())
        # the sigmoid's slope is at most 1/4, that of z sigma(z) 1.1, of its slope 1/2; the exponential and quotient 8 roundings
        ey = 1.1 * ez + 12 * U * (z * q).abs() if silu else ez
        bounds = [ey[:, None]]
        if L:
            bounds.append(U * (D1 / 2 + 8) * parts[1].abs())
        out["out"] = (y.detach(), torch.cat(bounds, dim=1))
    if g is None:
        return out
    g = g.double()
    (y * g).sum().backward()
    with torch.no_grad():
        slope = q * (1 + z * (1 - q)) if silu else torch.ones_like(z)
        dz = g[:, 0] * slope
        # (terms of the slope: q and q z (1 - q), 8 roundings of the exponential each and those of their sum)
        edz = g[:, 0].abs() * (0.5 * ez + 24 * U * q * (1 + (z * (1 - q)).abs())) if silu else torch.zeros_like(dz)
        u = dz * w[0]
        eu = edz * w[0].abs() + U * u.abs()
        mu, muh = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
        emu = eu.mean(1, keepdim=True) + U * D * u.abs().mean(1, keepdim=True)
        emuh = ((h.abs() + eh) * eu + u.abs() * eh).mean(1, keepdim=True) + (U * (D + 6) + er) * (u * h).abs().mean(1, keepdim=True)
        size = r0 * (u.abs() + mu.abs() + (h * muh).abs())
        egx = [(r0 * (eu + emu + (h.abs() + eh) * emuh + muh.abs() * eh) + (er + 6 * U) * size)[:, None]]
        # sums over rows: those of a thread, 6 exchanges, 16 rows of a workgroup; then float64
        R = min(n, 32 + n // 64)
        dzh, ew, ebs = (dz * h).abs(), (dz.abs() + edz) * eh + edz * h.abs(), edz
        egw = [ew.sum(0) + U * (R + 30) * dzh.sum(0)]
        if L:
            u1 = g[:, 1:] * w[l[1:]]
            s = (u1 * x1).abs().sum((1, 2), keepdim=True)
            egx.append(U * (2 * D1 + 20) * (r1 * u1.abs() + r1 ** 3 * a * x1.abs() * s))
            t = (g[:, 1:] * x1 * r1).abs().sum(0)
            egw += [U * (R + D1) * t[k * k - 1:(k + 1) ** 2 - 1].sum(0) for k in range(1, L + 1)]
        out["grad_x"] = (x.grad, torch.cat(egx, dim=1))
        out["grad_w"] = (w.grad, torch.stack(egw))
        out["grad_b"] = (b.grad, ebs.sum(0) + U * (R + 30) * dz.abs().sum(0))
    return out


# ------------------------------------------------------------------ orthogonalised updates
MUON = (3.4445, -4.7750, 2.0315)


def orthogonalize(g, moment=None, weight=None, momentum=0.95, nesterov=True, coefs=(MUON,) * 5, scale=1.0, decay=0.0,
                  eps=1e-7):
    """(out, new moment, X, room): float64, for one matrix; room: of X's error in the Frobenius norm.

    A step X -> p(X) takes an error of X by at most the largest |p'| up to the largest singular value (the divided differences of
    the odd p).  Each step adds its own: operands of 22 bits and sums of float, 2^-22 of each entry's share, which
    over a matrix of r rows with singular values up to s add up as independent errors to 2^-22 (|b| s^2 + 2 |c| s^4 + |a|) s sqrt(r)
    or so: 4 times that is allowed."""
    u = g.double()
    new = None
    if moment is not None:
        # (the momentum as it is stored)
        new = momentum * moment.double() + u
        u = u + momentum * new if nesterov else new
    x = u / (u.norm() + eps)
    r = min(x.shape)
    grid = torch.linspace(0, 1, 2001, dtype=torch.float64)
    room = 4 * U * float(x.norm())
    for a, b, c in coefs:
        if x.shape[0] <= x.shape[1]:
            p = x @ x.T
            y = a * x + (b * p + c * p @ p) @ x
        else:
            p = x.T @ x
            y = a * x + x @ (b * p + c * p @ p)
        s = float(torch.linalg.matrix_norm(x, 2)) if r else 0.0
        t = grid * s
        lip = float((a + 3 * b * t ** 2 + 5 * c * t ** 4).abs().max())
        own = 4 * 2.0 ** -22 * (abs(a) + abs(b) * s ** 2 + 2 * abs(c) * s ** 4) * s * math.sqrt(r)
        room = lip * room + own
        x = y
    out = scale * x
    if weight is not None and decay:
        out = out + decay * weight.double()
    return out, new, x, room
