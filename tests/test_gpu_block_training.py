"""One Transformer block around the Wigner-6j convolution, forward, backward
and the clipping of its gradients, as a training step runs them: norm, q and k
from the scalars, capped attention, convolution with mixing, norm, gate and
residual sum, next norm.  Against float64 with automatic differentiation of
the definitions.  Run with -m gpu."""
import math

import numpy as np
import pytest
import torch

import block_reference as ref
import oracle as o
from cases import TOL_F32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
L, C, H, DK, R, RC, CAP = 2, 16, 4, 8, 8, 5.0, 5.0
K = (L + 1) ** 2


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(L, 0)
    yield c
    c.close()


def harmonics(v):
    rows, one = [torch.ones_like(v[:, :1])], torch.stack([v[:, 1], v[:, 2], v[:, 0]], dim=1)
    for l in range(1, L + 1):
        rows.append(torch.einsum("ea,eb,abc->ec", rows[-1], one, torch.from_numpy(o.cg_real(l - 1, 1, l))))
    return rows


def convolution(pos, feat, i, j, alpha, mix):
    """The layer by its definition, float64, differentiable."""
    sh = harmonics(pos[i] - pos[j])
    a_full = alpha.repeat_interleave(C // H, dim=1)[:, None, :]
    out = []
    for oo in range(L + 1):
        y = torch.zeros(pos.shape[0], 2 * oo + 1, C, dtype=torch.float64)
        for a in range(L + 1):
            for f in range(abs(a - oo), min(a + oo, L) + 1):
                cg = torch.from_numpy(o.cg_real(a, f, oo))
                m = torch.einsum("eac,ef,afo->eoc", feat[j, a * a:(a + 1) ** 2], sh[f], cg) * RC ** -f
                y = y.index_add(0, i, m * a_full)
        out.append(y @ mix[oo].t())
    return torch.cat(out, dim=1)


def reference(p, i, j, g_out, g_normed):
    v = {name: t.double().requires_grad_(True) for name, t in p.items()}
    norm = lambda x, w: x * ((x * x * torch.cat([torch.full((2 * l + 1, 1), 1.0 / ((L + 1) * (2 * l + 1) * C)) for l in range(L + 1)]).double())  # noqa: E731
                             .sum((1, 2), keepdim=True) + 1e-5).rsqrt() * ref.spread(w, L)
    n = v["x"].shape[0]
    n1 = norm(v["x"], v["pre1"])
    q, k = (n1[:, 0] @ v[w] for w in ("wq", "wk"))
    q, k = q.view(n, H, DK), k.view(n, H, DK)
    d = (v["pos"][i] - v["pos"][j]).norm(dim=1)
    z = d[:, None] * ((R - 1) / RC) - torch.arange(R)
    s = CAP * torch.tanh(((q[i] * k[j]).sum(2) * DK ** -0.5 + torch.exp(-z * z) @ v["rbf"].t()) / CAP)
    ex = torch.exp(s)
    alpha = 0.5 * (torch.cos(math.pi * d / RC) + 1)[:, None] * ex / torch.zeros(n, H, dtype=torch.float64).index_add(0, i, ex)[i]
    y = convolution(v["pos"], n1, i, j, alpha, v["mix"])
    out = v["x"] + norm(y, v["post"]) * ref.spread(v["scale"], L) * ref.spread(torch.sigmoid(v["gate"]), L)
    normed = norm(out, v["pre2"])
    ((out * g_out.double()).sum() + (normed * g_normed.double()).sum()).backward()
    return out.detach(), normed.detach(), {name: t.grad for name, t in v.items() if name != "mix"}


def close(got, want, name, tol=TOL_F32):
    err = float((got.cpu().double() - want).abs().max() / want.abs().max())
    print("%s: %.2e" % (name, err))
    assert err <= tol, (name, err)


def test_block_training_step(e2f, ctx):
    n = 40
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    pos = torch.from_numpy(np.random.default_rng(5).uniform(0, 7.5, size=(n, 3)).astype(np.float32))
    rp, ci = (torch.from_numpy(a) for a in o.neighbor_list(pos.numpy(), RC))
    i, j = torch.arange(n).repeat_interleave(rp.diff()), ci.long()
    p = dict(pos=pos, x=r(n, K, C), gate=r(n, L + 1, C), pre1=1 + 0.2 * r(L + 1, C), pre2=1 + 0.2 * r(L + 1, C),
             post=1 + 0.2 * r(L + 1, C), scale=r(L + 1, C), wq=r(C, H * DK) / 4, wk=r(C, H * DK) / 4, rbf=r(H, R),
             mix=r(L + 1, C, C) / 4)
    g_out, g_normed = r(n, K, C), r(n, K, C)
    want_out, want_normed, want = reference(p, i, j, g_out, g_normed)

    d = {name: t.to(DEV) for name, t in p.items()}
    row_ptr, col, go, gn = rp.to(DEV), ci.to(DEV), g_out.to(DEV), g_normed.to(DEV)
    got_rp, got_ci = e2f.e2f_neighbor_list(ctx, d["pos"], RC)
    assert torch.equal(got_rp, row_ptr) and torch.equal(got_ci, col)
    # forward
    _, n1, rstd1 = e2f.e2f_block_norm_forward(ctx, d["x"], L, pre_w=d["pre1"])
    qk = n1[:, 0] @ torch.cat([d["wq"], d["wk"]], dim=1)
    q, k = qk[:, :H * DK].view(n, H, DK), qk[:, H * DK:].view(n, H, DK)
    att = dict(q=q, k=k, rbf_w=d["rbf"], scale=DK ** -0.5, cap=CAP)
    alpha, lse = e2f.e2f_attention_forward(ctx, d["pos"], row_ptr, col, RC, **att)
    y = e2f.e2f_wigner6j_conv_forward(ctx, d["pos"], n1, row_ptr, col, alpha, L, H, RC, mix_w=d["mix"])
    res = dict(block=y, gate=d["gate"], post_w=d["post"], res_scale=d["scale"], pre_w=d["pre2"])
    out, normed, rstd = e2f.e2f_block_norm_forward(ctx, d["x"], L, **res)
    close(out, want_out, "out")
    close(normed, want_normed, "normed")
    # backward
    gx, gy, ggate, gpost, gscale, gpre2 = e2f.e2f_block_norm_backward(ctx, d["x"], rstd, L, grad_out=go,
                                                                      grad_normed=gn, **res)
    gn1, galpha, gpos = e2f.e2f_wigner6j_conv_backward(ctx, d["pos"], n1, gy, row_ptr, col, alpha, L, H, RC,
                                                       mix_w=d["mix"], want_pos=True)
    t = e2f.e2f_transpose_graph(ctx, n, row_ptr, col)
    gq, gk, grbf, gpos2 = e2f.e2f_attention_backward(ctx, d["pos"], row_ptr, col, RC, alpha, lse, galpha, *t, **att)
    gq, gk = gq.view(n, -1), gk.view(n, -1)
    gn1[:, 0] += gq @ d["wq"].t() + gk @ d["wk"].t()
    gx1, _, _, _, _, gpre1 = e2f.e2f_block_norm_backward(ctx, d["x"], rstd1, L, pre_w=d["pre1"], grad_normed=gn1)
    got = dict(pos=gpos + gpos2, x=gx + gx1, gate=ggate, pre1=gpre1, pre2=gpre2, post=gpost, scale=gscale,
               wq=n1[:, 0].t() @ gq, wk=n1[:, 0].t() @ gk, rbf=grbf)
    for name in got:
        close(got[name], want[name], name)
    # clipping of the weights' gradients
    names = ["pre1", "pre2", "post", "scale", "wq", "wk", "rbf"]
    total = math.sqrt(sum(float(want[m].square().sum()) for m in names))
    grads = [got[m].contiguous() for m in names]
    norm = e2f.e2f_clip_grad_norm(ctx, grads, 1.0)
    assert abs(float(norm) - total) <= TOL_F32 * total
    for m, t in zip(names, grads):
        close(t, want[m] / (total + 1e-6), "clipped " + m)
